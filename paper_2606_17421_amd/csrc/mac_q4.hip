// ct x pt MAC over 4-bit weights with one scale (and zero point) per group of
// inputs on the gfx950 matrix cores, exact.
//
// Per limb l, with u the 4-bit weights, z the zero points (8 without them) and
// S = rint(scale Delta) of the group,
//     out[j][col] = sum_g S[j][g] T[j][g][col] mod q_l,
//     T[j][g][col] = sum over the group of (u[j][i] - z[j][g]) x[i][col].
// T needs only the small integers u - z, one int8 digit and the same for every limb, against
// the residues' four balanced base-256 digits: four int8 products a modular MAC (the scalar
// weights' own digits take 12 or 16).  The scale enters once a group, in 64-bit
// integers: T = a + 2^16 b with a and b from two digits each, and the sum over g of
// (S mod q) a + (2^16 S mod q) b is reduced once an output.
//
// What bounds the large layers: issue, for four fifths of the cycles.  Beside each 32-cycle v_mfma_i32_32x32x32_i8
// run a shift-add and a 64-bit multiply-add for every output of a sub-group and digit pair (4 vector
// operations a matrix operation at groups of 128, 8 at 64, 16 at 32), the unpacking (1.5) and
// the closing reduction (1.2 at 768 inputs); at about 4.3 cycles each (8.8 the multiply-add), and
// 8.5 issue cycles a matrix operation, they take longer than the matrix pipe, which is busy 52% of
// the cycles at 768 -> 3072 (groups of 128, N = 2^15, 6 limbs: 3.70 to 3.78 ms, 1.0e15 int8 products/s), and
// the chip holds 1.7 GHz under both (2.05 GHz and the same cycles with zero residues).  The other fifth is
// waiting: for a row group's stores (contract()) and for the fill of a strip, at 2^14 and 4 limbs 79 of the 370 us of
// 768 -> 768, with the matrix cores idle.  At a few hundred inputs and outputs of wide batches these two
// weigh most: 256 -> 512 at 2^16 and 4 limbs takes 734 us, more than its products at the large layers' rate (277) and
// its bytes (340) one after the other.  Measured without effect: contractions and combinations interleaved by hand, fragments
// read ahead, three or four waves a SIMD with half the rows, 64-byte stores after a transpose over
// lanes.  One combination for two sub-groups that share a scale (groups of 256 and more) gave 1-3%,
// int8 fragments instead of 4-bit ones 4% for twice the memory; touching the next strip's lines before the
// last rows cost 5%.
#include <type_traits>

#include "digits.hpp"

namespace ckks {
namespace {

constexpr int kThreads = 256;        // encode kernels
constexpr uint32_t kStep = 32;       // inputs of one matrix-core step
constexpr uint32_t kCols = 32;       // columns of a workgroup
constexpr uint32_t kPadRows = 64;    // output rows are padded to this: two tiles a wave (one-tile waves contract the padding's zeros)
constexpr int kStepFrags = 4 * 64;   // 16-byte residue fragments of a step: four digits, 64 lanes
constexpr uint32_t kFold = 1024;     // most inputs between reductions of the 64-bit sums

// Encoded weights (written once a layer by two short kernels, the launches of which are most of their time: 8 to 9 us for
// 768 -> 768 and smaller, 17 us for 1024 -> 6144 at 8 limbs, whose bytes take 2):
//   fragments [tile][step][64 lanes] of row tile*32 + lane%32 and inputs step*32 + 16
//     (lane/32) + i, i < 16; rows are padded to kPadRows, steps to whole sub-groups.
//     Without zero points 8 bytes: v = u - 8 in four bits, two's complement.  Word d holds i =
//     8d .. 8d + 7: the low halves of its bytes the first four, the high halves the last four, so
//     two masks give four bytes 16 v each.
//     With zero points 16 bytes, 8 (u - z) each: u - z does not fit four bits, and to subtract z
//     from unpacked bytes takes three operations more a word (3072 -> 768 at 2^14, groups of
//     64: 1.97 ms with 4-bit u, 1.79 ms so).
//   scales [limb][tile][sub-group][32 rows] of {sa, sb}: sa = 2^32 S / 16, sb = 2^48 S / 16 mod q_l
//     (/ 8 with zero points), centred.  The 2^32 is what the closing reduction divides by.
// A sub-group is what one set of i32 sums covers: 128, 96 or 64 inputs that divide
// the group (768 -> 768 at 2^14, 4 limbs, groups of 96: 394 us, as 32 + 32 + 32 548), else 32; a group that holds every input is cut freely.
struct Shape {
  uint32_t tiles, steps, groups, sub_len, subs;
  size_t frag_bytes, scale_bytes;
};

Shape shape_of(uint32_t d_out, uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros) {
  Shape s;
  s.tiles = (d_out + kPadRows - 1) / kPadRows * (kPadRows / 32);
  s.groups = (d_in - 1) / group + 1;  // a group may end past 2^32
  if (s.groups == 1)
    s.sub_len = d_in <= 32 ? 32 : d_in <= 64 ? 64 : d_in <= 96 ? 96 : 128;
  else
    s.sub_len = group % 128 == 0 ? 128 : group % 96 == 0 ? 96 : group % 64 == 0 ? 64 : 32;
  s.subs = (d_in + s.sub_len - 1) / s.sub_len;
  s.steps = s.subs * (s.sub_len / kStep);
  s.frag_bytes = static_cast<size_t>(s.tiles) * s.steps * 64 * (zeros ? 16 : 8);
  s.scale_bytes = static_cast<size_t>(limbs) * s.tiles * s.subs * 32 * 8;
  return s;
}

// A lane's weight fragment.
template <bool kZeros>
using Frag = std::conditional_t<kZeros, v4i, uint2>;

template <bool kZeros>
__global__ __launch_bounds__(kThreads) void q4_frag_kernel(const uint8_t* __restrict__ w4,
                                                           const uint8_t* __restrict__ zeros, uint32_t d_out,
                                                           uint32_t d_in, uint32_t group, uint32_t groups,
                                                           uint32_t steps, size_t lanes, size_t group0,
                                                           Frag<kZeros>* __restrict__ frag) {
  const size_t idx = (group0 + blockIdx.x) * kThreads + threadIdx.x;
  if (idx >= lanes) return;
  const uint32_t lane = idx & 63;
  const uint32_t step = static_cast<uint32_t>((idx >> 6) % steps), tile = static_cast<uint32_t>((idx >> 6) / steps);
  const uint32_t row = tile * 32 + (lane & 31), k0 = step * kStep + 16 * (lane >> 5);
  const uint8_t* w = w4 + static_cast<size_t>(row) * ((d_in + 1) / 2);
  // past the layer's edges the weight is zero: u = z
  uint32_t z = 8;
  if (kZeros && row < d_out && k0 < d_in) z = zeros[static_cast<size_t>(row) * groups + k0 / group] & 15u;
  auto weight = [&](uint32_t k) { return row < d_out && k < d_in ? (w[k >> 1] >> (4 * (k & 1))) & 15u : z; };
  if constexpr (kZeros) {
    v4i f;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t v = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) v |= ((8 * (weight(k0 + 4 * d + e) - z)) & 0xffu) << (8 * e);
      f[d] = static_cast<int>(v);
    }
    frag[idx] = f;
  } else {
    uint32_t word[2];
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      uint32_t v = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) v |= (weight(k0 + 8 * d + e) ^ 8u) << (8 * (e & 3) + 4 * (e >> 2));  // u ^ 8 is u - 8 in four bits
      word[d] = v;
    }
    frag[idx] = make_uint2(word[0], word[1]);
  }
}

__global__ __launch_bounds__(kThreads) void q4_scale_kernel(Tables tb, const float* __restrict__ scales,
                                                            bool zeros, uint32_t d_out, uint32_t group,
                                                            uint32_t groups, uint32_t sub_len, uint32_t subs,
                                                            uint32_t tiles, size_t total, size_t group0, double scale,
                                                            int2* __restrict__ out) {
  const size_t idx = (group0 + blockIdx.x) * kThreads + threadIdx.x;  // [limb][tile][sub][32]
  if (idx >= total) return;
  const uint32_t sub = static_cast<uint32_t>((idx >> 5) % subs);
  const size_t lt = (idx >> 5) / subs;
  const uint32_t l = static_cast<uint32_t>(lt / tiles);
  const uint32_t row = static_cast<uint32_t>(lt % tiles) * 32 + (idx & 31);
  const uint32_t q = tb.q[l];
  int32_t sa = 0, sb = 0;
  if (row < d_out) {
    const size_t at = static_cast<size_t>(row) * groups + static_cast<uint32_t>(static_cast<size_t>(sub) * sub_len / group);
    uint32_t r = reduce_f64_int(rint(static_cast<double>(scales[at]) * scale), q, tb.q_recip[l]);
    r = static_cast<uint32_t>((static_cast<uint64_t>(r) << (zeros ? 29 : 28)) % q);  // 2^32 / 8 or 2^32 / 16
    sa = centred(r, q);
    sb = centred(static_cast<uint32_t>((static_cast<uint64_t>(r) << 16) % q), q);
  }
  out[idx] = make_int2(sa, sb);
}

// Where a workgroup finds its part of the layer.
struct Job {
  const void* frag;        // the whole layer's
  const int2* scales;      // the limb's
  const uint32_t* src;     // input 0's word of column 0 of the workgroup
  uint32_t* dst;           // output 0's
  uint32_t row_bytes, d_out, d_in, steps, subs;
};

// A weight fragment as a matrix operand: 16 v (8 (u - z) with zero points) in each byte.
__device__ __forceinline__ v4i unpack(uint2 w) {
  constexpr uint32_t m = 0xf0f0f0f0u;
  return v4i{static_cast<int>((w.x << 4) & m), static_cast<int>(w.x & m), static_cast<int>((w.y << 4) & m),
             static_cast<int>(w.y & m)};
}
__device__ __forceinline__ v4i unpack(v4i w) { return w; }

// 16 consecutive inputs of one column a thread and pass: pass p of the inputs from
// `first` on holds blocks b0 + p * blockDim/32 + threadIdx.x/32 of 16 inputs.  Inputs past
// d_in, and blocks past `blocks`, read as zero through the buffer range check.
template <int kPasses>
__device__ __forceinline__ void fetch(const Job& job, uint32_t first, uint32_t b0, uint32_t blocks,
                                      uint32_t (&x)[kPasses][16]) {
  const uint32_t tid = threadIdx.x, col = tid & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t row_words = job.row_bytes >> 2;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const uint32_t b = b0 + p * (blockDim.x >> 5) + 2 * wave, base = first + b * 16;  // the wave's two blocks
    const uint32_t rows = b < blocks && base < job.d_in ? min(job.d_in - base, 32u) : 0;
    const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint32_t*>(job.src) + (rows ? static_cast<size_t>(base) * row_words : 0), 0,
        static_cast<int>(rows * job.row_bytes), kRsrcWord3);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[p][i] = __builtin_amdgcn_raw_buffer_load_b32(rs, (((tid >> 5) & 1) * 16 + i) * job.row_bytes + col * 4, 0, 0);
  }
}

// The fetched residues as digit fragments in LDS.
template <int kPasses>
__device__ __forceinline__ void place(uint32_t b0, uint32_t blocks, const uint32_t (&x)[kPasses][16], v4i* lds) {
  const uint32_t tid = threadIdx.x, col = tid & 31;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const uint32_t b = b0 + p * (blockDim.x >> 5) + (tid >> 5);
    if (b < blocks) {
      v4i f[4];
      to_fragments(x[p], f);
#pragma unroll
      for (int d = 0; d < 4; ++d) lds[(b >> 1) * kStepFrags + d * 64 + col + 32 * (b & 1)] = f[d];
    }
  }
}

// T / 2^32 mod q in [0, q) for |T| <= 0.88 q 2^32 (Montgomery's reduction): with m = T /
// q mod 2^32 the difference T - m q is a multiple of 2^32, its quotient s = hi(T) -
// hi(m q) in (-1.88 q, 0.88 q], so the smaller of s and s + 2q, unsigned, lies in
// [0, 2q) and one conditional subtraction finishes.  The bound holds over kFold
// inputs: |16 v| <= 128 times digit pairs of at most 128 * 257 and 128 + 64 * 256,
// times centred scales of at most q / 2, is 0.754 q 2^32, and a sum carried over
// from earlier inputs adds q q / 2 < 0.125 q 2^32.
__device__ __forceinline__ uint32_t reduce(int64_t t, const Modulus& m) {
  const uint32_t k = static_cast<uint32_t>(t) * m.qinv;
  const uint32_t s = static_cast<uint32_t>(t >> 32) - __umulhi(k, m.q);
  const uint32_t u = min(s, s + 2 * m.q);
  return min(u, u - m.q);
}

// A wave's next weights and scales: of one sub-group of kTiles row tiles, asked for before the sub-group ahead of it
// is combined, and across row groups and chunks (768 -> 3072, groups of 128: 3.78 -> 3.69 ms against a
// fresh start a row group; 3072 -> 768 1.53 -> 1.45 ms).  The source asks first thing, but the compiler places the
// loads behind 27 of the 32 matrix operations of a sub-group of 128 and two row tiles (7 of 8 of the chunked kernel's at
// 64), so what covers them is the combination.
template <int kSteps, bool kZeros, int kTiles>
struct Ahead {
  Frag<kZeros> raw[kSteps][kTiles];
  int2 sc[kTiles];
  __device__ __forceinline__ void load(const Job& job, uint32_t tile0, uint32_t sub) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const Frag<kZeros>* w = static_cast<const Frag<kZeros>*>(job.frag) +
                              (static_cast<size_t>(tile0 + t) * job.steps + static_cast<size_t>(sub) * kSteps) * 64;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) raw[s][t] = w[s * 64 + lane];
      sc[t] = job.scales[(static_cast<size_t>(tile0 + t) * job.subs + sub) * 32 + (lane & 31)];
    }
  }
};

// A wave's kTiles row tiles from tile0 on over `subs` sub-groups: sub0 + g of the layer,
// whose residues are sub-group g of the LDS.  Two digits at a time: their sums of a sub-group
// in i32 (below 128 * 128 * 257 * 128 < 2^30), a = S0 + 2^8 S1, then scale times a into
// the 64-bit sums.  `next` holds the first sub-group's weights, and is left with those of (tile1, sub1).
template <int kSteps, bool kZeros, int kTiles>
__device__ __forceinline__ void contract(const Job& job, uint32_t tile0, uint32_t sub0, uint32_t subs, uint32_t tile1,
                                         uint32_t sub1, const v4i* lds, Ahead<kSteps, kZeros, kTiles>& next,
                                         int64_t (&acc)[kTiles][16]) {
  const uint32_t lane = threadIdx.x & 63;
  auto body = [&](uint32_t g) {
    v4i w[kSteps][kTiles];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) w[s][t] = unpack(next.raw[s][t]);
    int2 sg[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sg[t] = next.sc[t];
    const bool more = g + 1 < subs;
    next.load(job, more ? tile0 : tile1, more ? sub0 + g + 1 : sub1);
    const v4i* f = lds + static_cast<size_t>(g) * kSteps * kStepFrags + lane;
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // digits 0 and 1, then 2 and 3
      v16i m[kTiles][2];
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int d = 0; d < 2; ++d) m[t][d] = v16i{};
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const v4i x = f[s * kStepFrags + (2 * half + d) * 64];
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
            m[t][d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w[s][t], m[t][d], 0, 0, 0);
        }
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int32_t sv = half ? sg[t].y : sg[t].x;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[t][r] += static_cast<int64_t>(sv) * (m[t][0][r] + (m[t][1][r] << 8));
      }
    }
  };
  // Loads and stores share one counter, which the loop waits down to zero: the first sub-group of a row
  // group waits for the last outputs' stores too.  For the shortest sub-groups it stands before the loop, with a wait
  // of its own for weights that came before those stores (768 -> 3072, groups of 32: 6.40 -> 6.17 ms; longer
  // sub-groups lose more to registers: groups of 128 3.69 -> 4.02 ms).
  uint32_t g = 0;
  if constexpr (kSteps == 1) body(g++);
  for (; g < subs; ++g) body(g);
}

template <int kTiles>
__device__ __forceinline__ void clear(int64_t (&acc)[kTiles][16]) {
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0;
}

// The row tiles' outputs; rows past d_out are out of range.
template <int kTiles>
__device__ __forceinline__ void store(const Job& job, uint32_t tile0, const Modulus& q, const int64_t (&acc)[kTiles][16]) {
  const uint32_t lane = threadIdx.x & 63, row0 = tile0 * 32;
  const uint32_t rows = row0 < job.d_out ? min(job.d_out - row0, 32u * kTiles) : 0;
  const rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(
      job.dst + (rows ? static_cast<size_t>(row0) * (job.row_bytes >> 2) : 0), 0, static_cast<int>(rows * job.row_bytes),
      kRsrcWord3);
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {  // four adjacent columns
      v4i u;
#pragma unroll
      for (int r = 0; r < 4; ++r) u[r] = static_cast<int>(reduce(acc[t][4 * r4 + r], q));
      __builtin_amdgcn_raw_buffer_store_b128(
          u, out, (t * 32 + (lane & 31)) * job.row_bytes + (8 * r4 + 4 * (lane >> 5)) * 4, 0, 0);
    }
}

// The workgroup's limb, columns and share of the row tiles.  Consecutive workgroup ids
// alternate XCDs: each XCD takes a contiguous range of (limb, column tile, row split),
// so that workgroups which share columns or weights meet in one L2.
struct Place {
  uint32_t limb, split;
};
__device__ __forceinline__ Place place_of(const Tables& tb, const void* frag, const int2* scales,
                                          const uint32_t* ct_in, uint32_t* ct_out, uint32_t d_out, uint32_t d_in,
                                          uint32_t limbs, uint32_t steps, uint32_t subs, uint32_t tiles, uint32_t splits,
                                          Job* job) {
  const uint32_t G = gridDim.x;
  uint32_t lid = blockIdx.x;
  if ((G & 7u) == 0) lid = (lid & 7u) * (G >> 3) + (lid >> 3);
  const uint32_t split = lid % splits, lc = lid / splits, tiles_n = 2 * tb.n / kCols;
  const uint32_t l = lc / tiles_n, ntile = lc - l * tiles_n;
  const uint32_t n = tb.n, col0 = ntile * kCols, c = col0 >> tb.log_n, k0 = col0 & (n - 1);
  const size_t at = (static_cast<size_t>(c) * limbs + l) * n + k0;
  *job = {frag, scales + static_cast<size_t>(l) * tiles * subs * 32, ct_in + at, ct_out + at,
          2u * limbs * n * 4u, d_out, d_in, steps, subs};
  return {l, split};
}

// Inputs that fit the LDS (d_in <= kFold): the workgroup converts its 32 columns once and its
// waves walk groups of kTiles row tiles without further synchronisation.  Two tiles a wave leave
// registers for two waves a SIMD: one workgroup of eight waves a CU, or two of four where both strips fit
// the LDS (640 inputs), so that one converts while the other contracts (2^14, 2 limbs, groups of 128, one : two
// workgroups, us: 384 -> 384 70 : 61, 512 -> 512 102 : 90, 384 -> 1536 210 : 200; four waves alone at 768 ->
// 768 209 against 197).  One tile a wave leaves them for four waves a SIMD, and four strips of up to 320 inputs
// fit: there the fill counts for more than the residues' second reading.  Three instances with zero points spill
// one register: both of two tiles in groups of 128, and one tile in groups of 96.
constexpr uint32_t kLdsBytes = 160 << 10;
template <int kSteps, bool kZeros, int kWaves, int kTiles>
__global__ __launch_bounds__(kWaves * 64, kTiles == 1 ? 4 : 2) void mac_q4_whole_kernel(
    Tables tb, const void* __restrict__ frag, const int2* __restrict__ scales, const uint32_t* __restrict__ ct_in,
    uint32_t* __restrict__ ct_out, uint32_t d_out, uint32_t d_in, uint32_t limbs, uint32_t steps, uint32_t subs,
    uint32_t tiles, uint32_t splits) {
  extern __shared__ v4i lds[];
  Job job;
  const Place at = place_of(tb, frag, scales, ct_in, ct_out, d_out, d_in, limbs, steps, subs, tiles, splits,
                            &job);
  const Modulus q = modulus(tb.q[at.limb]);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t groups = tiles / kTiles, each = (groups + splits - 1) / splits;
  const uint32_t end = min(groups, (at.split + 1) * each);
  constexpr int kPasses = 4;
  for (uint32_t b0 = 0; b0 < 2 * steps; b0 += kPasses * kWaves * 2) {
    uint32_t x[kPasses][16];
    fetch<kPasses>(job, 0, b0, 2 * steps, x);
    place<kPasses>(b0, 2 * steps, x, lds);
  }
  __syncthreads();
  Ahead<kSteps, kZeros, kTiles> next;
  uint32_t rg = at.split * each + wave;
  if (rg >= end) return;
  next.load(job, rg * kTiles, 0);
  for (; rg < end; rg += kWaves) {
    int64_t acc[kTiles][16];
    clear<kTiles>(acc);
    const uint32_t after = rg + kWaves < end ? rg + kWaves : rg;
    contract<kSteps, kZeros, kTiles>(job, rg * kTiles, 0, subs, after * kTiles, 0, lds, next, acc);
    store<kTiles>(job, rg * kTiles, q, acc);
  }
}

// More inputs than that: the workgroup's waves take one row tile each and go through
// chunks of kChunk steps together, the next chunk's residues in flight in registers
// while the matrix cores work on this one's out of the other half of the LDS.
constexpr int kDeepWaves = 12, kDeepTiles = 1;
constexpr uint32_t kChunk = kDeepWaves;  // steps of a chunk: 16 inputs of one column a thread
static_assert(kChunk % 3 == 0 && kChunk % 4 == 0 && 2 * kChunk * kStep <= kFold, "whole sub-groups, and a reduction every other chunk");
template <int kSteps, bool kZeros>
__global__ __launch_bounds__(kDeepWaves * 64, 1) void mac_q4_deep_kernel(
    Tables tb, const void* __restrict__ frag, const int2* __restrict__ scales, const uint32_t* __restrict__ ct_in,
    uint32_t* __restrict__ ct_out, uint32_t d_out, uint32_t d_in, uint32_t limbs, uint32_t steps, uint32_t subs,
    uint32_t tiles, uint32_t splits) {
  __shared__ v4i lds[2][kChunk * kStepFrags];
  Job job;
  const Place at = place_of(tb, frag, scales, ct_in, ct_out, d_out, d_in, limbs, steps, subs, tiles, splits,
                            &job);
  const Modulus q = modulus(tb.q[at.limb]);
  const int32_t c32 = centred(tb.pow256[at.limb * 8 + 4], q.q);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t each = (tiles + splits - 1) / splits, tile = at.split * each + wave;
  const bool mine = wave < each && tile < tiles;
  int64_t acc[kDeepTiles][16];
  clear<kDeepTiles>(acc);
  uint32_t x[1][16];
  fetch<1>(job, 0, 0, 2 * kChunk, x);
  place<1>(0, 2 * kChunk, x, lds[0]);
  __syncthreads();
  Ahead<kSteps, kZeros, kDeepTiles> next;
  if (mine) next.load(job, tile, 0);
  uint32_t buf = 0;
  for (uint32_t s0 = 0; s0 < steps; s0 += kChunk, buf ^= 1) {
    const bool more = s0 + kChunk < steps;
    if (more) fetch<1>(job, (s0 + kChunk) * kStep, 0, 2 * kChunk, x);
    if (mine) {
      if (buf == 0 && s0 != 0) {  // every other chunk: the sum so far, reduced, goes on as a product
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][r] = static_cast<int64_t>(static_cast<int32_t>(reduce(acc[0][r], q))) * c32;
      }
      contract<kSteps, kZeros, kDeepTiles>(job, tile, s0 / kSteps, min(kChunk, steps - s0) / kSteps, tile,
                                           more ? (s0 + kChunk) / kSteps : 0, lds[buf], next, acc);
    }
    if (more) place<1>(0, 2 * kChunk, x, lds[buf ^ 1]);
    __syncthreads();
  }
  if (mine) store<kDeepTiles>(job, tile, q, acc);
}

// Few outputs: a lane has one column and kRows rows, and four-byte dot products take the matrix
// instructions' place, on the same operands: a lane's digits of 16 inputs, and weights that are the
// same for all lanes and so come into scalar registers.  No LDS and small workgroups, so that many loads
// are in flight: it is bound by memory up to 8 outputs (2^16, 4 limbs, 1 -> 8 outputs, us, groups of 128: 1 input
// 13 -> 15, 64 inputs 30 -> 33, 1024 inputs 430 -> 450, 4.8 to 5.0 TB/s; 150, 155, 860 with a
// matrix tile of 32 mostly empty rows), by the dot products and the digits above.  Sixteen rows a lane for more
// outputs share the digits (1024 -> 16: 600 us, 748 with eight).  A workgroup is 64 columns: `blocks` waves of kRows
// rows each, times `slices` shares of the sub-groups where the columns alone are too few waves; their sums meet in LDS.
constexpr int kThinWaves = 8, kThinCols = 64;
template <int kSteps, bool kZeros, int kRows>
__global__ __launch_bounds__(kThinWaves * 64, kRows == 8 ? 4 : 2) void mac_q4_thin_kernel(
    Tables tb, const Frag<kZeros>* __restrict__ frag, const int2* __restrict__ scales, const uint32_t* __restrict__ ct_in,
    uint32_t* __restrict__ ct_out, uint32_t d_out, uint32_t d_in, uint32_t limbs, uint32_t steps, uint32_t subs,
    uint32_t tiles, uint32_t blocks, uint32_t slices) {
  extern __shared__ uint32_t sums[];  // with slices: [waves][kRows][kThinCols]
  constexpr uint32_t kSub = kSteps * kStep, kFoldSubs = kFold / kSub;
  const uint32_t n = tb.n, strips = 2 * n / kThinCols, l = blockIdx.x / strips, col0 = (blockIdx.x - l * strips) * kThinCols;
  const uint32_t row_words = 2 * limbs * n, lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slice = wave / blocks, block = wave - slice * blocks;
  const uint32_t row0 = block * kRows, tile = row0 / 32, r32 = row0 % 32;
  const size_t at = (static_cast<size_t>(col0 >> tb.log_n) * limbs + l) * n + (col0 & (n - 1));
  const Modulus q = modulus(tb.q[l]);
  const int32_t c32 = centred(tb.pow256[l * 8 + 4], q.q);
  const uint32_t each = (subs + slices - 1) / slices, sub0 = slice * each, sub1 = min(subs, sub0 + each);
  int64_t acc[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) acc[r] = 0;
  for (uint32_t g = sub0; g < sub1; ++g) {
    if (g != sub0 && (g - sub0) % kFoldSubs == 0) {  // the sum so far, reduced, goes on as a product
#pragma unroll
      for (int r = 0; r < kRows; ++r) acc[r] = static_cast<int64_t>(static_cast<int32_t>(reduce(acc[r], q))) * c32;
    }
    int32_t m[kRows][4];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int d = 0; d < 4; ++d) m[r][d] = 0;
#pragma unroll 1
    for (uint32_t b = 0; b < 2 * kSteps; ++b) {
      const uint32_t base = g * kSub + b * 16;
      if (base >= d_in) break;
      const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint32_t*>(ct_in) + at + static_cast<size_t>(base) * row_words, 0,
          static_cast<int>(min(d_in - base, 16u) * row_words * 4), kRsrcWord3);
      uint32_t x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b32(rs, (i * row_words + lane) * 4, 0, 0);
      v4i f[4];
      to_fragments(x, f);
      const Frag<kZeros>* w = frag + (static_cast<size_t>(tile) * steps + g * kSteps + b / 2) * 64 + 32 * (b & 1) + r32;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const v4i wr = unpack(w[r]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < 4; ++d) m[r][d] = __builtin_amdgcn_sdot4(f[d][e], wr[e], m[r][d], false);
      }
    }
    const int2* sg = scales + ((static_cast<size_t>(l) * tiles + tile) * subs + g) * 32 + r32;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      acc[r] += static_cast<int64_t>(sg[r].x) * (m[r][0] + (m[r][1] << 8));
      acc[r] += static_cast<int64_t>(sg[r].y) * (m[r][2] + (m[r][3] << 8));
    }
  }
  uint32_t y[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) y[r] = reduce(acc[r], q);
  if (slices > 1) {
    if (slice != 0) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) sums[(wave * kRows + r) * kThinCols + lane] = y[r];
    }
    __syncthreads();
    if (slice != 0) return;
    for (uint32_t k = 1; k < slices; ++k)
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const uint32_t v = y[r] + sums[((k * blocks + block) * kRows + r) * kThinCols + lane];
        y[r] = min(v, v - q.q);
      }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    if (row0 + r < d_out) ct_out[at + static_cast<size_t>(row0 + r) * row_words + lane] = y[r];
}

template <int kSteps, bool kZeros>
hipError_t launch(const Tables& t, const Shape& sh, const void* w_q4, const uint32_t* ct_in, uint32_t* ct_out,
                  uint32_t d_out, uint32_t d_in, uint32_t limbs, hipStream_t s) {
  const uint8_t* base = static_cast<const uint8_t*>(w_q4);
  const void* frag = base;
  const int2* scales = reinterpret_cast<const int2*>(base + sh.frag_bytes);
  const uint32_t strips = 2 * t.n / kCols * limbs;  // column tiles of every limb
  // Enough columns for four strips a CU.  Below that every call takes 10 to 20 us, and the forms made for many
  // strips lose up to half of it (2^12, 3 limbs, 256 -> 1: 17.8 us one row tile a wave, 12.8 chunked).
  const bool many = strips >= 4 * t.num_cus;
  // Dot products against the matrix forms, us, groups of 128: 2^16, 4 limbs, 1024 -> 8 450 : 856, 64 -> 16 44 : 57, 256 ->
  // 16 156 : 163, 1024 -> 16 600 : 875, 16 -> 32 35 : 52, 64 -> 32 77 : 66; 2^14, 4 limbs, 64 -> 16 15 : 17, 256 -> 16 47 :
  // 28, 512 -> 16 89 : 61, 1024 -> 16 181 : 175 (groups of 32 196 : 261), 32 -> 32 16 : 18, 64 -> 32 25 : 17.  From 65 to
  // 640 inputs the two rings differ for 9 to 16 outputs: the matrix form loses 4% at 2^16 and wins 40% at 2^14.
  if (many && (d_out <= 8 || (d_out <= 16 && (d_in <= 64 || d_in > 640)) || (d_out <= 32 && d_in <= 32))) {
    const uint32_t rows = d_out <= 8 ? 8 : 16, cols = strips / (kThinCols / kCols), blocks = (d_out + rows - 1) / rows;
    const uint32_t want = t.num_cus * 16;
    uint32_t slices = 1;
    while (cols * blocks * slices < want && 2 * slices * blocks <= kThinWaves && 2 * slices <= sh.subs) slices *= 2;
    const auto k = rows == 8 ? mac_q4_thin_kernel<kSteps, kZeros, 8> : mac_q4_thin_kernel<kSteps, kZeros, 16>;
    k<<<cols, blocks * slices * 64, slices > 1 ? blocks * slices * rows * kThinCols * 4 : 0, s>>>(
        t, static_cast<const Frag<kZeros>*>(frag), scales, ct_in, ct_out, d_out, d_in, limbs, sh.steps, sh.subs, sh.tiles,
        blocks, slices);
    return hipGetLastError();
  }
  // 2^16, 4 limbs, groups of 128, us, one tile a wave : two : chunked: 4 -> 64 76 : 93 : 181, 256 -> 64 214 : 241 :
  // 339, 256 -> 512 785 : 808, 512 -> 128 481 : 491 : 623, 512 -> 200 646 : 607 : 782; 2^14, 4 limbs, one tile : two, 128 ->
  // 320 55 : 66, 256 -> 512 147 : 151, 256 -> 1024 255 : 239, 64 -> 2048 314 : 287.
  // Past 640 inputs one strip fills a CU, and with few outputs most of its waves idle behind the one conversion: the
  // chunked kernel overlaps the two (2^14, 2 limbs, whole : chunked, 1024 -> 128 102 : 93, 1024 -> 384 158 : 166,
  // 768 -> 768 196 : 239).
  const size_t strip_bytes = size_t(sh.steps) * kStepFrags * 16;
  const bool four = 4 * strip_bytes <= kLdsBytes, two = 2 * strip_bytes <= kLdsBytes;  // strips that fit a CU
  const bool one_tile = many && ((four && d_out <= 512) || (two && d_out <= 128));
  if (one_tile || (d_in <= kFold && (d_out > 256 || (many && two)))) {
    const uint32_t row_tiles = one_tile ? 1 : 2, waves = two ? 4 : 8;
    const auto k = row_tiles == 1 ? mac_q4_whole_kernel<kSteps, kZeros, 4, 1>
                   : two          ? mac_q4_whole_kernel<kSteps, kZeros, 4, 2>
                                  : mac_q4_whole_kernel<kSteps, kZeros, 8, 2>;
    // Row splits only where the column strips alone leave CUs idle: each split converts the strip again.
    const uint32_t groups = sh.tiles / row_tiles, blocks = (groups + waves - 1) / waves;
    const uint32_t want = (t.num_cus * (8 / waves) + strips - 1) / strips, splits = want < blocks ? want : blocks;
    k<<<strips * splits, waves * 64, strip_bytes, s>>>(t, frag, scales, ct_in, ct_out, d_out, d_in, limbs, sh.steps, sh.subs,
                                                      sh.tiles, splits);
  } else {
    const uint32_t splits = (sh.tiles + kDeepWaves - 1) / kDeepWaves;
    mac_q4_deep_kernel<kSteps, kZeros><<<strips * splits, kDeepWaves * 64, 0, s>>>(
        t, frag, scales, ct_in, ct_out, d_out, d_in, limbs, sh.steps, sh.subs, sh.tiles, splits);
  }
  return hipGetLastError();
}

}  // namespace

size_t q4_weight_bytes(uint32_t d_out, uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros) {
  if (d_out == 0 || d_in == 0) return 0;
  const Shape s = shape_of(d_out, d_in, group, limbs, zeros);
  return s.frag_bytes + s.scale_bytes;
}

hipError_t launch_encode_q4(const Tables& t, const uint8_t* w4, const float* scales, const uint8_t* zeros,
                            uint32_t d_out, uint32_t d_in, uint32_t group, uint32_t limbs, double scale, void* w_q4,
                            hipStream_t s) {
  const Shape sh = shape_of(d_out, d_in, group, limbs, zeros != nullptr);
  uint8_t* base = static_cast<uint8_t*>(w_q4);
  const size_t lanes = static_cast<size_t>(sh.tiles) * sh.steps * 64;
  const size_t total = static_cast<size_t>(limbs) * sh.tiles * sh.subs * 32;
  hipError_t e = in_pieces((lanes + kThreads - 1) / kThreads, [&](uint64_t first, uint32_t groups) {
    if (zeros)
      q4_frag_kernel<true><<<groups, kThreads, 0, s>>>(w4, zeros, d_out, d_in, group, sh.groups, sh.steps, lanes, first,
                                                       reinterpret_cast<v4i*>(base));
    else
      q4_frag_kernel<false><<<groups, kThreads, 0, s>>>(w4, zeros, d_out, d_in, group, sh.groups, sh.steps, lanes, first,
                                                        reinterpret_cast<uint2*>(base));
  });
  if (e != hipSuccess) return e;
  return in_pieces((total + kThreads - 1) / kThreads, [&](uint64_t first, uint32_t groups) {
    q4_scale_kernel<<<groups, kThreads, 0, s>>>(t, scales, zeros != nullptr, d_out, group, sh.groups, sh.sub_len, sh.subs,
                                                sh.tiles, total, first, scale, reinterpret_cast<int2*>(base + sh.frag_bytes));
  });
}

hipError_t launch_mac_q4(const Tables& t, const void* w_q4, const uint32_t* ct_in, uint32_t* ct_out, uint32_t d_out,
                         uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros, hipStream_t s) {
  const Shape sh = shape_of(d_out, d_in, group, limbs, zeros);
  switch (sh.sub_len) {
    case 32: return (zeros ? launch<1, true> : launch<1, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
    case 64: return (zeros ? launch<2, true> : launch<2, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
    case 96: return (zeros ? launch<3, true> : launch<3, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
    default: return (zeros ? launch<4, true> : launch<4, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
  }
}

}  // namespace ckks
