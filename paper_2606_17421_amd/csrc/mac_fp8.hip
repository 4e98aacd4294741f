// ct x pt MAC over 8-bit floating-point (e4m3) weights with one scale per block of
// 128 inputs and some outputs on the gfx950 matrix cores, exact over the plaintexts:
// one layer, or requests that each name an expert's layer and a bundle of inputs.
//
// Per limb l, with f the weights, v = rint(64 f) and S = rint(scale Delta / 64) of a block,
//     out[j][col] = sum_b S[j][b] T[j][b][col] mod q_l,
//     T[j][b][col] = sum over the 128 inputs of v[j][i] x[i][col].
// |v| <= 64 * 448 = 28672 is two balanced base-256 digits, the same for every limb, against the
// residues' four: eight int8 products a modular MAC.  Every step of e4m3 (2^-9) would take three
// digits and twelve; what the rounding to 64ths costs is 2^-7 at most of a weight below 1/8, 2^-15.8 of the largest one.
// With a unit for each row and block, v = rint(u f) and S = rint(scale Delta / u) for u up to 512, the two digits keep rows that
// are small beside their block's largest as well; the constants are a row's anyway, so the kernels are the same.
// T = a + 2^16 b + 2^32 c with a and b from two digit sums each and c from one; a block's scale enters
// in 64-bit integers, and the sum over the blocks is reduced once an output.
//
// Four kernels share the arithmetic, chosen in launch():
//   short    one block of inputs, their digits in registers (at 2^14, 4 limbs: 64 -> 256 39 us, 4.3 TB/s, outputs for the
//            most part; 128 -> 512 89 us, 3.8 TB/s).
//   thin     few outputs or few columns: residues go from memory through registers to the matrix cores; bound by
//            memory (1024 -> 16 at 2^13, 3 limbs: 42 us, 4.8 TB/s, what a large copy reaches).
//   chunked  a row tile a wave, all inputs in turn (2048 -> 768 at 2^14, 4 limbs: 1.57-1.65 ms over boxes,
//            1.0e15 int8 products/s).
//   whole    up to 1024 inputs: they stay in LDS while the waves walk the row tiles (1024 -> 2048 at 2^15, 4 limbs: 3.64-3.85
//            ms, 1.15e15 products/s; large int8 matrix products of the library's make 1.0e15 to 1.2e15).
// What bounds the last two: issue and power.  A block of a row tile takes a SIMD 1680 cycles in 1024 -> 2048: its 32 matrix
// operations keep the matrix pipe busy for 1024 of them (61%) and take 16 issue cycles each, beside 48 multiply-adds of 8.7
// and 72 other vector operations of 4.5, 1250 of the 1680 (measured alone: 20 matrix operations and 80 shift-adds of
// another wave take 309 and 192 ns, 320 together; with 80 multiply-adds 313 and 311, 411 together).  The chip holds 1.83-1.87
// GHz (1.96-2.06 GHz and 50% chunked; a loop of nothing but matrix operations on random numbers makes 1.75e15 products/s at
// 1.7 GHz).  Without the weights' loads it takes 7% less, without the residues' 3%.  Measured without effect or worse:
// sums combined between the same wave's matrix operations (3.65 -> 3.85 ms), wave priorities by phase or by half, a
// delayed half, four-wave workgroups for the chunked kernel (4.2 -> 4.8 ms), loads past the caches.
#include <algorithm>

#include "digits.hpp"

namespace ckks {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kStep = 32;        // inputs of one matrix-core step
constexpr uint32_t kBlock = 128;      // inputs that share a scale
constexpr uint32_t kBlockSteps = kBlock / kStep;
constexpr uint32_t kFoldBlocks = 8;   // most blocks between reductions of the 64-bit sums
constexpr uint32_t kFewBlocks = 4;    // of a layer whose sums take the shorter of them
constexpr int kPairs = 5;             // digit sums of a block: weight digit a times residue digit b in sum a + b
constexpr int kDigits = 2;            // of a weight
constexpr uint32_t kChunkBlocks = 2, kChunk = kChunkBlocks * kBlockSteps;  // blocks and steps that go into LDS at a time
constexpr int kNonTemporal = 2;        // cache policy of a buffer instruction
constexpr int kStepFrags = 4 * 64;    // 16-byte residue fragments of a step: four digits, 64 lanes

// Encoded weights (written once a layer):
//   fragments [tile][step][digit][64 lanes] of 16 bytes: digit of row tile*32 + lane%32 and inputs
//     step*32 + 16 (lane/32) + i, i < 16; rows are padded to 32, inputs to 32.
//   scales [limb][tile][block][3][32 rows]: 2^32 S, 2^48 S and 2^64 S mod q_l, centred.  The
//     2^32 is what the closing reduction divides by.
struct Shape {
  uint32_t tiles, steps, blocks;
  size_t frag_bytes, scale_bytes;
};

Shape shape_of(uint32_t d_out, uint32_t d_in, uint32_t limbs) {
  Shape s;
  s.tiles = (d_out + 31) / 32;
  s.steps = (d_in + kStep - 1) / kStep;
  s.blocks = (d_in + kBlock - 1) / kBlock;
  s.frag_bytes = static_cast<size_t>(s.tiles) * s.steps * kDigits * 64 * 16;
  s.scale_bytes = static_cast<size_t>(limbs) * s.tiles * s.blocks * 3 * 32 * 4;
  return s;
}

// rint(64 2^fine f) of an e4m3 code, half to even, fine at most 3.  A code is a sign, four bits of exponent and three of
// mantissa; 512 f is a whole number.  NaN (all of exponent and mantissa set) counts as 0.
__device__ __forceinline__ int32_t units_of(uint32_t code, uint32_t fine, bool* nan, bool* rounded) {
  const uint32_t e = code >> 3 & 15, m = code & 7;
  const uint32_t u = e == 0 ? m : (8 + m) << (e - 1);  // 512 |f|
  const uint32_t drop = 3 - fine, half = (1u << drop) >> 1;
  const int32_t v = static_cast<int32_t>((u + half - (half != 0 && (u >> drop & 1) == 0)) >> drop);
  *nan = (code & 0x7f) == 0x7f;
  *rounded = !*nan && (u & ((1u << drop) - 1)) != 0;
  return *nan ? 0 : code & 0x80 ? -v : v;
}

// The finest unit that two digits hold for all weights of a row and block, 2^-6-fine with 64 2^fine |f| <= 28672, into the
// places of the constants that fp8_scale_kernel replaces, of every limb.  The size of a number goes with its code.  A lane
// reads a row's 128 codes one by one: 1024 -> 6144 at 8 limbs takes 41 us encoded so and 20 in 64ths, once a layer.
__global__ __launch_bounds__(kThreads) void fp8_unit_kernel(const uint8_t* __restrict__ w8, uint32_t d_out, uint32_t d_in,
                                                            uint32_t blocks, uint32_t tiles, uint32_t limbs, size_t total,
                                                            size_t group0, int32_t* __restrict__ out) {
  const size_t idx = (group0 + blockIdx.x) * kThreads + threadIdx.x;  // [tile][block][32]
  if (idx >= total) return;
  const size_t tb = idx >> 5;
  const uint32_t block = static_cast<uint32_t>(tb % blocks), row = static_cast<uint32_t>(tb / blocks) * 32 + (idx & 31);
  uint32_t most = 0;
  if (row < d_out) {
    const uint8_t* w = w8 + static_cast<size_t>(row) * d_in;
    for (uint32_t k = block * kBlock; k < min(d_in, (block + 1) * kBlock); ++k) {
      const uint32_t size = w[k] & 0x7f;
      most = max(most, size == 0x7f ? 0 : size);
    }
  }
  const int32_t fine = (most <= 0x66) + (most <= 0x6e) + (most <= 0x76);  // 56, 112 and 224
  for (uint32_t l = 0; l < limbs; ++l) out[(static_cast<size_t>(l) * tiles * blocks + tb) * 96 + (idx & 31)] = fine;
}

// With kUnits by what fp8_unit_kernel wrote, else 64ths throughout.
template <bool kUnits>
__global__ __launch_bounds__(kThreads) void fp8_frag_kernel(const uint8_t* __restrict__ w8, uint32_t d_out, uint32_t d_in,
                                                            uint32_t steps, size_t lanes, size_t group0,
                                                            const int32_t* __restrict__ units, int32_t* bad, int32_t* rounded,
                                                            v4i* __restrict__ frag) {
  const size_t idx = (group0 + blockIdx.x) * kThreads + threadIdx.x;
  if (idx >= lanes) return;
  const uint32_t lane = idx & 63;
  const uint32_t step = static_cast<uint32_t>((idx >> 6) % steps), tile = static_cast<uint32_t>((idx >> 6) / steps);
  const uint32_t row = tile * 32 + (lane & 31), k0 = step * kStep + 16 * (lane >> 5);
  const uint8_t* w = w8 + static_cast<size_t>(row) * d_in;
  const uint32_t blocks = (steps + kBlockSteps - 1) / kBlockSteps;
  const uint32_t fine = kUnits ? units[(static_cast<size_t>(tile) * blocks + step / kBlockSteps) * 96 + (lane & 31)] : 0;
  v4i f[kDigits];
  int32_t nans = 0, off = 0;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = k0 + 4 * d + e;
      bool nan = false, moved = false;
      const int32_t v = row < d_out && k < d_in ? units_of(w[k], fine, &nan, &moved) : 0;
      nans += nan;
      if (kUnits) off += moved;
      const uint32_t b = (static_cast<uint32_t>(v) + 0x8080u) ^ 0x8080u;  // its low two bytes, as int8, are the digits
      lo |= (b & 0xffu) << (8 * e);
      hi |= (b >> 8 & 0xffu) << (8 * e);
    }
    f[0][d] = static_cast<int>(lo);
    f[1][d] = static_cast<int>(hi);
  }
  if (bad && nans) atomicAdd(bad, nans);
  if (kUnits && rounded && off) atomicAdd(rounded, off);
#pragma unroll
  for (int d = 0; d < kDigits; ++d) frag[((idx >> 6) * kDigits + d) * 64 + lane] = f[d];
}

template <bool kUnits>
__global__ __launch_bounds__(kThreads) void fp8_scale_kernel(Tables tb, const float* __restrict__ scales, uint32_t d_out,
                                                             uint32_t block_rows, uint32_t blocks, uint32_t tiles,
                                                             size_t total, size_t group0, double scale,
                                                             int32_t* bad, int32_t* __restrict__ out) {
  const size_t idx = (group0 + blockIdx.x) * kThreads + threadIdx.x;  // [limb][tile][block][32]
  if (idx >= total) return;
  const uint32_t block = static_cast<uint32_t>((idx >> 5) % blocks);
  const size_t lt = (idx >> 5) / blocks;
  const uint32_t l = static_cast<uint32_t>(lt / tiles);
  const uint32_t row = static_cast<uint32_t>(lt % tiles) * 32 + (idx & 31);
  const uint32_t q = tb.q[l];
  uint32_t r = 0;
  if (row < d_out) {
    const double s = scales[static_cast<size_t>(row / block_rows) * blocks + block], v = s * scale;
    // no infinity and no NaN; and a scale too small for `scale`, in its finest unit, takes its block's weights with it
    const bool fine = fabs(v) < 9223372036854775808.0 && (s == 0 || rint(kUnits ? v / 8 : v) != 0);
    if (fine) r = reduce_f64_int(rint(kUnits ? ldexp(v, -out[(idx >> 5) * 96 + (idx & 31)]) : v), q, tb.q_recip[l]);
    if (bad && !fine && l == 0 && row % block_rows == 0) atomicAdd(bad, 1);
  }
#pragma unroll
  for (int d = 0; d < 3; ++d) {
    r = static_cast<uint32_t>((static_cast<uint64_t>(r) << (d == 0 ? 32 : 16)) % q);
    out[((idx >> 5) * 3 + d) * 32 + (idx & 31)] = centred(r, q);
  }
}

// LDS that the digits of 32 columns take.
constexpr size_t kLdsBytes = 160 << 10;
size_t strip_bytes(const Shape& s) { return static_cast<size_t>(s.steps + kChunk - 1) / kChunk * kChunk * kStepFrags * 16; }

constexpr size_t kWaveSums = 16 * 64 * 4;  // a wave's outputs of a row tile, on their way to another wave or to memory

// A layer, or a layer for each expert, and what it is applied to.
struct Layers {
  const uint8_t* w;       // [experts]: fragments, then scales
  size_t w_bytes;         // of one expert
  const uint32_t* ct_in;  // [bundles][d_in][2][limbs][N]
  uint32_t* ct_out;       // [requests][d_out][2][limbs][N]
  const int32_t* expert;  // [requests], or null: expert 0
  const int32_t* bundle;  // [requests], or null: the request's own number
  int32_t* status;        // [requests], or null
  uint32_t experts, bundles, count, d_out, d_in, limbs;
  Shape sh;
};

// Where a workgroup finds its part of a request.
struct Job {
  const v4i* frag;
  const int32_t* scales;   // the limb's
  const uint32_t* src;     // input 0's word of column 0 of the workgroup
  uint32_t* dst;           // output 0's
  uint32_t limb, split;
};

__device__ __forceinline__ uint32_t row_bytes(const Tables& tb, const Layers& a) { return 8u * a.limbs * tb.n; }

__device__ __forceinline__ bool named(const Layers& a, uint32_t request, uint32_t* expert, uint32_t* bundle) {
  *expert = a.expert ? static_cast<uint32_t>(a.expert[request]) : 0;
  *bundle = a.bundle ? static_cast<uint32_t>(a.bundle[request]) : request;
  return *expert < a.experts && *bundle < a.bundles;
}

// The status of requests for layers without outputs.
__global__ __launch_bounds__(kThreads) void experts_status_kernel(Layers a, uint32_t count) {
  const uint32_t r = blockIdx.x * kThreads + threadIdx.x;
  uint32_t e, b;
  if (r < count) a.status[r] = named(a, r, &e, &b) ? kExpertOk : kExpertBadRequest;
}

// Request, limb, `cols` columns and share of the row tiles of a workgroup's job; false where the request names no
// expert or no bundle.  An XCD has an eighth of every limb's columns (`cols` at most 128 of 2^11 and more, so there are
// that many), its jobs numbered by limb, request, column strip and row split: neighbours share weights or columns, and a
// limb of a bundle stays in the caches for the requests that name it too (16 requests of 4 bundles of 1024 -> 64 at 2^12, 3
// limbs: 415 us with all limbs of a request in turn, 343 so).
__device__ __forceinline__ bool place_of(const Tables& tb, const Layers& a, uint32_t cols, uint32_t splits, uint32_t id, Job* job) {
  const uint32_t n = tb.n, strips = 2 * n / cols / 8, split = id % splits, u = id / splits, v = u / strips;
  const uint32_t l = v / a.count, r = v - l * a.count, col0 = ((blockIdx.x & 7) * strips + u - v * strips) * cols;
  uint32_t e, b;
  const bool good = named(a, r, &e, &b);
  if (a.status && l == 0 && col0 == 0 && split == 0 && threadIdx.x == 0) a.status[r] = good ? kExpertOk : kExpertBadRequest;
  if (!good) return false;
  const uint8_t* w = a.w + e * a.w_bytes;
  const size_t at = (static_cast<size_t>(col0 >> tb.log_n) * a.limbs + l) * n + (col0 & (n - 1));
  const size_t row_words = static_cast<size_t>(2) * a.limbs * n;
  *job = {reinterpret_cast<const v4i*>(w),
          reinterpret_cast<const int32_t*>(w + a.sh.frag_bytes) + static_cast<size_t>(l) * a.sh.tiles * a.sh.blocks * 96,
          a.ct_in + b * row_words * a.d_in + at,
          a.ct_out + r * row_words * a.d_out + at, l, split};
  return true;
}

// Consecutive workgroup ids alternate XCDs; each XCD has an eighth of every request's columns, so that requests that name
// nothing leave no XCD idle (13 of 16 requests of 200 -> 333 at 2^11 and 2 limbs: 103 -> 86 us), and its workgroups take
// jobs next to each other at any time: `first`, then every `stride`-th below `end`.
struct Range {
  uint32_t first, stride, end;
};
__device__ __forceinline__ Range range_of(uint32_t jobs) {
  const uint32_t xcd = blockIdx.x & 7;
  return {blockIdx.x >> 3, (gridDim.x - xcd + 7) / 8, jobs / 8};
}

// A persistent workgroup's jobs in turn, those of requests that name nothing left out.
struct Jobs {
  Range range;
  __device__ __forceinline__ bool next(const Tables& tb, const Layers& a, uint32_t cols, uint32_t splits, Job* job) {
    while (range.first < range.end) {
      const uint32_t id = range.first;
      range.first += range.stride;
      if (place_of(tb, a, cols, splits, id, job)) return true;
    }
    return false;
  }
};

// 16 consecutive inputs of one column a lane: lane l has column l % 32 of those at `src`, and the first or the second
// half of the 32 inputs from `base` on.  Inputs past d_in read as zero through the buffer range check.
__device__ __forceinline__ void fetch_step(const Tables& tb, const Layers& a, const uint32_t* src, uint32_t base,
                                           uint32_t (&x)[16]) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t bytes = row_bytes(tb, a);
  asm volatile("" : "+s"(bytes));  // else the 16 rows' offsets are kept in registers
  const uint32_t rows = base < a.d_in ? min(a.d_in - base, kStep) : 0;
  const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint32_t*>(src) + (rows ? static_cast<size_t>(base) * (bytes >> 2) : 0), 0, static_cast<int>(rows * bytes),
      kRsrcWord3);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    x[i] = __builtin_amdgcn_raw_buffer_load_b32(rs, ((lane >> 5) * 16 + i) * bytes + (lane & 31) * 4, 0, 0);
}

// Residues on their way to LDS.  Unit u of a chunk is step u / kColWaves of columns 32 (u % kColWaves) and on; a wave
// takes every kWaves-th, one a pass.
template <int kWaves, int kColWaves>
struct Stage {
  uint32_t x[16];
  __device__ __forceinline__ void fetch(const Tables& tb, const Layers& a, const Job& job, uint32_t step0, int pass) {
    const uint32_t u = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) + pass * kWaves;
    fetch_step(tb, a, job.src + u % kColWaves * 32, (step0 + u / kColWaves) * kStep, x);
  }
  // As digit fragments [column tile][step] in LDS.
  __device__ __forceinline__ void place(v4i* lds, int pass) const {
    const uint32_t lane = threadIdx.x & 63, u = (threadIdx.x >> 6) + pass * kWaves;
    v4i f[4];
    to_fragments(x, f);
#pragma unroll
    for (int d = 0; d < 4; ++d) lds[(u % kColWaves * kChunk + u / kColWaves) * kStepFrags + d * 64 + lane] = f[d];
  }
};

// T / 2^32 mod q in [0, q) for |T| <= 1.88 q 2^32 (Montgomery's reduction): with m = T / q mod 2^32 the
// difference T - m q is a multiple of 2^32 whose quotient is hi(T) - hi(m q).  h = hi(T) is taken to [0,
// 2q) first (for h < 0 the sum h + 2q is below 2^31 and h itself, unsigned, above; for h >= 0 h is the smaller), the
// difference lies in (-q, 2q), and two conditional corrections finish.  The bound holds over kFoldBlocks
// blocks: per block |a| <= 128 (128 * 128 + 256 (128 * 128 + 112 * 128)) < 1.010e9, |b| <= 128 (128 * 128 + 112 *
// 128 + 256 (128 * 64 + 112 * 128)) < 0.743e9, |c| <= 128 * 112 * 64 < 0.001e9 times centred scales of at
// most q / 2 is 0.877e9 q, eight of them and a sum carried over from earlier blocks, at most q q / 2 < 0.537e9 q, are
// 7.56e9 q < 1.77 q 2^32 (and below 2^63).
__device__ __forceinline__ uint32_t reduce(int64_t t, const Modulus& m) {
  const uint32_t h = static_cast<uint32_t>(t >> 32);
  const uint32_t k = static_cast<uint32_t>(t) * m.qinv;
  const uint32_t s = min(h, h + 2 * m.q) - __umulhi(k, m.q);
  const uint32_t u = min(s, s + m.q);
  return min(u, u - m.q);
}

// The same for sums of at most kFewBlocks blocks, |T| <= 4 * 0.877e9 q < 0.82 q 2^32.  With the factor m of
// q signed the quotient of T - m q lies within (0.82 + 0.5) q, which one conditional correction by 2 q and one by q take
// to [0, q); one 64-bit multiply-add gives it (256 -> 1024 at 2^14 and 4 limbs: 294 -> 281 us, 128 -> 512: 92 -> 89).
__device__ __forceinline__ uint32_t reduce_few(int64_t t, const Modulus& m) {
  const int32_t k = static_cast<int32_t>(static_cast<uint32_t>(t) * m.qinv);
  const uint32_t h = static_cast<uint32_t>((t - static_cast<int64_t>(k) * static_cast<int32_t>(m.q)) >> 32);
  const uint32_t u = min(h, h + 2 * m.q);
  return min(u, u - m.q);
}

// Which of its row tile's outputs a lane has.
//   kRows     residues times weights: row l % 32, and of the 32 columns 4 (l / 32) + 8 i + 0 .. 3.
//   kColumns  weights times residues: column l % 32, rows 4 (l / 32) + 8 i + 0 .. 3.  Stores fill whole lines and can pass
//             the caches by, but scales are 16 times as many registers.
//   kFew      kColumns for at most 8 rows: the rows of i = 0 alone, a quarter of the steps that close a block and an
//             output (52 requests of 11 -> 1 at 2^16 and 3 limbs: 479 -> 388 us).
enum Form { kRows, kColumns, kFew };
constexpr uint32_t kFewRows = 8;
template <Form kForm>
constexpr int kOuts = kForm == kFew ? 4 : 16;

template <Form kForm>
__device__ __forceinline__ v16i product(v4i x, v4i w, v16i m) {
  return kForm == kRows ? __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w, m, 0, 0, 0)
                        : __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, m, 0, 0, 0);
}

// A lane's three scale constants of a block, for each of its rows.
template <Form kForm>
struct Scales {
  int32_t of[3][kForm == kRows ? 1 : kOuts<kForm>];
  __device__ __forceinline__ void load(const int32_t* block) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if constexpr (kForm == kRows) {
        of[i][0] = block[i * 32 + (threadIdx.x & 31)];
      } else {
#pragma unroll
        for (int r4 = 0; r4 < kOuts<kForm> / 4; ++r4) {
          const v4i v = *reinterpret_cast<const v4i*>(block + i * 32 + 8 * r4 + 4 * ((threadIdx.x >> 5) & 1));
#pragma unroll
          for (int r = 0; r < 4; ++r) of[i][4 * r4 + r] = v[r];
        }
      }
    }
  }
};

// A block's digit sums, times its scales, onto the 64-bit sums.
template <Form kForm>
__device__ __forceinline__ void combine(const v16i (&m)[kPairs], const Scales<kForm>& sc, int64_t (&acc)[kOuts<kForm>]) {
#pragma unroll
  for (int r = 0; r < kOuts<kForm>; ++r) {
    const int k = kForm == kRows ? 0 : r;
    acc[r] += static_cast<int64_t>(sc.of[0][k]) * (m[0][r] + (m[1][r] << 8));
    acc[r] += static_cast<int64_t>(sc.of[1][k]) * (m[2][r] + (m[3][r] << 8));
    acc[r] += static_cast<int64_t>(sc.of[2][k]) * m[4][r];
  }
}

template <int kN>
__device__ __forceinline__ void clear(int64_t (&acc)[kN]) {
#pragma unroll
  for (int r = 0; r < kN; ++r) acc[r] = 0;
}

template <bool kFewOf = false, int kN>
__device__ __forceinline__ void reduce(const int64_t (&acc)[kN], const Modulus& q, uint32_t (&y)[kN]) {
#pragma unroll
  for (int r = 0; r < kN; ++r) y[r] = kFewOf ? reduce_few(acc[r], q) : reduce(acc[r], q);
}

// The sum so far, reduced, goes on as a product.
template <int kN>
__device__ __forceinline__ void fold(const Modulus& q, int32_t c32, int64_t (&acc)[kN]) {
#pragma unroll
  for (int r = 0; r < kN; ++r) acc[r] = static_cast<int64_t>(static_cast<int32_t>(reduce(acc[r], q))) * c32;
}

// Where a wave finds a row tile's weights.
struct Source {
  rsrc_t frag;
  const int32_t* scales;
};
__device__ __forceinline__ Source source_of(const Layers& a, const Job& job, uint32_t tile) {
  return {__builtin_amdgcn_make_buffer_rsrc(const_cast<v4i*>(job.frag) + static_cast<size_t>(tile) * a.sh.steps * (kDigits * 64), 0,
                                            static_cast<int>(a.sh.steps * kDigits * 1024), kRsrcWord3),
          job.scales + static_cast<size_t>(tile) * a.sh.blocks * 96};
}

// A wave's weights and scales of one block.  They are loaded again, for the block after the next, as soon as they are
// used, so that two blocks' contractions cover the loads (and the residues' before them, since a wave's loads are
// waited for in order); steps past the layer's last read as zero through the buffer range check.
template <Form kForm>
struct Weights {
  v4i w[kBlockSteps][kDigits];
  Scales<kForm> sc;
  __device__ __forceinline__ void load_step(const Source& src, uint32_t block, uint32_t s) {
    const uint32_t at = (block * kBlockSteps + s) * (kDigits * 1024) + (threadIdx.x & 63) * 16;
#pragma unroll
    for (int d = 0; d < kDigits; ++d) w[s][d] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(src.frag, at + d * 1024, 0, 0);
  }
  __device__ __forceinline__ void load_scales(const Source& src, uint32_t block, uint32_t blocks) {
    sc.load(src.scales + static_cast<size_t>(min(block, blocks - 1)) * 96);
  }
};

// Residue digits of a step, from LDS.
__device__ __forceinline__ void read(const v4i* f, v4i (&x)[4]) {
#pragma unroll
  for (int b = 0; b < 4; ++b) x[b] = f[b * 64];
}

// One block of `steps` steps, none included, whose residues are at `f` (the first step's already in x): its digit sums,
// and onto the 64-bit sums.  A digit of the next step's residues is read as soon as this step's is used, those at
// `f_next` during the last one; the weights of block `after` of `next` take the place of those used.
__device__ __forceinline__ void contract(const v4i* f, uint32_t steps, const v4i* f_next, const Source& next, uint32_t after,
                                         uint32_t blocks, Weights<kRows>& w, v4i (&x)[4], int64_t (&acc)[16]) {
  v16i m[kPairs];
#pragma unroll
  for (uint32_t s = 0; s < kBlockSteps; ++s) {
    if (s < steps) {
      const v4i* ahead = s + 1 < kBlockSteps ? f + (s + 1) * kStepFrags : f_next;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int d = kDigits - 1; d >= 0; --d) {
          const bool first = s == 0 && (b == 0 || d == 1);  // of sum b + d
          m[b + d] = product<kRows>(x[b], w.w[s][d], first ? v16i{} : m[b + d]);
        }
        x[b] = ahead[b * 64];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    w.load_step(next, after, s);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (steps != 0) combine<kRows>(m, w.sc, acc);
  w.load_scales(next, after, blocks);
}

// LDS accesses of a wave's lanes before it come before those after it: the hardware keeps a wave's order, the compiler
// would not.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A row tile's outputs; rows past d_out are out of range.  With kRows through the wave's 4 KiB of LDS at `turn`.
template <Form kForm>
__device__ __forceinline__ void store(uint32_t* dst, uint32_t bytes, uint32_t d_out, uint32_t tile,
                                      const uint32_t (&y)[kOuts<kForm>], v4i* turn = nullptr) {
  uint32_t lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // else the addresses below are kept in registers, and others are spilled
  const uint32_t row0 = tile * 32;
  const uint32_t rows = min(d_out - row0, 32u);
  const rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(dst + static_cast<size_t>(row0) * (bytes >> 2), 0,
                                                       static_cast<int>(rows * bytes), kRsrcWord3);
  if constexpr (kForm != kRows) {  // past the caches: 16 -> 512 at 2^14 and 4 limbs 66 -> 57 us; partial lines so, 269
#pragma unroll
    for (int r = 0; r < kOuts<kForm>; ++r)
      __builtin_amdgcn_raw_buffer_store_b32(y[r], out, (8 * (r / 4) + 4 * (lane >> 5) + r % 4) * bytes + (lane & 31) * 4, 0,
                                            kNonTemporal);
  } else {  // lanes exchange rows and columns through LDS: 16-byte piece k of row r is at k ^ (r % 8), free of bank conflicts
    const uint32_t row = lane & 31, h = lane >> 5;
#pragma unroll
    for (uint32_t r4 = 0; r4 < 4; ++r4)
      turn[row * 8 + ((2 * r4 + h) ^ (row & 7))] = v4i{static_cast<int>(y[4 * r4]), static_cast<int>(y[4 * r4 + 1]),
                                                       static_cast<int>(y[4 * r4 + 2]), static_cast<int>(y[4 * r4 + 3])};
    wave_fence();
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t r = 8 * i + (lane >> 3), k = lane & 7;
      __builtin_amdgcn_raw_buffer_store_b128(turn[r * 8 + (k ^ (r & 7))], out, r * bytes + k * 16, 0, kNonTemporal);
    }
    wave_fence();
  }
}

// Onto the sums of a workgroup's lower waves those of its upper half's, through LDS [waves / 2][outputs / 4][64], and so on
// until the first waves / slices have the sums of all.
template <int kN>
__device__ __forceinline__ void join(uint32_t (&y)[kN], uint32_t q, v4i* sums, uint32_t wave, uint32_t waves, uint32_t slices) {
  for (uint32_t half = waves / 2; slices > 1; half /= 2, slices /= 2) {
    v4i* at = sums + (wave % half) * (kN / 4 * 64) + (threadIdx.x & 63);
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int r4 = 0; r4 < kN / 4; ++r4) {
        v4i v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = static_cast<int>(y[4 * r4 + r]);
        at[r4 * 64] = v;
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int r4 = 0; r4 < kN / 4; ++r4) {
        const v4i v = at[r4 * 64];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[4 * r4 + r] = add_mod(y[4 * r4 + r], static_cast<uint32_t>(v[r]), q);
      }
    }
    if (slices > 2) __syncthreads();
  }
  wave_fence();  // the sums' place, a wave's own by now, is written again
}

// A wave has 32 columns, one row tile and one of `slices` shares of the blocks, and its residues go from memory to
// registers to the matrix cores: a lane's digits of 16 inputs of one column are its operand, so there is no LDS and
// nothing to wait for but the loads, of which those of four steps are in flight.
constexpr int kThinWaves = 8;  // of a workgroup, at most
template <Form kForm>
__global__ __launch_bounds__(kThinWaves * 64, 2) void mac_fp8_thin_kernel(Tables tb, Layers a, uint32_t slices) {
  __shared__ v4i sums[kThinWaves * kOuts<kForm> * 16];
  Job job;
  const uint32_t waves = blockDim.x / 64, strips = waves / slices;
  if (!place_of(tb, a, strips * 32, a.sh.tiles, range_of(gridDim.x).first, &job)) return;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), strip = wave % strips, slice = wave / strips;
  const uint32_t blocks = a.sh.blocks, each = (blocks + slices - 1) / slices, steps = a.sh.steps;
  const uint32_t begin = min(blocks, slice * each), end = min(blocks, begin + each);
  const Modulus q = modulus(tb.q[job.limb]);
  const int32_t c32 = centred(tb.pow256[job.limb * 8 + 4], q.q);
  const Source src = source_of(a, job, job.split);
  job.src += strip * 32;
  uint32_t x[kBlockSteps][16];
  Weights<kForm> w;
#pragma unroll
  for (uint32_t s = 0; s < kBlockSteps; ++s)
    // Always so, a layer of one block has its own kernel; but a branch keeps the compiler from mixing the steps' loads (1000 -> 8 at
    // 2^14 and 4 limbs: 92.0 us with it, 94.3 without, 94.0 with a scheduling barrier in its place; 300 -> 5: 33.8, 35.1, 34.1).
    if (s == 0 || s < steps) {
      fetch_step(tb, a, job.src, (begin * kBlockSteps + s) * kStep, x[s]);
      w.load_step(src, begin, s);
    }
  w.load_scales(src, begin, blocks);
  int64_t acc[kOuts<kForm>];
  clear(acc);
  for (uint32_t g = begin; g < end; ++g) {
    if (g != begin && (g - begin) % kFoldBlocks == 0) fold(q, c32, acc);
    const uint32_t left = steps - g * kBlockSteps;
    const bool more = g + 1 < end;
    v16i m[kPairs];
#pragma unroll
    for (uint32_t s = 0; s < kBlockSteps; ++s) {
      if (s < left) {
        v4i f[4];
        to_fragments(x[s], f);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int d = kDigits - 1; d >= 0; --d) {
            const bool first = s == 0 && (b == 0 || d == 1);
            m[b + d] = product<kForm>(f[b], w.w[s][d], first ? v16i{} : m[b + d]);
          }
      }
      if (more) {
        fetch_step(tb, a, job.src, ((g + 1) * kBlockSteps + s) * kStep, x[s]);
        w.load_step(src, g + 1, s);
      }
    }
    combine<kForm>(m, w.sc, acc);
    if (more) w.load_scales(src, g + 1, blocks);
  }
  uint32_t y[kOuts<kForm>];
  reduce(acc, q, y);
  join(y, q.q, sums, wave, waves, slices);
  if (slice == 0) store<kForm>(job.dst + strip * 32, row_bytes(tb, a), a.d_out, job.split, y, sums + wave * (kOuts<kForm> * 16));
}

// One block of inputs: a wave converts its 32 columns once, keeps their digits in registers and goes through the row tiles
// of its split, the next tile's weights in flight (its scales would be 48 registers more).  No LDS, and nothing that waves
// wait for together (64 -> 256 at 2^14 and 4 limbs: 39 us; as chunks through LDS 72).
constexpr int kShortWaves = 4;  // of a workgroup, next to each other
template <int kSteps, Form kForm>
__global__ __launch_bounds__(kShortWaves * 64, 2) void mac_fp8_short_kernel(Tables tb, Layers a, uint32_t splits) {
  Job job;
  if (!place_of(tb, a, kShortWaves * 32, splits, range_of(gridDim.x).first, &job)) return;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tiles = a.sh.tiles;
  const uint32_t each = (tiles + splits - 1) / splits, begin = job.split * each, end = min(tiles, begin + each);
  if (begin >= end) return;
  const Modulus q = modulus(tb.q[job.limb]);
  job.src += wave * 32;
  job.dst += wave * 32;
  Weights<kForm> w;
  auto load = [&](uint32_t tile) {
    const Source src = source_of(a, job, tile);
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) w.load_step(src, 0, s);
  };
  v4i f[kSteps][4];
  {
    uint32_t x[kSteps][16];
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) fetch_step(tb, a, job.src, s * kStep, x[s]);
    load(begin);
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) to_fragments(x[s], f[s]);
  }
  for (uint32_t tile = begin; tile < end; ++tile) {
    w.load_scales(source_of(a, job, tile), 0, 1);
    v16i m[kPairs];
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s)
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int d = kDigits - 1; d >= 0; --d) {
          const bool first = s == 0 && (b == 0 || d == 1);
          m[b + d] = product<kForm>(f[s][b], w.w[s][d], first ? v16i{} : m[b + d]);
        }
    load(min(tile + 1, end - 1));
    int64_t acc[kOuts<kForm>];
    clear(acc);
    combine<kForm>(m, w.sc, acc);
    uint32_t y[kOuts<kForm>];
    reduce<true>(acc, q, y);
    store<kForm>(job.dst, row_bytes(tb, a), a.d_out, tile, y);
  }
}

// A workgroup has kColWaves tiles of 32 columns and 8 / kColWaves row tiles, a wave one of each, and goes through
// jobs and their chunks of two blocks of inputs without a pause: the next chunk's residues, of this job or the
// next, are in flight in registers while the matrix cores work on this one's out of the other half of the LDS.
template <int kColWaves>
__global__ __launch_bounds__(512, 2) void mac_fp8_chunked_kernel(Tables tb, Layers a, uint32_t splits, uint32_t jobs) {
  constexpr int kWaves = 8, kPasses = kChunk * kColWaves / kWaves;  // a pass a chunk, or one a block
  constexpr uint32_t kCols = kColWaves * 32;
  static_assert(kFoldBlocks % kChunkBlocks == 0, "reductions between chunks");
  __shared__ v4i lds[2][kColWaves * kChunk * kStepFrags];
  __shared__ v4i turn[kWaves * 256];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col_wave = wave % kColWaves, row_wave = wave / kColWaves;
  const uint32_t tiles = a.sh.tiles, each = (tiles + splits - 1) / splits;
  Jobs list{range_of(jobs)};
  auto seek = [&](Job* job) { return list.next(tb, a, kCols, splits, job); };
  Job job;
  if (!seek(&job)) return;
  const uint32_t steps = a.sh.steps, blocks = a.sh.blocks, bytes = row_bytes(tb, a);
  // waves without a row tile in a job's last split contract the last tile again, so that no weights are merged from two
  // paths, which costs registers; those without one in any have no steps
  auto source = [&](const Job& j) { return source_of(a, j, min(j.split * each + row_wave, tiles - 1)); };
  const uint32_t my_steps = row_wave < each ? steps : 0;
  Stage<kWaves, kColWaves> stage;
  Weights<kRows> w[kChunkBlocks];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    stage.fetch(tb, a, job, 0, p);
    stage.place(lds[0], p);
  }
  Source src = source(job);
#pragma unroll
  for (uint32_t g = 0; g < kChunkBlocks; ++g) {
#pragma unroll
    for (uint32_t s = 0; s < kBlockSteps; ++s) w[g].load_step(src, g, s);
    w[g].load_scales(src, g, blocks);
  }
  __syncthreads();
  uint32_t buf = 0;
  for (bool going = true; going;) {
    const Modulus q = modulus(tb.q[job.limb]);
    const int32_t c32 = centred(tb.pow256[job.limb * 8 + 4], q.q);
    const uint32_t tile = job.split * each + row_wave;
    int64_t acc[16];
    clear(acc);
    Job after = job;
    for (uint32_t g0 = 0; g0 < blocks; g0 += kChunkBlocks, buf ^= 1) {
      const bool last = g0 + kChunkBlocks >= blocks;
      if (last) {
        going = seek(&after);
        src = source(after);
      }
      // where the next chunk begins; past the last job's end there is nothing to fetch
      const uint32_t g1 = last ? 0 : g0 + kChunkBlocks, s0 = g0 * kBlockSteps, s1 = !last || going ? g1 * kBlockSteps : steps;
      const v4i* f = lds[buf] + col_wave * kChunk * kStepFrags + (threadIdx.x & 63);
      v4i x[4];
      stage.fetch(tb, a, after, s1, 0);
      if (g0 != 0 && g0 % kFoldBlocks == 0) fold(q, c32, acc);
      read(f, x);
      contract(f, max(my_steps, s0) - s0, f + kBlockSteps * kStepFrags, src, g1, blocks, w[0], x, acc);
      if (kPasses == 2) {
        stage.place(lds[buf ^ 1], 0);
        stage.fetch(tb, a, after, s1, 1);
      }
      f += kBlockSteps * kStepFrags;
      contract(f, max(my_steps, s0 + kBlockSteps) - (s0 + kBlockSteps), f, src, g1 + 1, blocks, w[1], x, acc);
      if (last && row_wave < each && tile < tiles) {
        uint32_t y[16];
        reduce(acc, q, y);
        store<kRows>(job.dst + col_wave * 32, bytes, a.d_out, tile, y, turn + wave * 256);
      }
      stage.place(lds[buf ^ 1], kPasses - 1);
      __syncthreads();
    }
    job = after;
  }
}

// Inputs whose digits all fit the LDS: a workgroup converts its columns once a job and its waves walk the row tiles of
// the job's split, kWaves apart, with nothing to wait for but their weights.  The next job's residues are converted
// meanwhile: where the LDS has room for both (kTwice) a piece with each chunk, from the first on, and one barrier a
// job; else during the last pass, when a chunk's place is given to them as soon as every wave is through with it.
//
// The row tiles that are no multiple of kWaves come first.  Where they are at most half of it (and others
// follow) two waves take a tile's chunks half and half and their sums meet in LDS.
// Four waves have at most kFewBlocks blocks, eight at most kFoldBlocks, so the sums need no reduction on the way.
template <int kWaves, bool kTwice>
__global__ __launch_bounds__(kWaves * 64, 2) void mac_fp8_whole_kernel(Tables tb, Layers a, uint32_t splits, uint32_t jobs) {
  constexpr int kPasses = kChunk / kWaves;
  static_assert(kPasses == 1 || kPasses == 2, "a pass a chunk, or one a block");
  constexpr uint32_t kChunkFrags = kChunk * kStepFrags;
  extern __shared__ v4i lds[];  // [chunks][kChunkFrags], with kTwice twice, then [kWaves][256]
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles = a.sh.tiles, each = (tiles + splits - 1) / splits, passes = (each + kWaves - 1) / kWaves;
  const uint32_t rest = each - (passes - 1) * kWaves;  // row tiles of the first pass
  Jobs list{range_of(jobs)};
  auto seek = [&](Job* job) { return list.next(tb, a, 32, splits, job); };
  Job job;
  if (!seek(&job)) return;
  const uint32_t steps = a.sh.steps, blocks = a.sh.blocks, bytes = row_bytes(tb, a);
  const uint32_t chunks = (blocks + kChunkBlocks - 1) / kChunkBlocks;
  // the wave's row tile of a pass, counted in the split, and its chunks
  const bool joins = passes > 1 && rest <= kWaves / 2 && chunks > 1, upper = joins && wave >= kWaves / 2;
  const uint32_t at0 = upper ? wave - kWaves / 2 : wave, half = joins ? (chunks + 1) / 2 : chunks;
  const uint32_t begin0 = upper ? half : 0, end0 = upper ? chunks : half;
  auto at_of = [&](uint32_t pass) { return pass == 0 ? at0 : rest + (pass - 1) * kWaves + wave; };
  auto source = [&](const Job& j, uint32_t at) { return source_of(a, j, min(j.split * each + at, tiles - 1)); };
  const uint32_t pieces = chunks * kPasses, strip = chunks * kChunkFrags;
  v4i *const sums = lds + (kTwice ? 2 : 1) * strip, *whole = lds, *other = lds + strip;
  Stage<kWaves, 1> stage;
  Weights<kRows> w[kChunkBlocks];
  for (uint32_t g0 = 0; g0 < blocks; g0 += kChunkBlocks)
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      stage.fetch(tb, a, job, g0 * kBlockSteps, p);
      stage.place(whole + g0 / kChunkBlocks * kChunkFrags, p);
    }
  Source src = source(job, at0);
#pragma unroll
  for (uint32_t g = 0; g < kChunkBlocks; ++g) {
#pragma unroll
    for (uint32_t s = 0; s < kBlockSteps; ++s) w[g].load_step(src, begin0 * kChunkBlocks + g, s);
    w[g].load_scales(src, begin0 * kChunkBlocks + g, blocks);
  }
  __syncthreads();
  for (bool going = true; going;) {
    const Modulus q = modulus(tb.q[job.limb]);
    Job after = job;
    if (kTwice) going = seek(&after);
    const uint32_t wanted = kTwice && going ? pieces : 0;
    uint32_t fetched = 0, placed = 0;  // pieces of the next job
    auto place_piece = [&] {
      stage.place(other + placed / kPasses * kChunkFrags, placed % kPasses);
      ++placed;
    };
    auto fetch_piece = [&] {
      stage.fetch(tb, a, after, fetched / kPasses * kChunk, fetched % kPasses);
      ++fetched;
    };
    for (uint32_t pass = 0; pass < passes; ++pass) {
      const uint32_t at = at_of(pass), tile = job.split * each + at;
      const bool last = pass + 1 == passes, works = (pass != 0 || at < rest) && tile < tiles;
      const uint32_t my_steps = works ? steps : 0, begin = pass == 0 ? begin0 : 0, end = pass == 0 ? end0 : chunks;
      if (!kTwice && last) going = seek(&after);
      int64_t acc[16];
      clear(acc);
      for (uint32_t c = begin; c < end; ++c) {
        if (c + 1 == end) src = last ? source(after, at0) : source(job, at_of(pass + 1));
        const uint32_t g0 = c * kChunkBlocks, g1 = c + 1 < end ? g0 + kChunkBlocks : last ? begin0 * kChunkBlocks : 0;
        const uint32_t s0 = g0 * kBlockSteps, s1 = going ? s0 : steps;
        v4i* chunk = whole + c * kChunkFrags;
        const v4i* f = chunk + (threadIdx.x & 63);
        v4i x[4];
        if (!kTwice && last) stage.fetch(tb, a, after, s1, 0);
        if (kTwice) {
          if (placed < fetched) place_piece();
          if (fetched < wanted) fetch_piece();
        }
        read(f, x);
        contract(f, max(my_steps, s0) - s0, f + kBlockSteps * kStepFrags, src, g1, blocks, w[0], x, acc);
        if (!kTwice && kPasses == 2 && last) {
          __syncthreads();
          stage.place(chunk, 0);
          stage.fetch(tb, a, after, s1, 1);
        }
        f += kBlockSteps * kStepFrags;
        contract(f, max(my_steps, s0 + kBlockSteps) - (s0 + kBlockSteps), f, src, g1 + 1, blocks, w[1], x, acc);
        if (!kTwice && last) {
          __syncthreads();
          stage.place(chunk, kPasses - 1);
        }
      }
      uint32_t y[16];
      reduce<kWaves == 4>(acc, q, y);
      if (joins && pass == 0) join(y, q.q, sums, wave, kWaves, 2);
      if (works && !(upper && pass == 0)) store<kRows>(job.dst, bytes, a.d_out, tile, y, sums + wave * 256);
    }
    if (kTwice) {
      while (placed < wanted) {
        if (placed == fetched) fetch_piece();
        place_piece();
      }
      v4i* const done = whole;
      whole = other;
      other = done;
    }
    __syncthreads();
    job = after;
  }
}

// Zeros, for layers without inputs.
__global__ __launch_bounds__(kThreads) void experts_zero_kernel(Tables tb, Layers a, uint32_t count) {
  const size_t words = static_cast<size_t>(a.d_out) * 2 * a.limbs * tb.n;
  for (uint32_t r = blockIdx.y; r < count; r += gridDim.y) {
    uint32_t e, b;
    const bool good = named(a, r, &e, &b);
    if (a.status && blockIdx.x == 0 && threadIdx.x == 0) a.status[r] = good ? kExpertOk : kExpertBadRequest;
    if (!good) continue;
    for (size_t i = static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x; i < words; i += static_cast<size_t>(gridDim.x) * kThreads)
      a.ct_out[r * words + i] = 0;
  }
}

uint32_t ceil_div(uint64_t a, uint32_t b) { return static_cast<uint32_t>((a + b - 1) / b); }

hipError_t launch_thin(const Tables& t, const Layers& a, uint64_t waves, hipStream_t s) {
  uint32_t slices = 1;  // up to eight waves a CU, as many as run at a time (1024 -> 16 at 2^13, 3 limbs, twelve : six, 48.9 : 42.6 us)
  while (slices < kThinWaves && 2 * slices <= a.sh.blocks && 2 * waves * slices <= t.num_cus * 8ull) slices *= 2;
  const uint32_t group = slices < 4 ? 4 : slices;  // waves of a workgroup
  const uint32_t grid = static_cast<uint32_t>(waves * slices / group);
  const auto k = a.d_out <= kFewRows ? mac_fp8_thin_kernel<kFew> : mac_fp8_thin_kernel<kRows>;
  k<<<grid, group * 64, 0, s>>>(t, a, slices);
  return hipGetLastError();
}

hipError_t launch_short(const Tables& t, const Layers& a, uint64_t strips, hipStream_t s) {
  // eight waves a CU where the row tiles allow it
  const uint32_t splits = static_cast<uint32_t>(std::min<uint64_t>(a.sh.tiles, (t.num_cus * 8ull + strips - 1) / strips));
  const uint32_t grid = static_cast<uint32_t>(strips / kShortWaves * splits);
  const auto k = a.d_out <= kFewRows ? (a.sh.steps == 1   ? mac_fp8_short_kernel<1, kFew>
                                        : a.sh.steps == 2 ? mac_fp8_short_kernel<2, kFew>
                                                          : mac_fp8_short_kernel<4, kFew>)
                                     : (a.sh.steps == 1   ? mac_fp8_short_kernel<1, kColumns>
                                        : a.sh.steps == 2 ? mac_fp8_short_kernel<2, kColumns>
                                                          : mac_fp8_short_kernel<4, kColumns>);
  k<<<grid, kShortWaves * 64, 0, s>>>(t, a, splits);
  return hipGetLastError();
}

template <int kColWaves>
hipError_t launch_chunked(const Tables& t, const Layers& a, uint64_t strips, hipStream_t s) {
  const uint32_t splits = ceil_div(a.sh.tiles, 8 / kColWaves);
  const uint64_t jobs = strips / kColWaves * splits;
  if (jobs > 0x7FFFFFFFull) return hipErrorInvalidConfiguration;
  mac_fp8_chunked_kernel<kColWaves><<<static_cast<uint32_t>(std::min<uint64_t>(jobs, t.num_cus)), 512, 0, s>>>(
      t, a, splits, static_cast<uint32_t>(jobs));
  return hipGetLastError();
}

template <int kWaves>
hipError_t launch_whole(const Tables& t, const Layers& a, uint64_t strips, uint32_t splits, hipStream_t s) {
  const uint64_t jobs = strips * splits;
  if (jobs > 0x7FFFFFFFull) return hipErrorInvalidConfiguration;
  const uint32_t grid = static_cast<uint32_t>(std::min<uint64_t>(jobs, t.num_cus * (8 / kWaves)));
  const size_t strip = strip_bytes(a.sh), sums = kWaves * kWaveSums;
  const uint32_t n = static_cast<uint32_t>(jobs);
  if (a.sh.blocks > (kWaves == 4 ? kFewBlocks : kFoldBlocks)) return hipErrorInvalidConfiguration;
  if constexpr (kWaves == 4) {
    // two workgroups a CU; one strip or two (13 requests of 200 -> 333 at 2^11, 2 limbs, before the shorter reduction: 91 -> 88 us)
    if (2 * (2 * strip + sums) <= kLdsBytes)
      mac_fp8_whole_kernel<4, true><<<grid, 256, 2 * strip + sums, s>>>(t, a, splits, n);
    else
      mac_fp8_whole_kernel<4, false><<<grid, 256, strip + sums, s>>>(t, a, splits, n);
  } else {
    mac_fp8_whole_kernel<8, false><<<grid, 512, strip + sums, s>>>(t, a, splits, n);
  }
  return hipGetLastError();
}

// The time of the whole kernel in hundredths of that of a chunked job, and its row splits: rounds of jobs over the
// workgroups that fit the GPU, times `pass` for each pass over the row tiles and `fill` for the residues.
struct Plan {
  uint64_t time;
  uint32_t splits;
};
Plan plan_whole(const Tables& t, const Shape& sh, uint64_t strips, uint32_t waves, uint32_t pass, uint32_t fill) {
  Plan best{~0ull, 1};
  for (uint32_t splits = 1; splits <= 8 && splits <= sh.tiles; ++splits) {
    const uint32_t each = ceil_div(sh.tiles, splits), full = each / waves, rest = each % waves;
    const uint32_t halves = 2 * full + (rest == 0 ? 0 : full > 0 && rest <= waves / 2 && sh.steps > kChunk ? 1 : 2);
    const uint64_t rounds = ceil_div(strips * splits, t.num_cus * (8 / waves));
    const uint64_t time = rounds * (pass * halves / 2 + fill);
    if (time < best.time) best = {time, splits};
  }
  return best;
}

hipError_t launch(const Tables& t, const Layers& a, hipStream_t s) {
  const Shape& sh = a.sh;
  const uint64_t strips = static_cast<uint64_t>(a.count) * a.limbs * (2 * t.n / 32);
  if (sh.blocks == 1) return launch_short(t, a, strips, s);  // 2^14, 4 limbs, short : thin: 64 -> 256 39 : 72 us
  // No more than 32 outputs, or too few columns for the other kernels.  Thin : the best of the others, us, 2^14, 4 limbs:
  // 256 -> 16 31 : 41, 256 -> 64 48 : 45, 1024 -> 64 150 : 140; 2^10, 2 limbs: 512 -> 128 8.2 : 9.3, 1024 -> 256 16 : 18,
  // 1024 -> 512 27 : 19; 2^12, 2 limbs: 300 -> 64 10.3 : 10.9, 256 -> 256 18 : 13, 1024 -> 128 35 : 24.
  if (sh.tiles <= 1 || strips * sh.tiles <= t.num_cus * 4ull)
    return launch_thin(t, a, strips * sh.tiles, s);
  // A chunked job is 8 row tiles of one column tile or 4 of two; the others by a fit of their times.  2^14, 4 limbs, us, 4 x
  // 2 : 8 x 1 : whole (of four waves up to 512 inputs): 256 -> 128 58 : 70 : 62, 256 -> 256 101 : 97 : 94, 300 -> 333 190 :
  // 241 : 158, 512 -> 256 165 : 167 : 160, 512 -> 512 322 : 322 : 275, 1024 -> 256 298 : 302 : 310, 1024 -> 384 429 : 526 :
  // 425, 1024 -> 512 571 : 573 : 525; 2^15, 4 limbs, 1024 -> 2048 4530 : 4290 : 3640.
  const uint64_t wide = ceil_div(strips / 2 * ceil_div(sh.tiles, 4), t.num_cus) * 100ull;
  const uint64_t tall = ceil_div(strips * ceil_div(sh.tiles, 8), t.num_cus) * 100ull;
  const bool four = sh.blocks <= kFewBlocks;  // two workgroups' strips, and room for their outputs, fit the LDS
  static_assert(2 * (kFewBlocks * kBlockSteps * kStepFrags * 16 + 4 * kWaveSums) <= kLdsBytes, "two workgroups a CU");
  if (strip_bytes(sh) + 8 * kWaveSums <= kLdsBytes) {
    const Plan plan = four ? plan_whole(t, sh, strips, 4, 80, 38) : plan_whole(t, sh, strips, 8, 82, 23);
    if (plan.time < wide && plan.time < tall)
      return four ? launch_whole<4>(t, a, strips, plan.splits, s) : launch_whole<8>(t, a, strips, plan.splits, s);
  }
  return wide < tall ? launch_chunked<2>(t, a, strips, s) : launch_chunked<1>(t, a, strips, s);
}

}  // namespace

size_t fp8_weight_bytes(uint32_t d_out, uint32_t d_in, uint32_t limbs) {
  if (d_out == 0 || d_in == 0) return 0;
  const Shape s = shape_of(d_out, d_in, limbs);
  return s.frag_bytes + s.scale_bytes;
}

hipError_t launch_encode_fp8(const Tables& t, const uint8_t* w8, const float* scales, uint32_t d_out, uint32_t d_in,
                             uint32_t block_rows, uint32_t limbs, double scale, void* w_fp8, int32_t* bad, bool units,
                             int32_t* rounded, hipStream_t s) {
  const Shape sh = shape_of(d_out, d_in, limbs);
  uint8_t* base = static_cast<uint8_t*>(w_fp8);
  int32_t* constants = reinterpret_cast<int32_t*>(base + sh.frag_bytes);
  for (int32_t* count : {bad, rounded})
    if (count)
      if (hipError_t e = launch_zero(reinterpret_cast<uint32_t*>(count), 1, s); e != hipSuccess) return e;
  if (units) {
    const size_t total = static_cast<size_t>(sh.tiles) * sh.blocks * 32;
    hipError_t e = in_pieces((total + kThreads - 1) / kThreads, [&](uint64_t first, uint32_t groups) {
      fp8_unit_kernel<<<groups, kThreads, 0, s>>>(w8, d_out, d_in, sh.blocks, sh.tiles, limbs, total, first, constants);
    });
    if (e != hipSuccess) return e;
  }
  const size_t lanes = static_cast<size_t>(sh.tiles) * sh.steps * 64;
  const auto frag = units ? fp8_frag_kernel<true> : fp8_frag_kernel<false>;
  hipError_t e = in_pieces((lanes + kThreads - 1) / kThreads, [&](uint64_t first, uint32_t groups) {
    frag<<<groups, kThreads, 0, s>>>(w8, d_out, d_in, sh.steps, lanes, first, constants, bad, rounded, reinterpret_cast<v4i*>(base));
  });
  if (e != hipSuccess) return e;
  const size_t total = static_cast<size_t>(limbs) * sh.tiles * sh.blocks * 32;
  const auto constant = units ? fp8_scale_kernel<true> : fp8_scale_kernel<false>;
  return in_pieces((total + kThreads - 1) / kThreads, [&](uint64_t first, uint32_t groups) {
    constant<<<groups, kThreads, 0, s>>>(t, scales, d_out, block_rows, sh.blocks, sh.tiles, total, first, scale / 64, bad, constants);
  });
}

hipError_t launch_mac_fp8(const Tables& t, const void* w_fp8, uint32_t experts, const int32_t* expert,
                          const int32_t* bundle, uint32_t count, const uint32_t* ct_in, uint32_t bundles, uint32_t* ct_out,
                          uint32_t d_out, uint32_t d_in, uint32_t limbs, int32_t* status, hipStream_t s) {
  Layers a{static_cast<const uint8_t*>(w_fp8), fp8_weight_bytes(d_out, d_in, limbs), ct_in, ct_out, expert, bundle, status,
           experts, bundles, count, d_out, d_in, limbs, shape_of(d_out, d_in, limbs)};
  if (d_out == 0) {
    if (!status) return hipSuccess;
    experts_status_kernel<<<(count + kThreads - 1) / kThreads, kThreads, 0, s>>>(a, count);
    return hipGetLastError();
  }
  if (d_in == 0) {
    experts_zero_kernel<<<dim3(64, count < 1024 ? count : 1024), kThreads, 0, s>>>(t, a, count);
    return hipGetLastError();
  }
  // In pieces of as many requests as the short and the thin kernel have kMostGroups workgroups for, of four column strips and
  // one share of the row tiles each (of fewer strips, where there are many shares).
  const uint32_t most = kMostGroups / (limbs * (2 * t.n / 32) / 4);
  for (uint32_t r = 0; r < count; r += most) {
    Layers part = a;
    part.count = count - r < most ? count - r : most;
    part.ct_out += r * (static_cast<size_t>(2) * limbs * t.n * d_out);
    if (expert) part.expert += r;
    if (status) part.status += r;
    if (bundle) {
      part.bundle += r;
    } else {  // a request's own number
      part.ct_in += r * (static_cast<size_t>(2) * limbs * t.n * d_in);
      part.bundles = bundles > r ? bundles - r : 0;
    }
    if (const hipError_t e = launch(t, part, s); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ckks
