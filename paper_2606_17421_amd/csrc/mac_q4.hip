// ct x pt MAC over 4-bit weights with one scale (and zero point) per group of
// inputs (gfx950).
//
// Per limb l, with u the 4-bit weights, z the zero points (8 without them) and
// S = rint(scale Delta) of the group,
//     out[j][col] = sum_g S[j][g] T[j][g][col] mod q_l,
//     T[j][g][col] = sum over the group of (u[j][i] - z[j][g]) x[i][col].
// T needs only the small integers u, which are the same for every limb; the
// scale enters once a group.
#include "digits.hpp"

namespace ckks {
namespace {

typedef int v16i __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;        // encode kernels
constexpr uint32_t kStep = 32;       // inputs of one matrix-core step
constexpr uint32_t kCols = 32;       // columns of a workgroup
constexpr uint32_t kWaveRows = 64;   // output rows of a wave: two tiles of 32
constexpr int kStepFrags = 4 * 64;   // 16-byte residue fragments of a step: four digits, 64 lanes
constexpr uint32_t kFold = 1024;     // inputs after which the 64-bit sums are reduced

// Encoded weights:
//   fragments [tile][step][64 lanes] of 8 bytes: a 4-bit v of row tile*32 + lane%32
//     and inputs step*32 + 16 (lane/32) + i, i < 16; v = u - 8 in two's complement,
//     or u itself with zero points.  Word d holds i = 8d .. 8d + 7: the low halves of
//     its bytes the first four, the high halves the last four, so two masks give
//     four bytes 16 v each (8 u with zero points).  Rows are padded to kWaveRows, steps
//     to whole sub-groups.
//   scales [limb][tile][sub-group][32 rows] of {sa, sb} (with zero points {sa, sb, nz,
//     0}): sa = 2^32 S / 16, sb = 2^48 S / 16 mod q_l (/ 8 with zero points), centred;
//     nz = -8 z.  The 2^32 is what the closing reduction divides by.
// A sub-group is what one set of i32 sums covers: 128 or 64 inputs that divide
// the group, else 32; a group that holds every input is cut freely.
struct Shape {
  uint32_t tiles, steps, groups, sub_len, subs;
  size_t frag_bytes, scale_bytes;
};

Shape shape_of(uint32_t d_out, uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros) {
  Shape s;
  s.tiles = (d_out + kWaveRows - 1) / kWaveRows * (kWaveRows / 32);
  s.groups = (d_in + group - 1) / group;
  if (s.groups == 1)
    s.sub_len = d_in <= 32 ? 32 : d_in <= 64 ? 64 : 128;
  else
    s.sub_len = group % 128 == 0 ? 128 : group % 64 == 0 ? 64 : 32;
  s.subs = (d_in + s.sub_len - 1) / s.sub_len;
  s.steps = s.subs * (s.sub_len / kStep);
  s.frag_bytes = static_cast<size_t>(s.tiles) * s.steps * 64 * 8;
  s.scale_bytes = static_cast<size_t>(limbs) * s.tiles * s.subs * 32 * (zeros ? 16 : 8);
  return s;
}

__global__ __launch_bounds__(kThreads) void q4_frag_kernel(const uint8_t* __restrict__ w4, uint32_t d_out,
                                                           uint32_t d_in, uint32_t steps, size_t lanes,
                                                           uint32_t flip, uint2* __restrict__ frag) {
  const size_t idx = static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (idx >= lanes) return;
  const uint32_t lane = idx & 63;
  const uint32_t step = static_cast<uint32_t>((idx >> 6) % steps), tile = static_cast<uint32_t>((idx >> 6) / steps);
  const uint32_t row = tile * 32 + (lane & 31);
  const uint8_t* w = w4 + static_cast<size_t>(row) * ((d_in + 1) / 2);
  uint32_t word[2];
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const uint32_t k0 = step * kStep + 16 * (lane >> 5) + 8 * d;
    uint32_t v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = k0 + e;
      const uint32_t u = row < d_out && k < d_in ? (w[k >> 1] >> (4 * (k & 1))) & 15u : flip;
      v |= (u ^ flip) << (8 * (e & 3) + 4 * (e >> 2));  // flip 8: u ^ 8 is u - 8 in four bits
    }
    word[d] = v;
  }
  frag[idx] = make_uint2(word[0], word[1]);
}

__device__ __forceinline__ int32_t centred(uint32_t r, uint32_t q) {
  return r > (q >> 1) ? static_cast<int32_t>(r - q) : static_cast<int32_t>(r);
}

__global__ __launch_bounds__(kThreads) void q4_scale_kernel(Tables tb, const float* __restrict__ scales,
                                                            const uint8_t* __restrict__ zeros, uint32_t d_out,
                                                            uint32_t group, uint32_t groups, uint32_t sub_len,
                                                            uint32_t subs, uint32_t tiles, size_t total,
                                                            double scale, int32_t* __restrict__ out) {
  const size_t idx = static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x;  // [limb][tile][sub][32]
  if (idx >= total) return;
  const uint32_t sub = static_cast<uint32_t>((idx >> 5) % subs);
  const size_t lt = (idx >> 5) / subs;
  const uint32_t l = static_cast<uint32_t>(lt / tiles);
  const uint32_t row = static_cast<uint32_t>(lt % tiles) * 32 + (idx & 31);
  const uint32_t q = tb.q[l];
  int32_t sa = 0, sb = 0, nz = 0;
  if (row < d_out) {
    const size_t at = static_cast<size_t>(row) * groups + static_cast<uint32_t>(static_cast<size_t>(sub) * sub_len / group);
    uint32_t r = reduce_f64_int(rint(static_cast<double>(scales[at]) * scale), q, tb.q_recip[l]);
    r = static_cast<uint32_t>((static_cast<uint64_t>(r) << (zeros ? 29 : 28)) % q);  // 2^32 / 8 or 2^32 / 16
    sa = centred(r, q);
    sb = centred(static_cast<uint32_t>((static_cast<uint64_t>(r) << 16) % q), q);
    if (zeros) nz = -8 * static_cast<int32_t>(zeros[at] & 15u);
  }
  if (zeros)
    reinterpret_cast<int4*>(out)[idx] = make_int4(sa, sb, nz, 0);
  else
    reinterpret_cast<int2*>(out)[idx] = make_int2(sa, sb);
}

// Where a workgroup finds its part of the layer.
struct Job {
  const uint2* frag;       // the whole layer's
  const int32_t* scales;   // the limb's
  const uint32_t* src;     // input 0's word of column 0 of the workgroup
  uint32_t* dst;           // output 0's
  uint32_t row_bytes, d_out, d_in, steps, subs;
};

// 8 bytes of a weight fragment -> 16 bytes, 16 v each (8 u with zero points).
template <bool kZeros>
__device__ __forceinline__ v4i unpack(uint2 w) {
  constexpr uint32_t m = kZeros ? 0x78787878u : 0xf0f0f0f0u;
  constexpr int up = kZeros ? 3 : 4, down = kZeros ? 1 : 0;
  return v4i{static_cast<int>((w.x << up) & m), static_cast<int>((w.x >> down) & m), static_cast<int>((w.y << up) & m),
             static_cast<int>((w.y >> down) & m)};
}

// The residues of inputs from `first` on, `steps` steps of them, as digit fragments
// in LDS; inputs past d_in read as zero through the buffer range check.  Thread:
// one column, 16 consecutive inputs a pass.  With zero points also the
// sub-groups' sums of the residues' two low and two high digits.
template <int kSteps, bool kZeros>
__device__ __forceinline__ void fill(const Job& job, uint32_t first, uint32_t steps, v4i* lds, int32_t* sums) {
  constexpr int kPasses = 4;
  const uint32_t tid = threadIdx.x, col = tid & 31, kb = tid >> 5, blocks = blockDim.x >> 5;  // blocks of 16 inputs
  const uint32_t subs = steps / kSteps;
  if constexpr (kZeros) {
    for (uint32_t i = tid; i < subs * 2 * kCols; i += blockDim.x) sums[i] = 0;
    __syncthreads();
  }
  const uint32_t rows_pass = blocks * 16, row_words = job.row_bytes >> 2;
  for (uint32_t b0 = 0; b0 < 2 * steps; b0 += kPasses * blocks) {
    uint32_t x[kPasses][16];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const uint32_t base = first + (b0 + p * blocks) * 16;
      const uint32_t rows = base < job.d_in && b0 + p * blocks < 2 * steps ? min(job.d_in - base, rows_pass) : 0;
      const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint32_t*>(job.src) + (rows ? static_cast<size_t>(base) * row_words : 0), 0,
          static_cast<int>(rows * job.row_bytes), kRsrcWord3);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[p][i] = __builtin_amdgcn_raw_buffer_load_b32(rs, (kb * 16 + i) * job.row_bytes + col * 4, 0, 0);
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const uint32_t b = b0 + p * blocks + kb;
      if (b < 2 * steps) {
        v4i f[4];
        to_fragments(x[p], f);
#pragma unroll
        for (int d = 0; d < 4; ++d) lds[(b >> 1) * kStepFrags + d * 64 + col + 32 * (b & 1)] = f[d];
        if constexpr (kZeros) {
          int32_t lo = -16 * 0x8080, hi = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t y = x[p][i] + 0x8080u;
            lo += static_cast<int32_t>(y & 0xffffu);
            hi += static_cast<int32_t>(y >> 16);
          }
          const uint32_t sub = (b >> 1) / kSteps;
          atomicAdd(&sums[(sub * 2) * kCols + col], lo);
          atomicAdd(&sums[(sub * 2 + 1) * kCols + col], hi);
        }
      }
    }
  }
}

// T / 2^32 mod q in [0, q) for |T| < 2^61.8 (Montgomery's reduction): with m = T /
// q mod 2^32 the difference T - m q is a multiple of 2^32, its quotient hi(T) -
// hi(m q) in (-2^29.8 - q, 2^29.8); 3q (q > 2^29) makes it positive and below 4.74
// q < 2^32, and three conditional subtractions finish.  A contraction of kFold
// inputs stays below: |16 v| <= 128 times digit pairs of at most 128 * 257 and 128 +
// 64 * 256, times centred scales below 2^29, is 2^51.6 an input.
struct Modulus {
  uint32_t q, qinv;  // qinv = 1 / q mod 2^32
};
__device__ __forceinline__ Modulus modulus(uint32_t q) {
  uint32_t v = q;  // right mod 2^3 for odd q; each step doubles the bits
#pragma unroll
  for (int i = 0; i < 4; ++i) v *= 2u - q * v;
  return {q, v};
}
__device__ __forceinline__ uint32_t reduce(int64_t t, const Modulus& m) {
  const uint32_t k = static_cast<uint32_t>(t) * m.qinv;
  uint32_t u = static_cast<uint32_t>(t >> 32) - __umulhi(k, m.q) + 3 * m.q;
  u = min(u, u - 2 * m.q);
  u = min(u, u - m.q);
  return min(u, u - m.q);
}

// The wave's 64 rows over the sub-groups [sub0, sub0 + subs), whose residues lie in LDS.
template <int kSteps, bool kZeros>
__device__ __forceinline__ void contract(const Job& job, uint32_t tile0, uint32_t sub0, uint32_t subs, const v4i* lds,
                                         const int32_t* sums, int64_t (&acc)[2][16]) {
  const uint32_t lane = threadIdx.x & 63;
  constexpr int kScaleWords = kZeros ? 4 : 2;
  const uint2* wp[2];
  const int32_t* sp[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    wp[t] = job.frag + (static_cast<size_t>(tile0 + t) * job.steps + static_cast<size_t>(sub0) * kSteps) * 64;
    sp[t] = job.scales + (static_cast<size_t>(tile0 + t) * job.subs + sub0) * 32 * kScaleWords;
  }
  uint2 raw[kSteps][2];
  int2 sc[2];
  int32_t nz[2] = {0, 0};
  auto load = [&](uint32_t g) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) raw[s][t] = wp[t][(g * kSteps + s) * 64 + lane];
      const int32_t* p = sp[t] + (g * 32 + (lane & 31)) * kScaleWords;
      if constexpr (kZeros) {
        const int4 v = *reinterpret_cast<const int4*>(p);
        sc[t] = make_int2(v.x, v.y);
        nz[t] = v.z;
      } else {
        sc[t] = *reinterpret_cast<const int2*>(p);
      }
    }
  };
  load(0);
  for (uint32_t g = 0; g < subs; ++g) {
    v4i w[kSteps][2];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) w[s][t] = unpack<kZeros>(raw[s][t]);
    const int2 sg[2] = {sc[0], sc[1]};
    const int32_t zg[2] = {nz[0], nz[1]};
    if (g + 1 < subs) load(g + 1);
    const v4i* f = lds + static_cast<size_t>(g) * kSteps * kStepFrags + lane;
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // digits 0 and 1, then 2 and 3
      v16i m[2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < 2; ++d) m[t][d] = v16i{};
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const v4i x = f[s * kStepFrags + (2 * half + d) * 64];
#pragma unroll
          for (int t = 0; t < 2; ++t) m[t][d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w[s][t], m[t][d], 0, 0, 0);
        }
      v4i xs[4];
      if constexpr (kZeros) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          xs[r] = *reinterpret_cast<const v4i*>(sums + (g * 2 + half) * kCols + 8 * r + 4 * (lane >> 5));
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int32_t sv = half ? sg[t].y : sg[t].x;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          int32_t a = m[t][0][r] + (m[t][1][r] << 8);
          if constexpr (kZeros) a += __mul24(zg[t], xs[r >> 2][r & 3]);
          acc[t][r] += static_cast<int64_t>(sv) * a;
        }
      }
    }
  }
}

// chunk: steps of inputs held in LDS at a time (a multiple of the sub-group's).
// The workgroup's waves take its 64-row groups [rg0, rg1) in turn.
template <int kSteps, bool kZeros>
__global__ __launch_bounds__(512, 1) void mac_q4_kernel(Tables tb, const uint2* __restrict__ frag,
                                                        const int32_t* __restrict__ scales,
                                                        const uint32_t* __restrict__ ct_in,
                                                        uint32_t* __restrict__ ct_out, uint32_t d_out, uint32_t d_in,
                                                        uint32_t limbs, uint32_t steps, uint32_t subs, uint32_t tiles,
                                                        uint32_t tiles_n, uint32_t splits, uint32_t chunk) {
  extern __shared__ v4i lds[];
  int32_t* sums = reinterpret_cast<int32_t*>(lds + static_cast<size_t>(chunk) * kStepFrags);
  // Consecutive workgroup ids alternate XCDs: each XCD takes a contiguous range
  // of (limb, column tile, row split), so that workgroups which share columns or
  // weights meet in one L2.
  const uint32_t G = gridDim.x;
  uint32_t lid = blockIdx.x;
  if ((G & 7u) == 0) lid = (lid & 7u) * (G >> 3) + (lid >> 3);
  const uint32_t split = lid % splits, lc = lid / splits;
  const uint32_t l = lc / tiles_n, ntile = lc - l * tiles_n;
  const uint32_t n = tb.n, col0 = ntile * kCols, c = col0 >> tb.log_n, k0 = col0 & (n - 1);
  const size_t at = (static_cast<size_t>(c) * limbs + l) * n + k0;
  const Job job = {frag, scales + static_cast<size_t>(l) * tiles * subs * 32 * (kZeros ? 4 : 2), ct_in + at, ct_out + at,
                   2u * limbs * n * 4u, d_out, d_in, steps, subs};
  const Modulus q = modulus(tb.q[l]);
  const uint32_t waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t groups = tiles / 2, each = (groups + splits - 1) / splits;
  const uint32_t rg0 = split * each, rg1 = min(groups, rg0 + each);
  const bool whole = chunk >= steps;
  if (whole) {
    fill<kSteps, kZeros>(job, 0, steps, lds, sums);
    __syncthreads();
  }
  for (uint32_t rb = rg0; rb < rg1; rb += waves) {
    const uint32_t rg = rb + wave;
    int64_t acc[2][16];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0;
    if (whole) {
      if (rg >= rg1) break;
      contract<kSteps, kZeros>(job, rg * 2, 0, subs, lds, sums, acc);
    } else {
      for (uint32_t s0 = 0; s0 < steps; s0 += chunk) {
        const uint32_t here = min(chunk, steps - s0);
        __syncthreads();  // the chunk before is read out
        fill<kSteps, kZeros>(job, s0 * kStep, here, lds, sums);
        __syncthreads();
        if (rg < rg1) {
          if (s0 != 0) {  // the sum so far, reduced, goes on as a product below 2^59
            const int32_t c32 = centred(tb.pow256[l * 8 + 4], q.q);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                acc[t][r] = static_cast<int64_t>(static_cast<int32_t>(reduce(acc[t][r], q))) * c32;
          }
          contract<kSteps, kZeros>(job, rg * 2, s0 / kSteps, here / kSteps, lds, sums, acc);
        }
      }
      if (rg >= rg1) continue;
    }
    const uint32_t row0 = rg * kWaveRows, rows = min(d_out - row0, kWaveRows);
    const rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(job.dst + static_cast<size_t>(row0) * (job.row_bytes >> 2), 0,
                                                         static_cast<int>(rows * job.row_bytes), kRsrcWord3);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {  // four adjacent columns; rows past d_out are out of range
        v4i u;
#pragma unroll
        for (int r = 0; r < 4; ++r) u[r] = static_cast<int>(reduce(acc[t][4 * r4 + r], q));
        __builtin_amdgcn_raw_buffer_store_b128(
            u, out, (t * 32 + (lane & 31)) * job.row_bytes + (8 * r4 + 4 * (lane >> 5)) * 4, 0, 0);
      }
  }
}

// A launch: waves of a workgroup, steps held in LDS, workgroups a column tile.
struct Launch {
  uint32_t waves, chunk, splits;
};

Launch plan_of(const Tables& t, const Shape& s, uint32_t limbs) {
  Launch p;
  const uint32_t per = s.sub_len / kStep, groups = s.tiles / 2, tiles_n = 2 * t.n / kCols;
  p.waves = 8;
  const uint32_t most = kFold / kStep / per * per;
  p.chunk = s.steps < most ? s.steps : most;
  const uint32_t blocks = (groups + p.waves - 1) / p.waves;  // row blocks of a column tile
  if (p.chunk < s.steps) {
    p.splits = blocks;
  } else {
    const size_t have = static_cast<size_t>(tiles_n) * limbs;
    const size_t want = (t.num_cus + have - 1) / have;
    p.splits = static_cast<uint32_t>(want < blocks ? want : blocks);
  }
  return p;
}

template <int kSteps, bool kZeros>
hipError_t launch(const Tables& t, const Shape& sh, const void* w_q4, const uint32_t* ct_in, uint32_t* ct_out,
                  uint32_t d_out, uint32_t d_in, uint32_t limbs, hipStream_t s) {
  const Launch p = plan_of(t, sh, limbs);
  const uint8_t* base = static_cast<const uint8_t*>(w_q4);
  const uint32_t tiles_n = 2 * t.n / kCols;
  const size_t lds = static_cast<size_t>(p.chunk) * kStepFrags * 16 + (kZeros ? p.chunk / kSteps * 2 * kCols * 4 : 0);
  const auto k = mac_q4_kernel<kSteps, kZeros>;
  k<<<tiles_n * limbs * p.splits, p.waves * 64, lds, s>>>(t, reinterpret_cast<const uint2*>(base),
                                                         reinterpret_cast<const int32_t*>(base + sh.frag_bytes), ct_in,
                                                         ct_out, d_out, d_in, limbs, sh.steps, sh.subs, sh.tiles, tiles_n,
                                                         p.splits, p.chunk);
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
  const size_t lanes = sh.frag_bytes / 8, total = static_cast<size_t>(limbs) * sh.tiles * sh.subs * 32;
  q4_frag_kernel<<<static_cast<uint32_t>((lanes + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      w4, d_out, d_in, sh.steps, lanes, zeros ? 0u : 8u, reinterpret_cast<uint2*>(base));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  q4_scale_kernel<<<static_cast<uint32_t>((total + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      t, scales, zeros, d_out, group, sh.groups, sh.sub_len, sh.subs, sh.tiles, total, scale,
      reinterpret_cast<int32_t*>(base + sh.frag_bytes));
  return hipGetLastError();
}

hipError_t launch_mac_q4(const Tables& t, const void* w_q4, const uint32_t* ct_in, uint32_t* ct_out, uint32_t d_out,
                         uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros, hipStream_t s) {
  const Shape sh = shape_of(d_out, d_in, group, limbs, zeros);
  switch (sh.sub_len) {
    case 32: return (zeros ? launch<1, true> : launch<1, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
    case 64: return (zeros ? launch<2, true> : launch<2, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
    default: return (zeros ? launch<4, true> : launch<4, false>)(t, sh, w_q4, ct_in, ct_out, d_out, d_in, limbs, s);
  }
}

}  // namespace ckks
