// ct x pt MAC over 4-bit weights with one scale (and zero point) per group of
// inputs (gfx950).
//
// Per limb l, with u the 4-bit weights, z the zero points (8 without them) and
// S = rint(scale Delta) of the group,
//     out[j][col] = sum_g S[j][g] T[j][g][col] mod q_l,
//     T[j][g][col] = sum over the group of (u[j][i] - z[j][g]) x[i][col].
// T needs only the small integers u, which are the same for every limb; the
// scale enters once a group.
#include "ckks_internal.hpp"

namespace ckks {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kBK = 64;      // inputs of one step of the weight fragments
constexpr uint32_t kTileRows = 64;  // output rows are padded to this

// Encoded weights:
//   fragments [mt][ks][64 lanes] of 8 bytes: the 4-bit v = u - 8 (two's
//     complement) of row mt*16 + lane%16 and the 16 inputs k(lane, i) of 64-input
//     step ks, i < 16: k = 8 (lane/16) + i for i < 8 (the step's first 32
//     inputs), 32 + 8 (lane/16) + i - 8 for the others.  Word d holds i = 8d ..
//     8d + 7: the low halves of its bytes the first four, the high halves the
//     last four, so two masks give four bytes 16 v each.
//   scales [limb][mt][sub][16 rows] of {sa, sb} (or {sa, sb, zc, 0} with zero
//     points): sub-groups of `sub_len` inputs; sa = S / 16, sb = 2^16 S / 16 mod
//     q_l, centred; zc = 16 (z - 8).
struct Shape {
  uint32_t mt_total, ks_total, groups, sub_len, subs;
  size_t frag_bytes, scale_bytes;
};

// A sub-group is what one set of i32 sums covers: 256, 128 or 64 inputs that
// divide the group, else 32; a group that holds every input is cut freely.
Shape shape_of(uint32_t d_out, uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros) {
  Shape s;
  s.mt_total = (d_out + kTileRows - 1) / kTileRows * (kTileRows / 16);
  s.ks_total = (d_in + kBK - 1) / kBK;
  s.groups = (d_in + group - 1) / group;
  s.sub_len = s.groups == 1 || group % 256 == 0 ? 256 : group % 128 == 0 ? 128 : group % 64 == 0 ? 64 : 32;
  s.subs = (d_in + s.sub_len - 1) / s.sub_len;
  s.frag_bytes = static_cast<size_t>(s.mt_total) * s.ks_total * 64 * 8;
  s.scale_bytes = static_cast<size_t>(limbs) * s.mt_total * s.subs * 16 * (zeros ? 16 : 8);
  return s;
}

__global__ __launch_bounds__(kThreads) void q4_frag_kernel(const uint8_t* __restrict__ w4, uint32_t d_out,
                                                           uint32_t d_in, uint32_t ks_total, size_t lanes,
                                                           uint2* __restrict__ frag) {
  const size_t idx = static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (idx >= lanes) return;
  const uint32_t lane = idx & 63;
  const uint32_t ks = static_cast<uint32_t>((idx >> 6) % ks_total), mt = static_cast<uint32_t>((idx >> 6) / ks_total);
  const uint32_t row = mt * 16 + (lane & 15);
  const uint8_t* w = w4 + static_cast<size_t>(row) * ((d_in + 1) / 2);
  uint32_t word[2];
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const uint32_t k0 = ks * kBK + 32 * d + 8 * (lane >> 4);
    uint32_t v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = k0 + e;
      const uint32_t u = row < d_out && k < d_in ? (w[k >> 1] >> (4 * (k & 1))) & 15u : 8u;
      v |= (u ^ 8u) << (8 * (e & 3) + 4 * (e >> 2));  // u ^ 8 is u - 8 in four bits
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
                                                            uint32_t subs, uint32_t mt_total, size_t total,
                                                            double scale, int32_t* __restrict__ out) {
  const size_t idx = static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x;  // [limb][mt][sub][16]
  if (idx >= total) return;
  const uint32_t sub = static_cast<uint32_t>((idx >> 4) % subs);
  const size_t lm = (idx >> 4) / subs;
  const uint32_t l = static_cast<uint32_t>(lm / mt_total);
  const uint32_t row = static_cast<uint32_t>(lm % mt_total) * 16 + (idx & 15);
  const uint32_t q = tb.q[l];
  int32_t sa = 0, sb = 0, zc = 0;
  if (row < d_out) {
    const size_t at = static_cast<size_t>(row) * groups + static_cast<uint32_t>(static_cast<size_t>(sub) * sub_len / group);
    uint32_t r = reduce_f64_int(rint(static_cast<double>(scales[at]) * scale), q, tb.q_recip[l]);
#pragma unroll
    for (int i = 0; i < 4; ++i) r = (r & 1) ? (r + q) >> 1 : r >> 1;  // r / 16 mod q
    sa = centred(r, q);
    sb = centred(static_cast<uint32_t>((static_cast<uint64_t>(r) << 16) % q), q);
    if (zeros) zc = 16 * (static_cast<int32_t>(zeros[at] & 15u) - 8);
  }
  if (zeros)
    reinterpret_cast<int4*>(out)[idx] = make_int4(sa, sb, zc, 0);
  else
    reinterpret_cast<int2*>(out)[idx] = make_int2(sa, sb);
}

// One thread: one column of one limb and 16 output rows.
template <bool kZeros>
__global__ __launch_bounds__(kThreads) void mac_q4_kernel(Tables tb, const uint2* __restrict__ frag,
                                                          const int32_t* __restrict__ scales,
                                                          const uint32_t* __restrict__ ct_in,
                                                          uint32_t* __restrict__ ct_out, uint32_t d_out, uint32_t d_in,
                                                          uint32_t limbs, uint32_t mt_total, uint32_t ks_total,
                                                          uint32_t sub_len, uint32_t subs) {
  const uint32_t n = tb.n, col = blockIdx.x * kThreads + threadIdx.x;  // < 2N
  const uint32_t c = col >> tb.log_n, k = col & (n - 1), mt = blockIdx.y, l = blockIdx.z;
  const uint32_t q = tb.q[l];
  const double qr = tb.q_recip[l];
  const size_t stride = 2ull * limbs * n;
  const uint32_t* x = ct_in + (static_cast<size_t>(c) * limbs + l) * n + k;
  uint32_t acc[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0;
  for (uint32_t g = 0; g < subs; ++g) {
    int64_t t[16], xs = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0;
    const uint32_t stop = min(d_in, (g + 1) * sub_len);
    for (uint32_t i = g * sub_len; i < stop; ++i) {
      const int64_t xi = x[i * stride];
      const uint32_t ks = i / kBK, in = i % kBK, quarter = (in % 32) / 8, e = in % 8;
      const uint2* f = frag + (static_cast<size_t>(mt) * ks_total + ks) * 64 + quarter * 16;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t word = in < 32 ? f[r].x : f[r].y;
        const int32_t v = static_cast<int32_t>(word << (28 - (8 * (e & 3) + 4 * (e >> 2)))) >> 28;
        t[r] += 16 * v * xi;
      }
      xs += xi;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const size_t at = (((static_cast<size_t>(l) * mt_total + mt) * subs + g) << 4) + r;
      int64_t v = t[r];
      if constexpr (kZeros) v -= scales[4 * at + 2] * xs;
      int64_t m = v % static_cast<int64_t>(q);
      m = (m * scales[kZeros ? 4 * at : 2 * at]) % static_cast<int64_t>(q);
      acc[r] = add_mod(acc[r], static_cast<uint32_t>(m < 0 ? m + q : m), q);
    }
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const uint32_t j = mt * 16 + r;
    if (j < d_out) ct_out[((static_cast<size_t>(j) * 2 + c) * limbs + l) * n + k] = acc[r];
  }
  (void)qr;
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
  const size_t lanes = sh.frag_bytes / 8, total = static_cast<size_t>(limbs) * sh.mt_total * sh.subs * 16;
  q4_frag_kernel<<<static_cast<uint32_t>((lanes + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      w4, d_out, d_in, sh.ks_total, lanes, reinterpret_cast<uint2*>(base));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  q4_scale_kernel<<<static_cast<uint32_t>((total + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      t, scales, zeros, d_out, group, sh.groups, sh.sub_len, sh.subs, sh.mt_total, total, scale,
      reinterpret_cast<int32_t*>(base + sh.frag_bytes));
  return hipGetLastError();
}

hipError_t launch_mac_q4(const Tables& t, const void* w_q4, const uint32_t* ct_in, uint32_t* ct_out, uint32_t d_out,
                         uint32_t d_in, uint32_t group, uint32_t limbs, bool zeros, hipStream_t s) {
  const Shape sh = shape_of(d_out, d_in, group, limbs, zeros);
  const uint8_t* base = static_cast<const uint8_t*>(w_q4);
  const uint2* frag = reinterpret_cast<const uint2*>(base);
  const int32_t* scales = reinterpret_cast<const int32_t*>(base + sh.frag_bytes);
  const dim3 grid(2 * t.n / kThreads, (d_out + 15) / 16, limbs);
  const auto k = zeros ? mac_q4_kernel<true> : mac_q4_kernel<false>;
  k<<<grid, kThreads, 0, s>>>(t, frag, scales, ct_in, ct_out, d_out, d_in, limbs, sh.mt_total, sh.ks_total, sh.sub_len,
                              sh.subs);
  return hipGetLastError();
}

}  // namespace ckks
