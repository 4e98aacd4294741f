// Gated sums of requests' outputs: out[t][j] = sum over a bundle's terms r of gates[r] (.) y[r][j] mod q_l,
// slot by slot in NTT form, the gate plaintexts the same for all features and both components.
//
// Bound by memory: a term's output is read once and a sum written once, and the gates, which all features
// share, stay in registers.  A workgroup has one bundle, limb and 1024 coefficients, and goes through a
// share of the features; a lane has four adjacent coefficients.
#include "ckks_internal.hpp"

namespace ckks {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kCols = kThreads * 4;  // coefficients of a workgroup: 2^10, the smallest ring
constexpr uint32_t kMostTerms = 8;        // gates that stay in registers
constexpr uint32_t kFold = 15;            // products below 2^60 that a 64-bit sum holds, with a residue

struct Sum {
  const uint32_t* gates;   // request 0's word of coefficient 0 of the lane
  const uint32_t* src;     // feature 0's of request 0
  uint32_t* dst;           // feature 0's of the bundle
  size_t gate_words, ct_words, request_words;  // from request to request, feature to feature, request to request
  uint32_t q, first, last, half;               // features; words from component to component
  double qr;
};

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint4 load4(const uint32_t* p) { return *reinterpret_cast<const uint4*>(p); }

// What is read or written once passes the caches by: 12 requests of 256 features at 2^13 and 3 limbs, two terms a
// bundle, 182 -> 174 us (5.2 TB/s); stores alone 179, loads alone 186.
__device__ __forceinline__ uint4 load4_once(const uint32_t* p) {
  const v4u v = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void store4_once(uint32_t* p, const uint64_t (&t)[4], uint32_t q, double qr) {
  const v4u v{reduce_u64(t[0], q, qr), reduce_u64(t[1], q, qr), reduce_u64(t[2], q, qr), reduce_u64(t[3], q, qr)};
  __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(p));
}

// kTerms requests, their gates in registers.
template <uint32_t kTerms>
__device__ __forceinline__ void sum_of(const Sum& s, const uint32_t (&req)[kMostTerms]) {
  uint4 g[kTerms ? kTerms : 1];
#pragma unroll
  for (uint32_t i = 0; i < kTerms; ++i) g[i] = load4(s.gates + req[i] * s.gate_words);
  for (uint32_t j = s.first; j < s.last; ++j) {
#pragma unroll
    for (uint32_t c = 0; c < 2; ++c) {
      const size_t at = j * s.ct_words + c * s.half;
      uint64_t t[4] = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t i = 0; i < kTerms; ++i) {
        const uint4 y = load4_once(s.src + req[i] * s.request_words + at);
        t[0] += static_cast<uint64_t>(g[i].x) * y.x;
        t[1] += static_cast<uint64_t>(g[i].y) * y.y;
        t[2] += static_cast<uint64_t>(g[i].z) * y.z;
        t[3] += static_cast<uint64_t>(g[i].w) * y.w;
      }
      store4_once(s.dst + at, t, s.q, s.qr);
    }
  }
}

__global__ __launch_bounds__(kThreads) void combine_kernel(Tables tb, const uint32_t* __restrict__ gates,
                                                           const uint32_t* __restrict__ ct_in, uint32_t count,
                                                           const int32_t* __restrict__ terms, uint32_t top,
                                                           uint32_t* __restrict__ ct_out, uint32_t features, uint32_t limbs,
                                                           uint32_t shares) {
  const uint32_t n = tb.n, chunks = n / kCols;
  uint32_t id = blockIdx.x;
  const uint32_t share = id % shares;
  id /= shares;
  const uint32_t chunk = id % chunks;
  id /= chunks;
  const uint32_t l = id % limbs, t = id / limbs;
  const uint32_t k = chunk * kCols + threadIdx.x * 4, each = (features + shares - 1) / shares;
  Sum s;
  s.gate_words = static_cast<size_t>(limbs) * n;
  s.ct_words = 2 * s.gate_words;
  s.request_words = s.ct_words * features;
  s.gates = gates + static_cast<size_t>(l) * n + k;
  s.src = ct_in + static_cast<size_t>(l) * n + k;
  s.dst = ct_out + t * s.request_words + static_cast<size_t>(l) * n + k;
  s.half = limbs * n;
  s.q = tb.q[l];
  s.qr = tb.q_recip[l];
  s.first = share * each;
  s.last = min(features, s.first + each);
  // the requests that the terms name, the first of them by value
  const int32_t* list = terms + static_cast<size_t>(t) * top;
  uint32_t req[kMostTerms] = {}, found = 0;
  for (uint32_t i = 0; i < top; ++i) {
    const uint32_t r = static_cast<uint32_t>(list[i]);
    if (r >= count) continue;
#pragma unroll
    for (uint32_t f = 0; f < kMostTerms; ++f)
      if (found == f) req[f] = r;
    ++found;
  }
  switch (found) {
    case 0: return sum_of<0>(s, req);
    case 1: return sum_of<1>(s, req);
    case 2: return sum_of<2>(s, req);
    case 3: return sum_of<3>(s, req);
    case 4: return sum_of<4>(s, req);
    case 5: return sum_of<5>(s, req);
    case 6: return sum_of<6>(s, req);
    case 7: return sum_of<7>(s, req);
    case 8: return sum_of<8>(s, req);
  }
  // more: the list again for every feature, the gates from the caches (6 bundles of 64 features at 2^13 and 3 limbs: 8 terms
  // 143 us, 4.8 TB/s, 9 terms 178, 4.3, 16 terms 316, 4.1)
  for (uint32_t j = s.first; j < s.last; ++j)
    for (uint32_t c = 0; c < 2; ++c) {
      const size_t at = j * s.ct_words + c * s.half;
      uint64_t sum[4] = {0, 0, 0, 0};
      uint32_t held = 0;
      for (uint32_t i = 0; i < top; ++i) {
        const uint32_t r = static_cast<uint32_t>(list[i]);
        if (r >= count) continue;
        if (held == kFold) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] = reduce_u64(sum[e], s.q, s.qr);
          held = 0;
        }
        ++held;
        const uint4 g = load4(s.gates + r * s.gate_words), y = load4_once(s.src + r * s.request_words + at);
        sum[0] += static_cast<uint64_t>(g.x) * y.x;
        sum[1] += static_cast<uint64_t>(g.y) * y.y;
        sum[2] += static_cast<uint64_t>(g.z) * y.z;
        sum[3] += static_cast<uint64_t>(g.w) * y.w;
      }
      store4_once(s.dst + at, sum, s.q, s.qr);
    }
}

}  // namespace

hipError_t launch_combine(const Tables& t, const uint32_t* gates, const uint32_t* ct_in, uint32_t count,
                          const int32_t* terms, uint32_t bundles, uint32_t top, uint32_t* ct_out, uint32_t features,
                          uint32_t limbs, hipStream_t s) {
  const uint32_t each = limbs * (t.n / kCols);  // workgroups of a bundle and share, 2^10 at most
  const uint64_t groups = static_cast<uint64_t>(bundles) * each;
  // eight workgroups a CU where the features allow it
  const uint64_t want = (static_cast<uint64_t>(t.num_cus) * 8 + groups - 1) / groups;
  const uint32_t shares = static_cast<uint32_t>(want < features ? want : features);
  const uint32_t most = kMostGroups / (each * shares);  // bundles of a launch; shares are more than one of few groups only
  const size_t bundle_words = static_cast<size_t>(2) * limbs * t.n * features;
  for (uint32_t b = 0; b < bundles; b += most) {
    const uint32_t now = bundles - b < most ? bundles - b : most;
    combine_kernel<<<now * each * shares, kThreads, 0, s>>>(t, gates, ct_in, count, terms + static_cast<size_t>(b) * top, top,
                                                            ct_out + b * bundle_words, features, limbs, shares);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ckks
