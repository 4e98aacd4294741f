// Balanced base-256 digits of residues as int8 matrix-core operands, shared by
// the MACs that contract them.
#pragma once

#include "ckks_internal.hpp"

namespace ckks {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
constexpr uint32_t kBias = 0x80808080u;
constexpr int kRsrcWord3 = 0x00020000;  // buffer resource word 3: 32-bit raw data, range-checked

// o[b] byte e = p[e] byte b (4x4 byte transpose, eight v_perm_b32).
// __builtin_amdgcn_perm(hi, lo, sel): selector byte values 0-3 pick bytes of
// lo, 4-7 bytes of hi.
__device__ __forceinline__ void transpose4(uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3,
                                           uint32_t (&o)[4]) {
  const uint32_t x01l = __builtin_amdgcn_perm(p1, p0, 0x05010400u);  // p0.0 p1.0 p0.1 p1.1
  const uint32_t x01h = __builtin_amdgcn_perm(p1, p0, 0x07030602u);  // p0.2 p1.2 p0.3 p1.3
  const uint32_t x23l = __builtin_amdgcn_perm(p3, p2, 0x05010400u);
  const uint32_t x23h = __builtin_amdgcn_perm(p3, p2, 0x07030602u);
  o[0] = __builtin_amdgcn_perm(x23l, x01l, 0x05040100u);            // p0.0 p1.0 p2.0 p3.0
  o[1] = __builtin_amdgcn_perm(x23l, x01l, 0x07060302u);            // p0.1 p1.1 p2.1 p3.1
  o[2] = __builtin_amdgcn_perm(x23h, x01h, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(x23h, x01h, 0x07060302u);
}

// 16 residues (consecutive k) -> one 16-byte digit fragment per digit b:
// byte i of fragment b is digit b of residue i.  The bias is added before
// the byte transpose and removed after it (both are bytewise).
__device__ __forceinline__ void to_fragments(const uint32_t (&x)[16], v4i (&f)[4]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    uint32_t o[4];
    transpose4(x[4 * g] + kBias, x[4 * g + 1] + kBias, x[4 * g + 2] + kBias, x[4 * g + 3] + kBias, o);
#pragma unroll
    for (int b = 0; b < 4; ++b) f[b][g] = static_cast<int>(o[b] ^ kBias);
  }
}

}  // namespace ckks
