// Pieces of the attention kernels on the matrix cores (v_mfma_f32_32x32x16_bf16), shared by vit_attention_mfma.hip and rel_attention_mfma.h:
// the LDS layout of a matrix with a token a row, reads of it as operands, score tiles, stores.
// Planes of 32 features with 64-byte rows whose 16-byte chunks are XOR-swizzled by row bits 2-3; NK = features / 16, NM = planes.
#pragma once
#include "common.h"

namespace {
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
constexpr int ROW_B = 64;       // bytes of one token's 32 features of a plane

__device__ __forceinline__ int chunk_off(int row, int c16) { return row * ROW_B + ((c16 ^ ((row >> 2) & 3)) << 4); }

// 16-byte fragment read: token `row`, features d0 .. d0+7 (d0 a multiple of 8)
__device__ __forceinline__ bf16x8_t frag_read(const unsigned char* t, int plane_b, int row, int d0) {
  const unsigned char* p = t + (d0 >> 5) * plane_b + chunk_off(row, (d0 & 31) >> 3);
  return *reinterpret_cast<const bf16x8_t*>(p);
}
// Transposing fragment read for a product that reduces over tokens: the lane gets feature
// mt*32 + lane%32 of tokens rbase + h*4 + 0..3 and rbase + 8 + h*4 + 0..3 (h = lane / 32).
__device__ __forceinline__ bf16x8_t frag_read_tr(const unsigned char* t, int plane_b, int mt, int rbase, int lane) {
  const int g = lane >> 4, i16 = lane & 15;
  const int ch0 = (g & 1) * 16 + (i16 & 3) * 4;               // first of the 4 features this lane's address names
  const int row = rbase + (g >> 1) * 4 + (i16 >> 2);
  const unsigned char* base = t + mt * plane_b + (ch0 & 7) * 2;
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (s16x4_t __attribute__((address_space(3)))*)(base + chunk_off(row, ch0 >> 3)));
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (s16x4_t __attribute__((address_space(3)))*)(base + chunk_off(row + 8, ch0 >> 3)));
  const s16x8_t v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8_t, v);
}
__device__ __forceinline__ bf16x8_t pack_frag(const f32x16_t& a, int j) {
  uint4 v;
  v.x = pack_bf16x2(a[8 * j + 0], a[8 * j + 1]);
  v.y = pack_bf16x2(a[8 * j + 2], a[8 * j + 3]);
  v.z = pack_bf16x2(a[8 * j + 4], a[8 * j + 5]);
  v.w = pack_bf16x2(a[8 * j + 6], a[8 * j + 7]);
  return __builtin_bit_cast(bf16x8_t, v);
}
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// the fragments of the wavefront's own tokens, straight from memory (zeros past T)
template <int NK = 4>
__device__ __forceinline__ void own_frags(const bf16_t* src, size_t ld, int token, int T, int h, bf16x8_t* f) {
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (token < T) v = *reinterpret_cast<const uint4*>(src + (size_t)token * ld + ks * 16 + h * 8);
    f[ks] = __builtin_bit_cast(bf16x8_t, v);
  }
}
__device__ __forceinline__ float dot8(uint4 a, uint4 b) {
  float x[8], y[8], s = 0.f;
  unpack8(a, x);
  unpack8(b, y);
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  return s;
}
// What a workgroup of a launch over `heads` (image, head) pairs works on: which pair (false: none) and which of `parts` parts of it.  The parts of a
// pair run on one XCD (every 8th workgroup shares its L2), one behind the other.
__device__ __forceinline__ bool head_part(int heads, int parts, int* head, int* part) {
  const int l = blockIdx.x >> 3, g = l / parts;
  *part = l - g * parts;
  *head = g * 8 + (blockIdx.x & 7);
  return *head < heads;
}
// a 32 x 32 tile of X Y^T over the features: rows = tokens arow0.. of the LDS matrix `a`, columns =
// the wave's own tokens, whose fragments are in `b`
template <int NK = 4>
__device__ __forceinline__ f32x16_t tile_nt(const unsigned char* a, int plane_b, int arow0, const bf16x8_t* b, int lane) {
  f32x16_t acc = zero16();
#pragma unroll
  for (int ks = 0; ks < NK; ++ks)
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_read(a, plane_b, arow0 + (lane & 31), ks * 16 + (lane >> 5) * 8), b[ks], acc, 0, 0, 0);
  return acc;
}
// The accumulator of a [DH features] x [32 own tokens] product: a lane holds four consecutive features of every eight, its
// partner in the other half the other four.  They trade, so that a lane stores eight.
template <int DH = 64>
__device__ __forceinline__ void store_cols(bf16_t* dst_row, const f32x16_t* acc, int h, bool inside) {
#pragma unroll
  for (int mt = 0; mt < (DH + 31) / 32; ++mt)
#pragma unroll
    for (int i8 = 0; i8 < 2; ++i8) {
      if (mt * 32 + i8 * 16 >= DH) break;
      const f32x16_t& a = acc[mt];
      unsigned w[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const unsigned lo = pack_bf16x2(a[8 * i8 + 2 * k], a[8 * i8 + 2 * k + 1]), hi = pack_bf16x2(a[8 * i8 + 4 + 2 * k], a[8 * i8 + 5 + 2 * k]);
        const auto t = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);
        w[k] = t[0];
        w[2 + k] = t[1];
      }
      if (inside) *reinterpret_cast<uint4*>(dst_row + mt * 32 + i8 * 16 + h * 8) = uint4{w[0], w[1], w[2], w[3]};
    }
}

}  // namespace
