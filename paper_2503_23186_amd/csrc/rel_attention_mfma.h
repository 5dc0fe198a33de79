// Self-attention with a learned relative position bias, dropout of the probabilities and padded batches on the matrix cores (head sizes
// 16, 32, 64, 128, any number of tokens; bf16 storage on v_mfma_f32_32x32x16_bf16, fp32 on v_mfma_f32_32x32x2_f32): forward, gradients of q, k and v, gradient of the bias table.
//
// A wavefront owns 32 queries (keys) and walks over the keys (queries), which come into LDS 64 (fp32: 32) at a time by direct loads, two buffers: one
// barrier a stage, the loads of a stage under the products of the one before.  Rows past an image's tokens are out of the loads' range and
// arrive as zeros.  Score tiles as in vit_attention_mfma.hip: rows = keys, columns = queries in the forward pass and for dq, so that a
// query's statistics are a lane's own and the accumulator is the next product's operand; the other way round for dk and dv.
//
// The bias: the plan (rel.h) holds the bucket map in the order of the accumulator's registers, 32 bytes a lane and tile, as byte offsets into the head's
// column of the table, which lies in LDS; the entry behind its end is -infinity, which masked pairs and tokens past T name.
// Where 1 / sqrt(dh) is a power of two it goes into q (exact in bf16) and the bias into the accumulator that a score tile starts from; otherwise both
// meet in a multiply-add.  The reference is subtracted from the sum, so that tables with the lowest finite value keep their meaning; the
// exponential's base rides in the multiply-add behind it.
//
// dx = P (dP - delta) with delta = sum P dP.  do . o is delta up to what rounding took off o and off the probabilities in front of it (2^-7 of its terms),
// which is as exact as dq's own operands are but would show in the table's gradient, an fp32 sum.  The walk for dq takes it as an estimate; its
// dx' = P (dP - estimate) sum to what the estimate lacks, so that the walk behind it has delta to fp32.  With dropout both walks, and the sums for the table, have
// dx divided by the kept values' factor, so that dP and delta cancel in rows with a single pair without the rounding of a product.
//
// Dropout: a call of the generator gives eight draws, of four queries and two keys (include/cnnk_rel.h).  With a query a lane, four neighbouring
// lanes need the four words of the same calls: each makes a quarter of the calls and they transpose words among
// themselves; with a key a lane, two neighbours share a call, and each makes half of them.
#pragma once
#include "rel_attention.h"
#include "attn_tile.h"
#include "mfma_tile.h"

namespace {
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
// Online softmax (M. Milakov, N. Gimelshein, 2018) with a reference that is raised lazily (the conditional rescaling that T. Dao presented in 2025).
// Probabilities are summed as 2^((x - m) log2 e - down), where m is a reference that a row's largest score so far passes by at most `slack`, and 2^down is T times
// 2^(slack log2 e): sums over T keys stay below the largest value.  A reference that is raised lazily saves rescaling; fp32 storage, whose time the
// products take, has none of it, since the bits of `down` are missing in the exponent's fraction.
template <typename T> constexpr float kSlack = sizeof(T) == 2 ? 5.5f : 0.f;

// ---- storage types -----------------------------------------------------------------------------------------------------------
// Dim<T, DH>: the LDS layout of a stage's two matrices and the products with them.  EXACT: 1 / sqrt(DH) goes into one operand without a rounding that
// counts (a power of two, or fp32).
// A matrix in LDS has planes of 32 features.  bf16: attn_tile.h.  fp32: rows of 128 bytes in eight chunks of 16; in a pair of rows (256 bytes, all banks)
// chunk c of row r lies at ((r & 1) ^ (r >> 2 & 1)) * 8 + (c ^ (r >> 1 & 7)), so that sixteen rows read at one chunk, and rows r and r + 4 read whole, touch
// every bank once.
template <typename T, int DH> struct Dim;

template <int DH> struct Dim<bf16_t, DH> {
  static constexpr int NK = DH / 16, NM = (DH + 31) / 32, KB = 64;      // KB: rows of a stage
  static constexpr int PLANE = KB * ROW_B, MAT = NM * PLANE, STAGE = 2 * MAT, LOAD_ROWS = 16;
  static constexpr bool EXACT = DH == 16 || DH == 64;
  struct Own { bf16x8_t f[NK]; };      // 32 rows of a matrix as an operand, a row a lane
  // which row and byte of it a lane fetches in a load of 16 rows of a plane
  static __device__ __forceinline__ int load_row(int lane) { return lane >> 2; }
  static __device__ __forceinline__ int load_byte(int lane, int) { return ((lane & 3) ^ (lane >> 4 & 3)) * 16; }
  static __device__ __forceinline__ void own(const bf16_t* src, size_t ld, int row, int n, int h, Own& o) { own_frags<NK>(src, ld, row, n, h, o.f); }
  static __device__ __forceinline__ float dot(const Own& a, const Own& b) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) s += dot8(__builtin_bit_cast(uint4, a.f[k]), __builtin_bit_cast(uint4, b.f[k]));
    return s;
  }
  static __device__ __forceinline__ void scale(Own& o) {
    if (!EXACT) return;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      float v[8];
      unpack8(__builtin_bit_cast(uint4, o.f[k]), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= DH == 64 ? 0.125f : 0.25f;
      o.f[k] = __builtin_bit_cast(bf16x8_t, uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
    }
  }
  // acc + M Own^T: rows of M by own rows
  static __device__ __forceinline__ f32x16_t nt(const unsigned char* m, const Own& o, f32x16_t acc, int lane) {
#pragma unroll
    for (int k = 0; k < NK; ++k) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_read(m, PLANE, lane & 31, k * 16 + (lane >> 5) * 8), o.f[k], acc, 0, 0, 0);
    return acc;
  }
  // acc += M^T x: features by own rows
  static __device__ __forceinline__ void tn(const unsigned char* m, const f32x16_t& x, f32x16_t* acc, int lane) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x8_t xb = pack_frag(x, j);
#pragma unroll
      for (int mt = 0; mt < NM; ++mt) acc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_read_tr(m, PLANE, mt, 16 * j, lane), xb, acc[mt], 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void store(bf16_t* row, const f32x16_t* acc, int h, bool inside) { store_cols<DH>(row, acc, h, inside); }
};

template <int DH> struct Dim<float, DH> {
  static constexpr int NM = (DH + 31) / 32, NG = DH / 8, KB = 32;
  static constexpr int PLANE = KB * 128, MAT = NM * PLANE, STAGE = 2 * MAT, LOAD_ROWS = 8;
  static constexpr bool EXACT = true;
  struct Own { float4 f[NG]; };        // features 8 g + 4 h ..  + 3 of lane half h
  static __device__ __forceinline__ int load_row(int lane) { return (lane >> 4) * 2 + ((lane >> 3 & 1) ^ (lane >> 5)); }
  static __device__ __forceinline__ int load_byte(int lane, int group) { return ((lane & 7) ^ ((group & 1) * 4 + (lane >> 4))) * 16; }
  static __device__ __forceinline__ int at(int row, int chunk) {
    return (row >> 1) * 256 + (((row & 1) ^ (row >> 2 & 1)) << 7) + ((chunk ^ (row >> 1 & 7)) << 4);
  }
  static __device__ __forceinline__ void own(const float* src, size_t ld, int row, int n, int h, Own& o) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      o.f[g] = float4{0.f, 0.f, 0.f, 0.f};
      if (row < n) o.f[g] = *reinterpret_cast<const float4*>(src + (size_t)row * ld + g * 8 + h * 4);
    }
  }
  static __device__ __forceinline__ float dot(const Own& a, const Own& b) {
    float s = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) s += (a.f[g].x * b.f[g].x + a.f[g].y * b.f[g].y) + (a.f[g].z * b.f[g].z + a.f[g].w * b.f[g].w);
    return s;
  }
  static __device__ __forceinline__ void scale(Own& o) {
    constexpr float s = DH == 16 ? 0.25f : DH == 32 ? 0.17677669529663689f : DH == 64 ? 0.125f : 0.088388347648318447f;
#pragma unroll
    for (int g = 0; g < NG; ++g) o.f[g] = float4{o.f[g].x * s, o.f[g].y * s, o.f[g].z * s, o.f[g].w * s};
  }
  static __device__ __forceinline__ f32x16_t nt(const unsigned char* m, const Own& o, f32x16_t acc, int lane) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float4 v = *reinterpret_cast<const float4*>(m + (g >> 2) * PLANE + at(lane & 31, (g & 3) * 2 + (lane >> 5)));
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.x, o.f[g].x, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.y, o.f[g].y, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.z, o.f[g].z, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.w, o.f[g].w, acc, 0, 0, 0);
    }
    return acc;
  }
  // A step reduces over the two rows that register i of the halves stands for, and needs no conversion.
  static __device__ __forceinline__ void tn(const unsigned char* m, const f32x16_t& x, f32x16_t* acc, int lane) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = (i >> 2) * 8 + (lane >> 5) * 4 + (i & 3);
#pragma unroll
      for (int mt = 0; mt < NM; ++mt) {
        const float v = *reinterpret_cast<const float*>(m + mt * PLANE + at(row, (lane & 31) >> 2) + (lane & 3) * 4);
        acc[mt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x[i], acc[mt], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ void store(float* row, const f32x16_t* acc, int h, bool inside) {
#pragma unroll
    for (int mt = 0; mt < NM; ++mt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        if (mt * 32 + i4 * 8 >= DH) break;
        if (inside) *reinterpret_cast<float4*>(row + mt * 32 + i4 * 8 + h * 4) = float4{acc[mt][4 * i4], acc[mt][4 * i4 + 1], acc[mt][4 * i4 + 2], acc[mt][4 * i4 + 3]};
      }
  }
};

// acc += M^T x in the backward pass.  bf16: x is rounded to 2^-8, as is the result.  Two independent roundings of one size have sqrt(2) times the error of one; that is what operands
// in bf16 cost, and stays (1.43 measured over many pairs, from 33 tokens on).  Images of one tile were above it, up to 1.56: they add a product with what the rounding took off (1.05
// to 1.3; both walks together 21.8 -> 23.0 us at 64 images of 25 tokens and 12 heads of 64, where starting takes most of it).
template <typename T, int DH> __device__ __forceinline__ void tn_bwd(const unsigned char* m, const f32x16_t& x, f32x16_t* acc, int lane, bool one_tile) {
  Dim<T, DH>::tn(m, x, acc, lane);
  if (sizeof(T) == 2 && one_tile) {
    f32x16_t r;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const unsigned w = pack_bf16x2(x[i], x[i + 1]);
      r[i] = x[i] - __uint_as_float(w << 16);
      r[i + 1] = x[i + 1] - __uint_as_float(w & 0xffff0000u);
    }
    Dim<T, DH>::tn(m, r, acc, lane);
  }
}

// ---- stages: KB rows of two matrices -----------------------------------------------------------------------------------------
// A wavefront's direct load fills LOAD_ROWS rows of a plane, 1 KB.
template <typename T, int DH> struct Stager {
  using D = Dim<T, DH>;
  i32x4_t x, y;                      // the matrices' descriptors
  unsigned ld_x, ld_y;               // bytes of a row
  int lane;
  __device__ __forceinline__ void init(const T* px, const T* py, unsigned ldx, unsigned ldy, int n, int ln) {
    x = make_desc(px, n > 0 ? (unsigned)(n - 1) * ldx + DH * sizeof(T) : 0u);
    y = make_desc(py, n > 0 ? (unsigned)(n - 1) * ldy + DH * sizeof(T) : 0u);
    ld_x = ldx;
    ld_y = ldy;
    lane = ln;
  }
  __device__ __forceinline__ void load(int r0, unsigned lds, int wave, int waves) const {
    constexpr int GROUPS = D::KB / D::LOAD_ROWS, PER = D::NM * GROUPS;                  // loads of a matrix
    for (int q = wave; q < 2 * PER; q += waves) {
      const bool second = q >= PER;
      const int k = second ? q - PER : q, plane = k / GROUPS, group = k % GROUPS;
      const unsigned ld = second ? ld_y : ld_x;
      const unsigned at = (unsigned)(r0 + group * D::LOAD_ROWS + D::load_row(lane)) * ld + plane * 32 * sizeof(T) + D::load_byte(lane, group);
      load16_to_lds(second ? y : x, lds + q * 1024, at);
    }
  }
};

// ---- bias ------------------------------------------------------------------------------------------------------------------
struct MapRegs { uint4 v[2]; };
__device__ __forceinline__ void map_load(MapRegs& m, const unsigned short* map, int tile, int lane) {
  const uint4* p = reinterpret_cast<const uint4*>(map + (size_t)tile * 1024 + lane * 16);
  m.v[0] = p[0];
  m.v[1] = p[1];
}
__device__ __forceinline__ float bias_of(const unsigned char* table, const MapRegs& m, int i) {
  const uint4 q = m.v[i >> 3];
  const unsigned w = (i & 7) < 4 ? ((i & 7) < 2 ? q.x : q.y) : ((i & 7) < 6 ? q.z : q.w);
  return *reinterpret_cast<const float*>(table + (i & 1 ? w >> 16 : w & 0xffffu));
}
// the head's column of the table, straight into LDS (there with the first stage), -infinity behind it
__device__ __forceinline__ void table_load(unsigned lds, float* dst, const RelArgs& a, int head, int wave, int waves, int lane) {
  const i32x4_t desc = make_desc(a.table, (unsigned)a.buckets * a.heads * 4u);
  for (int k0 = wave * 64; k0 < a.buckets; k0 += waves * 64)
    if (k0 + lane < a.buckets) load4_to_lds(desc, lds + k0 * 4, (unsigned)((k0 + lane) * a.heads + head) * 4u);
  if (threadIdx.x == 0) dst[a.buckets] = -INFINITY;
}
// A tile of scores with their bias.  One operand has been through Dim::scale.
template <typename T, int DH, bool BIAS>
__device__ __forceinline__ f32x16_t score_tile(const unsigned char* m, const typename Dim<T, DH>::Own& o, const float* table, const MapRegs& map, float scale, int lane) {
  using D = Dim<T, DH>;
  const unsigned char* t = reinterpret_cast<const unsigned char*>(table);
  f32x16_t x = zero16();
  if (BIAS && D::EXACT) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = bias_of(t, map, i);
  }
  x = D::nt(m, o, x, lane);
  if (!D::EXACT) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = BIAS ? fmaf(x[i], scale, bias_of(t, map, i)) : x[i] * scale;
  }
  return x;
}

// ---- blocks that are not all masked ----------------------------------------------------------------------------------------------
// Which blocks of the other side a wavefront's block, and any of its workgroup's, has pairs with: in LDS, since few maps leave any out.
struct Live {
  const unsigned long long* w;       // bits of the wavefront's block
  const unsigned long long* all;     // of the workgroup's together
  bool some;                         // blocks are left out
};
template <bool BIAS>
__device__ __forceinline__ Live live_start(unsigned char* lds, const unsigned long long* p, int dead, int block0, int NT, int wave, int waves, int lane) {
  unsigned long long* m = reinterpret_cast<unsigned long long*>(lds);
  Live l = {m + wave * 4, m + 32, BIAS && dead != 0};
  if (l.some) {
    if (threadIdx.x < 32) {
      const unsigned long long v = block0 + (lane >> 2) < NT && lane >> 2 < waves ? p[(size_t)block0 * 4 + lane] : 0;      // word lane % 4 of block lane / 4
      m[lane] = v;
      unsigned lo = (unsigned)v, hi = (unsigned)(v >> 32);
#pragma unroll
      for (int d = 4; d < 32; d *= 2) {
        lo |= __shfl_xor(lo, d, 64);
        hi |= __shfl_xor(hi, d, 64);
      }
      if (lane < 4) m[32 + lane] = (unsigned long long)hi << 32 | lo;
    }
    workgroup_barrier();
  }
  return l;
}
// the first of blocks from .. end - 1 that is there, end if none is
__device__ __forceinline__ int live_next(const unsigned long long* w, bool some, int from, int end) {
  if (!some) return min(from, end);
  while (from < end) {
    const unsigned long long v = w[from >> 6];
    const unsigned long long m =
        ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v)) >> (from & 63);
    if (m) return min(end, from + (int)__builtin_ctzll(m));
    from = (from | 63) + 1;
  }
  return end;
}

// ---- dropout ---------------------------------------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ unsigned quad(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kSwap1 = 0xb1;      // the neighbour of two
// word j of this lane <-> word (lane % 4) of lane j of the four, with selects that read the other lane themselves (v_cndmask_b32_dpp; a move and a select
// each otherwise).  A value that a lane crossing reads is two instructions old.
__device__ __forceinline__ void transpose4(unsigned (&w)[4]) {
  const unsigned long long even = 0x5555555555555555ull, low = 0x3333333333333333ull;
  unsigned a0, a1, a2, a3, b0, b1, b2, b3;
  asm("s_mov_b64 vcc, %12\n\t"
      "s_nop 1\n\t"
      "v_cndmask_b32_dpp %0, %9, %8, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "v_cndmask_b32_dpp %2, %11, %10, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "s_not_b64 vcc, vcc\n\t"
      "v_cndmask_b32_dpp %1, %8, %9, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "v_cndmask_b32_dpp %3, %10, %11, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "s_mov_b64 vcc, %13\n\t"
      "v_cndmask_b32_dpp %4, %2, %0, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
      "v_cndmask_b32_dpp %5, %3, %1, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
      "s_not_b64 vcc, vcc\n\t"
      "v_cndmask_b32_dpp %6, %0, %2, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
      "v_cndmask_b32_dpp %7, %1, %3, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf"
      : "=&v"(a0), "=&v"(a1), "=&v"(a2), "=&v"(a3), "=&v"(b0), "=&v"(b1), "=&v"(b2), "=&v"(b3)
      : "v"(w[0]), "v"(w[1]), "v"(w[2]), "v"(w[3]), "s"(even), "s"(low)
      : "vcc", "scc");
  w[0] = b0, w[1] = b1, w[2] = b2, w[3] = b3;
}
// Draws of a tile, two to a word: register i's in half i % 2 of word i / 2.
__device__ __forceinline__ unsigned draw_of(const unsigned (&word)[8], int i) { return i & 1 ? word[i >> 1] >> 16 : word[i >> 1] & 0xffffu; }
// Lanes are queries: a word belongs to four queries, of which each lane has made a quarter of the calls.  t4: the lane's query / 4.
__device__ __forceinline__ void draws_by_query(unsigned (&word)[8], int key0, unsigned t4, unsigned bh, RelKey key, int lane) {
#pragma unroll
  for (int jp = 0; jp < 2; ++jp) {
    RelWords r = rel_words((unsigned)(key0 >> 1) + (lane & 3) * 4 + (lane >> 5) * 2 + jp, t4, bh, kDrawPairs, key);
    transpose4(r.w);
#pragma unroll
    for (int g = 0; g < 4; ++g) word[g * 2 + jp] = r.w[g];
  }
}
// Lanes are keys: two neighbours have the halves of the same words, and each has made half of the calls.  u2: the lane's key / 2.
__device__ __forceinline__ void draws_by_key(unsigned (&word)[8], int query0, unsigned u2, unsigned bh, RelKey key, int lane) {
  const bool odd = lane & 1;
  const unsigned own = odd ? 0x07060302u : 0x05040100u, others = odd ? 0x05040100u : 0x07060302u;      // that half of both words
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const RelWords r = rel_words(u2, (unsigned)(query0 >> 2) + (odd ? 4 : 0) + k * 2 + (lane >> 5), bh, kDrawPairs, key);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const unsigned mine = __builtin_amdgcn_perm(r.w[2 * j + 1], r.w[2 * j], own);
      const unsigned got = quad<kSwap1>(__builtin_amdgcn_perm(r.w[2 * j + 1], r.w[2 * j], others));
      word[k * 2 + j] = odd ? got : mine;
      word[4 + k * 2 + j] = odd ? mine : got;
    }
  }
}

// What a workgroup works on: which of `groups` (false: none) and which part of it.  The parts of one run on one XCD (every 8th workgroup shares its L2),
// one behind the other.  The last groups, where they are fewer than the XCDs, are dealt out by parts, so that each XCD has the same share: 36 heads of 1600 tokens 129 -> 91 us
// forward, 199 -> 135 for dk and dv.  Not where every workgroup has a CU of its own (32 to an XCD) either way: 12 heads of 1024 tokens take 39 us forward, dealt out 42, since
// two L2s read such a head.
__host__ __device__ __forceinline__ int whole_groups(int groups, int parts) { return (groups + 7) / 8 * parts > 32 ? groups >> 3 : (groups + 7) >> 3; }      // of an XCD
__host__ __device__ __forceinline__ int last_share(int groups, int whole, int parts) { return groups > whole * 8 ? ((groups - whole * 8) * parts + 7) >> 3 : 0; }
__device__ __forceinline__ bool group_part(int groups, FastDiv parts, int* group, int* part) {
  const int x = blockIdx.x & 7, y = (int)blockIdx.x >> 3, n = parts.d, whole = whole_groups(groups, n);
  int g;
  if (y < whole * n) {
    parts.divmod(y, &g, part);
    *group = g * 8 + x;
  } else {
    parts.divmod(x * last_share(groups, whole, n) + y - whole * n, &g, part);
    *group = whole * 8 + g;
  }
  return *group < groups;
}
__device__ __forceinline__ float both_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Keeps the compiler from turning a branch that one tile of a walk takes into selects in every tile (a tenth of the forward pass).
__device__ __forceinline__ void only_here() { asm volatile(""); }
// times f, or 0 in lanes whose rows are not `there`; most wavefronts have all of them
template <int N> __device__ __forceinline__ void scale_rows(f32x16_t* acc, float f, bool there) {
  if (__all(there)) {
    only_here();
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[k][i] *= f;
  } else {
    only_here();
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[k][i] = there ? acc[k][i] * f : 0.f;
  }
}
__device__ __forceinline__ int key_of(int i, int h) { return (i >> 2) * 8 + h * 4 + (i & 3); }

// ---- forward ---------------------------------------------------------------------------------------------------------------
// 128 registers leave four wavefronts to a SIMD (bf16, heads of up to 64); with heads of 64, bias and dropout one more is spilled (8 bytes of scratch).
template <typename T, int DH, bool BIAS, bool DROP>
__global__ void __launch_bounds__(512, sizeof(T) == 2 && DH <= 64 ? 4 : 2) rel_mfma_fwd_kernel(RelArgs a, const T* __restrict__ qkv, T* __restrict__ o,
                                                                             float* __restrict__ stats, FastDiv parts) {
  using D = Dim<T, DH>;
  constexpr int TS = D::KB / 32, TILE = D::PLANE / TS;      // tiles of a stage, bytes of a tile's rows in a plane
  extern __shared__ __align__(16) unsigned char smem[];
  int bh, part;
  if (!group_part(a.B * a.heads, parts, &bh, &part)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6, h = lane >> 5;
  const int b = a.by_heads.div(bh), head = bh - b * a.heads, d = a.heads * DH, n = rel_tokens(a, b);
  const size_t ld = 3 * (size_t)d;
  const int q0 = (part * waves + wave) * 32, q = q0 + (lane & 31), first = part * waves * 32;
  const T* base = qkv + (size_t)b * a.T * ld + head * DH;
  f32x16_t oacc[D::NM];
#pragma unroll
  for (int mt = 0; mt < D::NM; ++mt) oacc[mt] = zero16();
  float m = -INFINITY, l = 0.f;      // l: of this lane's half of the keys
  bool fits = true;
  if (first < n) {
    float* table = reinterpret_cast<float*>(smem + 2 * D::STAGE);
    Stager<T, DH> st;
    st.init(base + d, base + 2 * d, (unsigned)(ld * sizeof(T)), (unsigned)(ld * sizeof(T)), n, lane);
    st.load(0, 0, wave, waves);      // whether it is needed or not: which stages are is on its way
    const bool mine = q0 < n;
    const int tiles = (n + 31) >> 5, stages = (tiles + TS - 1) / TS;
    const unsigned short* map = BIAS ? a.by_query + (size_t)(q0 >> 5) * a.NT * 1024 : nullptr;
    MapRegs mr, next;
    RelAbout about = {0, 0};
    if (BIAS) {
      about = rel_about(a);
      if (mine) map_load(next, map, 0, lane);
      table_load(2 * D::STAGE, table, a, head, wave, waves, lane);
    }
    typename D::Own bq;
    D::own(base, ld, q, n, h, bq);
    D::scale(bq);
    RelKey key{0u, 0u};
    if (DROP) key = rel_key(a.rng, a.site);
    // stages that one of the workgroup's blocks needs, and of them the tiles that this wavefront's does
    const Live live = live_start<BIAS>(reinterpret_cast<unsigned char*>(table + a.buckets + 1 + (a.buckets + 1 & 1)), a.live_query, about.dead, first >> 5, a.NT, wave, waves, lane);
    auto tile_from = [&](int t) __attribute__((always_inline)) { return live_next(live.w, live.some, t, tiles); };
    auto stage_from = [&](int k) __attribute__((always_inline)) {
      const int t = live_next(live.all, live.some, k * TS, tiles);
      return t < tiles ? t / TS : stages;
    };
    if (BIAS) fits = rel_plan_fits(a, about);
    int tn = mine && fits ? tile_from(0) : tiles;
    if (BIAS && tn > 0 && tn < tiles) map_load(next, map, tn, lane);
    for (int stage = 0, buf = 0; stage < stages; buf ^= 1) {
      wait_vm<0>();
      workgroup_barrier();
      const int then = stage_from(stage + 1);
      if (then < stages) st.load(then * D::KB, (buf ^ 1) * D::STAGE, wave, waves);
      while (tn < min(tiles, (stage + 1) * TS)) {
        const int t = tn;
        tn = tile_from(t + 1);
        if (BIAS) {
          mr = next;
          if (tn < tiles) map_load(next, map, tn, lane);
        }
        const unsigned char *Ks = smem + buf * D::STAGE + (t - stage * TS) * TILE, *Vs = Ks + D::MAT;
        f32x16_t x = score_tile<T, DH, BIAS>(Ks, bq, table, mr, a.scale, lane);
        if (t * 32 + 32 > n) {
          only_here();
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (t * 32 + key_of(i, h) >= n) x[i] = -INFINITY;
        }
        float tm = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) tm = fmaxf(tm, x[i]);
        tm = both_halves_max(tm);
        if (__any(tm > m + kSlack<T>)) {
          const float mn = fmaxf(m, tm);
          const float f = m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * kLog2e);      // also where both are -infinity
          l *= f;
#pragma unroll
          for (int mt = 0; mt < D::NM; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[mt][i] *= f;
          m = mn;
        }
        const float ref = m > -INFINITY ? m : 0.f;
        float add[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[i] = __builtin_amdgcn_exp2f(fmaf(x[i] - ref, kLog2e, -a.down));
          add[i & 1] += x[i];
        }
        l += add[0] + add[1];
        if (DROP) {
          unsigned word[8];
          draws_by_query(word, t * 32, (unsigned)q >> 2, (unsigned)bh, key, lane);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = draw_of(word, i) < a.dr.q ? 0.f : x[i];
        }
        D::tn(Vs, x, oacc, lane);
      }
      stage = then;
    }
  }
  if (q0 >= a.T) return;
  l = fits ? both_halves_sum(l) : NAN;
  const bool any = q < n && !(l == 0.f);      // 0: every key masked, since the largest score adds 2^-down at least; NaN (in q, k or the table, or an overflow) is handed on
  scale_rows<D::NM>(oacc, a.dr.scale / l, any);
  D::store(o + ((size_t)b * a.T + q) * d + head * DH, oacc, h, q < a.T);
  if (stats && h == 0 && q < a.T)
    *reinterpret_cast<float2*>(stats + ((size_t)bh * a.T + q) * 2) = any ? float2{m > -INFINITY ? m : 0.f, kLn2 * __builtin_amdgcn_logf(l * a.up)} : float2{-INFINITY, 0.f};
}

// ---- backward: dq, and for the kernel behind it the rows' statistics and delta -----------------------------------------------
// rows [B * heads][3][Tp], Tp = T rounded up to 64: reference, log2 of the sum relative to it (+infinity for rows without a part: their probabilities
// come out as 0), delta.
template <typename T, int DH, bool BIAS, bool DROP>
__global__ void __launch_bounds__(DH <= 64 ? 512 : 256, sizeof(T) == 2 && DH <= 64 ? 3 : DH <= 64 ? 2 : 1) rel_mfma_dq_kernel(RelArgs a, const T* __restrict__ qkv, const T* __restrict__ o,
                                                                            const T* __restrict__ d_o, const float* __restrict__ stats,
                                                                            T* __restrict__ dqkv, float* __restrict__ rows, FastDiv parts) {
  using D = Dim<T, DH>;
  constexpr int TS = D::KB / 32, TILE = D::PLANE / TS;      // tiles of a stage, bytes of a tile's rows in a plane
  extern __shared__ __align__(16) unsigned char smem[];
  int bh, part;
  if (!group_part(a.B * a.heads, parts, &bh, &part)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6, h = lane >> 5;
  const int b = a.by_heads.div(bh), head = bh - b * a.heads, d = a.heads * DH, n = rel_tokens(a, b);
  const size_t ld = 3 * (size_t)d;
  const int q0 = (part * waves + wave) * 32, q = q0 + (lane & 31), first = part * waves * 32;
  const T* base = qkv + (size_t)b * a.T * ld + head * DH;
  const size_t head0 = (size_t)b * a.T * d + head * DH;
  constexpr bool FIX = sizeof(T) == 2;      // fp32: do . o is delta
  f32x16_t dq[D::NM];
#pragma unroll
  for (int mt = 0; mt < D::NM; ++mt) dq[mt] = zero16();
  float m = 0.f, L2 = INFINITY, delta = 0.f, lack = 0.f;
  bool fits = true;
  if (first < n) {
    float* table = reinterpret_cast<float*>(smem + 2 * D::STAGE);
    Stager<T, DH> st;
    st.init(base + d, base + 2 * d, (unsigned)(ld * sizeof(T)), (unsigned)(ld * sizeof(T)), n, lane);
    st.load(0, 0, wave, waves);      // whether it is needed or not: which stages are is on its way
    const bool mine = q0 < n;
    const int tiles = (n + 31) >> 5, stages = (tiles + TS - 1) / TS;
    const unsigned short* map = BIAS ? a.by_query + (size_t)(q0 >> 5) * a.NT * 1024 : nullptr;
    MapRegs mr, next;
    RelAbout about = {0, 0};
    if (BIAS) {
      about = rel_about(a);
      if (mine) map_load(next, map, 0, lane);
      table_load(2 * D::STAGE, table, a, head, wave, waves, lane);
    }
    typename D::Own bq, bg;
    D::own(base, ld, q, n, h, bq);
    D::scale(bq);
    D::own(d_o + head0, d, q, n, h, bg);
    {
      typename D::Own t;
      D::own(o + head0, d, q, n, h, t);
      delta = both_halves_sum(D::dot(t, bg)) * a.dr.keep;
    }
    if (q < n) {
      const float2 s = *reinterpret_cast<const float2*>(stats + ((size_t)bh * a.T + q) * 2);
      if (s.x > -INFINITY) {
        m = s.x;
        L2 = s.y * kLog2e;
      }
    }
    RelKey key{0u, 0u};
    if (DROP) key = rel_key(a.rng, a.site);
    // stages that one of the workgroup's blocks needs, and of them the tiles that this wavefront's does
    const Live live = live_start<BIAS>(reinterpret_cast<unsigned char*>(table + a.buckets + 1 + (a.buckets + 1 & 1)), a.live_query, about.dead, first >> 5, a.NT, wave, waves, lane);
    auto tile_from = [&](int t) __attribute__((always_inline)) { return live_next(live.w, live.some, t, tiles); };
    auto stage_from = [&](int k) __attribute__((always_inline)) {
      const int t = live_next(live.all, live.some, k * TS, tiles);
      return t < tiles ? t / TS : stages;
    };
    if (BIAS) fits = rel_plan_fits(a, about);
    int tn = mine && fits ? tile_from(0) : tiles;
    if (BIAS && tn > 0 && tn < tiles) map_load(next, map, tn, lane);
    for (int stage = 0, buf = 0; stage < stages; buf ^= 1) {
      wait_vm<0>();
      workgroup_barrier();
      const int then = stage_from(stage + 1);
      if (then < stages) st.load(then * D::KB, (buf ^ 1) * D::STAGE, wave, waves);
      while (tn < min(tiles, (stage + 1) * TS)) {
        const int t = tn;
        tn = tile_from(t + 1);
        if (BIAS) {
          mr = next;
          if (tn < tiles) map_load(next, map, tn, lane);
        }
        const unsigned char *Ks = smem + buf * D::STAGE + (t - stage * TS) * TILE, *Vs = Ks + D::MAT;
        f32x16_t p = score_tile<T, DH, BIAS>(Ks, bq, table, mr, a.scale, lane);
        f32x16_t dx = D::nt(Vs, bg, zero16(), lane);
        unsigned word[8];
        if (DROP) draws_by_query(word, t * 32, (unsigned)q >> 2, (unsigned)bh, key, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(p[i] - m, kLog2e, -L2));
          if (DROP) dx[i] = draw_of(word, i) < a.dr.q ? 0.f : dx[i];
          dx[i] = p[i] * (dx[i] - delta);
        }
        if (t * 32 + 32 > n) {       // keys past the image's tokens: rows of zeros, whose probabilities may be infinite
          only_here();
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (t * 32 + key_of(i, h) >= n) dx[i] = 0.f;
        }
        if (FIX) {
          float add[2] = {0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 16; ++i) add[i & 1] += dx[i];
          lack += add[0] + add[1];
        }
        tn_bwd<T, DH>(Ks, dx, dq, lane, a.NT == 1);
      }
      stage = then;
    }
  }
  if (q0 >= a.T) return;
  lack = both_halves_sum(lack);
  scale_rows<D::NM>(dq, fits ? a.scale * a.dr.scale : NAN, q < n);
  D::store(dqkv + (size_t)b * a.T * ld + head * DH + (size_t)q * ld, dq, h, q < a.T);
  if (h == 0) {
    float* r = rows + (size_t)bh * 3 * a.Tp + q;
    r[0] = m;
    r[a.Tp] = L2;
    r[2 * a.Tp] = delta + lack;
  }
}

// ---- backward: dk and dv, and dx of every pair summed over images ----------------------------------------------------------------
// A workgroup has the keys of its part for `units` (head, image) pairs, one after the other, images before heads.  Where the table learns, each wavefront adds
// dx of its keys to pairs [slot][heads][NT keys][NT queries][4][64][4], the slot being the workgroup's number among those that have images of the head: a
// tile's sums so far come in while its scores are formed; they are a wavefront's own, in the caches, so the sum over images has one order and needs
// no atomics.
// Registers are short: with bias and dropout 90 to 100 scalar ones lie in lanes of vector registers (about 15 reads a tile, 116 an image), and fp32 with heads of 64 has two
// vector registers in scratch (12 bytes).  Heads of 128 take 400 and more, one wavefront to a SIMD.
template <typename T, int DH, bool BIAS, bool DROP, bool RUNS>
__global__ void __launch_bounds__(DH <= 64 ? 512 : 256, DH <= 64 ? 2 : 1) rel_mfma_dkv_kernel(RelArgs a, const T* __restrict__ qkv, const T* __restrict__ d_o,
                                                                             const float* __restrict__ rows, T* __restrict__ dqkv, float* pairs, FastDiv parts,
                                                                             int units, int groups, unsigned own_lds) {
  using D = Dim<T, DH>;
  constexpr int TS = D::KB / 32, TILE = D::PLANE / TS;      // tiles of a stage, bytes of a tile's rows in a plane
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int STAGE = D::STAGE + 3 * D::KB * 4;
  int group, part;
  const int all = a.B * a.heads;
  if (!group_part(groups, parts, &group, &part)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6, h = lane >> 5, d = a.heads * DH;
  const size_t ld = 3 * (size_t)d;
  const int u0 = (part * waves + wave) * 32, u = u0 + (lane & 31), first = part * waves * 32;
  float* table = reinterpret_cast<float*>(smem + 2 * STAGE);
  float* block_lds = reinterpret_cast<float*>(smem + own_lds) + wave * 1024;      // RUNS: where a block becomes runs
  RelKey key{0u, 0u};
  if (DROP) key = rel_key(a.rng, a.site);
  const unsigned short* map = BIAS ? a.by_key + (size_t)(u0 >> 5) * a.NT * 1024 : nullptr;
  RelAbout about = {0, 0};
  if (BIAS) about = rel_about(a);
  const int end = min(all, (group + 1) * units);
  if (BIAS && !rel_plan_fits(a, about)) {
    f32x16_t none[D::NM];
#pragma unroll
    for (int mt = 0; mt < D::NM; ++mt) none[mt] = zero16();
    for (int unit = group * units; unit < end; ++unit) {
      const int head = a.by_images.div(unit), b = unit - head * a.B;
      T* out = dqkv + (size_t)b * a.T * ld + head * DH + d + (size_t)u * ld;
      if (u0 >= a.T) return;
      scale_rows<D::NM>(none, NAN, u < rel_tokens(a, b));
      D::store(out, none, h, u < a.T);
      D::store(out + d, none, h, u < a.T);
    }
    return;
  }
  const Live live = live_start<BIAS>(reinterpret_cast<unsigned char*>(table + a.buckets + 1 + (a.buckets + 1 & 1)), a.live_key, about.dead, first >> 5, a.NT, wave, waves, lane);
  int head = a.by_images.div(group * units), b = group * units - head * a.B;
  bool fresh = true;                 // the first image of its head here
  for (int unit = group * units; unit < end; ++unit, ++b) {
    if (b == a.B) b = 0, ++head, fresh = true;
    const bool first_image = fresh;
    fresh = false;
    const int n = rel_tokens(a, b), bh = b * a.heads + head;
    if (unit != group * units) workgroup_barrier();       // the image before is read
    if (BIAS && first_image) table_load(2 * STAGE, table, a, head, wave, waves, lane);
    float* sums = BIAS && pairs ? pairs + (((size_t)(group - rel_first_group(head, a.B, units)) * a.heads + head) * a.NT + (u0 >> 5)) * a.NT * 1024 + lane * 4 : nullptr;
    const T* base = qkv + (size_t)b * a.T * ld + head * DH;
    const int tiles = first < n ? (n + 31) >> 5 : 0, stages = (tiles + TS - 1) / TS;
    auto tile_from = [&](int t) __attribute__((always_inline)) { return live_next(live.w, live.some, t, tiles); };
    auto stage_from = [&](int k) __attribute__((always_inline)) {
      const int t = live_next(live.all, live.some, k * TS, tiles);
      return t < tiles ? t / TS : stages;
    };
    const int stage0 = stage_from(0);
    const bool mine = u0 < n;
    f32x16_t dk[D::NM], dv[D::NM];
#pragma unroll
    for (int mt = 0; mt < D::NM; ++mt) dk[mt] = dv[mt] = zero16();
    if (stage0 < stages) {
      Stager<T, DH> st;
      st.init(base, d_o + (size_t)b * a.T * d + head * DH, (unsigned)(ld * sizeof(T)), (unsigned)(d * sizeof(T)), n, lane);
      const i32x4_t rs = make_desc(rows + (size_t)bh * 3 * a.Tp, (unsigned)a.Tp * 12u);
      auto load = [&](int s, int buf) __attribute__((always_inline)) {
        const unsigned to = buf * STAGE;
        st.load(s * D::KB, to, wave, waves);
        if (lane < D::KB) {
          for (int k = waves - 1 - wave; k < 3; k += waves) load4_to_lds(rs, to + D::STAGE + k * D::KB * 4, (unsigned)(k * a.Tp + s * D::KB + lane) * 4u);
        }
      };
      load(stage0, 0);
      int tn = mine ? tile_from(0) : tiles;
      MapRegs mr, next;
      if (BIAS && tn < tiles) map_load(next, map, tn, lane);
      typename D::Own bk, bv;
      D::own(base + d, ld, u, n, h, bk);
      D::scale(bk);
      D::own(base + 2 * d, ld, u, n, h, bv);
      int stored = 0;                // tiles whose sums this wavefront has stored since it issued the loads that it waits for
      for (int stage = stage0, buf = 0; stage < stages; buf ^= 1) {
        // Each of those tiles has left four stores behind the loads.
        asm volatile("" ::: "memory");
        if (stored >= 2) wait_vm<8>();
        else if (stored == 1) wait_vm<4>();
        else wait_vm<0>();
        stored = 0;
        workgroup_barrier();
        const int then = stage_from(stage + 1);
        if (then < stages) load(then, buf ^ 1);
        while (tn < min(tiles, (stage + 1) * TS)) {
          const int t = tn;
          tn = tile_from(t + 1);
          if (BIAS) {
            mr = next;
            if (tn < tiles) map_load(next, map, tn, lane);
          }
          float4 was[4];
          if (BIAS && !RUNS && sums) {
#pragma unroll
            for (int k = 0; k < 4; ++k) was[k] = float4{0.f, 0.f, 0.f, 0.f};
            if (!first_image) {
#pragma unroll
              for (int k = 0; k < 4; ++k) was[k] = *reinterpret_cast<const float4*>(sums + (size_t)t * 1024 + k * 256);
            }
          }
          const unsigned char *S = smem + buf * STAGE, *Qs = S + (t - stage * TS) * TILE, *Gs = Qs + D::MAT;
          const float* R = reinterpret_cast<const float*>(S + D::STAGE) + (t - stage * TS) * 32;
          f32x16_t p = score_tile<T, DH, BIAS>(Qs, bk, table, mr, a.scale, lane);
          f32x16_t dx = D::nt(Gs, bv, zero16(), lane);
          unsigned word[8];
          if (DROP) draws_by_key(word, t * 32, (unsigned)u >> 1, (unsigned)bh, key, lane);
    #pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const float* r = R + i4 * 8 + h * 4;
            const float4 m4 = *reinterpret_cast<const float4*>(r), l4 = *reinterpret_cast<const float4*>(r + D::KB), d4 = *reinterpret_cast<const float4*>(r + 2 * D::KB);
            const float mm[4] = {m4.x, m4.y, m4.z, m4.w}, ll[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int i = i4 * 4 + k;
              const float pp = __builtin_amdgcn_exp2f(fmaf(p[i] - mm[k], kLog2e, -ll[k]));
              if (DROP) {
                const bool gone = draw_of(word, i) < a.dr.q;
                p[i] = gone ? 0.f : pp;
                dx[i] = pp * ((gone ? 0.f : dx[i]) - dd[k]);
              } else {
                p[i] = pp;
                dx[i] = pp * (dx[i] - dd[k]);
              }
            }
          }
          if (BIAS && sums) {
            if (u0 + 32 > n) {       // keys past the image's tokens: probabilities that may be infinite
              only_here();
#pragma unroll
              for (int i = 0; i < 16; ++i) dx[i] = u < n ? dx[i] : 0.f;
            }
            if (!RUNS) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                *reinterpret_cast<float4*>(sums + (size_t)t * 1024 + k * 256) =
                    float4{was[k].x + dx[4 * k], was[k].y + dx[4 * k + 1], was[k].z + dx[4 * k + 2], was[k].w + dx[4 * k + 3]};
              ++stored;
            } else {
              const size_t block = (size_t)(u0 >> 5) * a.NT + t;
              const uint4* op = reinterpret_cast<const uint4*>(a.order + block * 1024 + lane * 16);
              const float4 q[4] = {{dx[0], dx[1], dx[2], dx[3]}, {dx[4], dx[5], dx[6], dx[7]}, {dx[8], dx[9], dx[10], dx[11]}, {dx[12], dx[13], dx[14], dx[15]}};
              const int runs = rel_block_runs(block_lds, q, op[0], op[1], a.ends[block * 64 + lane], lane);
              float* m = sums - lane * 4 + (size_t)t * 1024;
              for (int k = lane; k < runs; k += 64) m[k] = block_lds[k];
              __builtin_amdgcn_wave_barrier();
            }
          }
          tn_bwd<T, DH>(Gs, p, dv, lane, a.NT == 1);
          tn_bwd<T, DH>(Qs, dx, dk, lane, a.NT == 1);
        }
        stage = then;
      }
    }
    if (u0 >= a.T) continue;
    if (BIAS && sums && first_image) {      // blocks that this image has no pairs in
      for (int t = mine ? tiles : 0; t < a.NT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<float4*>(sums + (size_t)t * 1024 + k * 256) = float4{0.f, 0.f, 0.f, 0.f};
    }
    scale_rows<D::NM>(dk, a.scale * a.dr.scale, u < n);
    scale_rows<D::NM>(dv, a.dr.scale, u < n);
    T* out = dqkv + (size_t)b * a.T * ld + head * DH + d + (size_t)u * ld;
    D::store(out, dk, h, u < a.T);
    D::store(out + d, dv, h, u < a.T);
  }
}

int grid_of(int groups, int parts) {
  const int whole = whole_groups(groups, parts);
  return (whole * parts + last_share(groups, whole, parts)) * 8;
}
// More than 64 KB has to be asked for, on the device that is current: always a CU's 160 KB, so that no call takes back what another host thread's asked for.
template <typename Kern> int allow_lds(Kern kern, size_t bytes) {
  if (bytes <= 65536) return CNNK_OK;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess ? CNNK_OK : CNNK_ERR_HIP;
}
template <typename T, int DH, bool BIAS, bool DROP>
int fwd_launch(const RelArgs& a, const T* qkv, T* o, float* stats, hipStream_t st) {
  static_assert(Dim<T, DH>::STAGE == rel_stage_bytes(DH), "");
  const RelLaunch l = rel_launch(sizeof(T) == 2, DH, a.NT, a.buckets, false);
  const size_t lds = l.lds;
  const int waves = l.waves, parts = l.parts, pairs = a.B * a.heads;
  const auto kern = rel_mfma_fwd_kernel<T, DH, BIAS, DROP>;
  if (allow_lds(kern, lds) != CNNK_OK) return CNNK_ERR_HIP;
  kern<<<grid_of(pairs, parts), 64 * waves, lds, st>>>(a, qkv, o, stats, fast_div(parts));
  return launch_status();
}
template <typename T, int DH, bool BIAS, bool DROP>
int bwd_launch(const RelArgs& a, const T* qkv, const T* o, const T* d_o, const float* stats, T* dqkv, float* rows, float* pairs, int units, bool* runs, hipStream_t st) {
  const RelLaunch l = rel_launch(sizeof(T) == 2, DH, a.NT, a.buckets, true);
  const size_t lds_kv = l.lds, lds = lds_kv - 2 * 3 * Dim<T, DH>::KB * 4;
  const int waves = l.waves, parts = l.parts, heads = a.B * a.heads;
  // The walk itself adds up a block's runs (which makes it longer) where a single image's sums of pairs are more than the caches hold, so that a kernel behind it would
  // read them from memory, and where the workgroup has a CU's LDS to itself.  us of the walk, the runs and the gather, 12 heads of 64 bf16, pairs written | runs written:
  // 1024 tokens (a table for 4096) 84 | 101, 3136 tokens 401 | 340, 4096 tokens 619 | 436, 4096 tokens in windows of 15 x 15 150 | 143.  With more images it would
  // have to be done in each: 8 x 1600 tokens 571 | 632, 4 x 4096 tokens 1749 | 1911.
  *runs = pairs && a.B == 1 && waves == 8 && (size_t)a.heads * a.NT * a.NT * 4096 > (size_t)256 << 20;
  const size_t lds_runs = *runs ? waves * 4096 : 0;
  const auto dq = rel_mfma_dq_kernel<T, DH, BIAS, DROP>;
  auto dkv = rel_mfma_dkv_kernel<T, DH, BIAS, DROP, false>;
  if constexpr (BIAS && DH <= 64)
    if (*runs) dkv = rel_mfma_dkv_kernel<T, DH, BIAS, DROP, true>;
  if (allow_lds(dq, lds) != CNNK_OK || allow_lds(dkv, lds_kv + lds_runs) != CNNK_OK) return CNNK_ERR_HIP;
  dq<<<grid_of(heads, parts), 64 * waves, lds, st>>>(a, qkv, o, d_o, stats, dqkv, rows, fast_div(parts));
  dkv<<<grid_of((heads + units - 1) / units, parts), 64 * waves, lds_kv + lds_runs, st>>>(a, qkv, d_o, rows, dqkv, pairs, fast_div(parts), units, (heads + units - 1) / units,
                                                                                                               (unsigned)lds_kv);
  return launch_status();
}
template <typename T, int DH> int fwd_of(const RelArgs& a, const T* qkv, T* o, float* stats, hipStream_t st) {
  if (a.buckets) return a.dr.q ? fwd_launch<T, DH, true, true>(a, qkv, o, stats, st) : fwd_launch<T, DH, true, false>(a, qkv, o, stats, st);
  return a.dr.q ? fwd_launch<T, DH, false, true>(a, qkv, o, stats, st) : fwd_launch<T, DH, false, false>(a, qkv, o, stats, st);
}
template <typename T, int DH>
int bwd_of(const RelArgs& a, const T* qkv, const T* o, const T* d_o, const float* stats, T* dqkv, float* rows, float* pairs, int units, bool* runs, hipStream_t st) {
  if (a.buckets)
    return a.dr.q ? bwd_launch<T, DH, true, true>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st)
                  : bwd_launch<T, DH, true, false>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
  return a.dr.q ? bwd_launch<T, DH, false, true>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st)
                : bwd_launch<T, DH, false, false>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
}
}  // namespace

template <typename T> int rel_mfma_fwd(const RelArgs& a, const T* qkv, T* o, float* stats, hipStream_t st) {
  switch (a.dh) {
    case 16: return fwd_of<T, 16>(a, qkv, o, stats, st);
    case 32: return fwd_of<T, 32>(a, qkv, o, stats, st);
    case 64: return fwd_of<T, 64>(a, qkv, o, stats, st);
    default: return fwd_of<T, 128>(a, qkv, o, stats, st);
  }
}
template <typename T>
int rel_mfma_bwd(const RelArgs& a, const T* qkv, const T* o, const T* d_o, const float* stats, T* dqkv, float* rows, float* pairs, int units, bool* runs, hipStream_t st) {
  switch (a.dh) {
    case 16: return bwd_of<T, 16>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
    case 32: return bwd_of<T, 32>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
    case 64: return bwd_of<T, 64>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
    default: return bwd_of<T, 128>(a, qkv, o, d_o, stats, dqkv, rows, pairs, units, runs, st);
  }
}
