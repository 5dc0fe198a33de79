// What the kernels behind include/cnnk_rel.h share: the generator of dropout, the layout of a bucket plan, argument checks.
#pragma once
#include "common.h"
#include "../../include/cnnk_rel.h"

// ---- generator -----------------------------------------------------------------------------------------------
// Philox4x32 with seven rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, SC 2011), the fewest with which its authors found no
// failing test.  A round is two 32 x 32 -> 64-bit products (v_mad_u64_u32).
// UNIFORM: of values that all lanes share, on the scalar unit
template <bool UNIFORM> __device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) {
  return UNIFORM ? a ^ b ^ c : __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}
struct RelWords { unsigned w[4]; };
struct RelKey { unsigned k0, k1; };
template <bool UNIFORM = false>
__device__ __forceinline__ RelWords rel_words(unsigned c0, unsigned c1, unsigned c2, unsigned c3, RelKey k) {
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = xor3<UNIFORM>((unsigned)(b >> 32), c1, k.k0);
    c1 = (unsigned)b;
    c2 = xor3<UNIFORM>((unsigned)(a >> 32), c3, k.k1);
    c3 = (unsigned)a;
    k.k0 += 0x9E3779B9u;
    k.k1 += 0xBB67AE85u;
  }
  return RelWords{{c0, c1, c2, c3}};
}
// the key of a call site in this step
__device__ __forceinline__ RelKey rel_key(const unsigned long long* rng, unsigned site) {
  const unsigned long long seed = rng[0], step = rng[1];
  const RelWords r = rel_words<true>((unsigned)step, (unsigned)(step >> 32), site, 0u, RelKey{(unsigned)seed, (unsigned)(seed >> 32)});
  return RelKey{r.w[0], r.w[1]};
}
constexpr unsigned kDrawElements = 0, kDrawGroups = 1, kDrawPairs = 2;      // last word of the counter

// p as a call takes it: elements whose 16-bit draw is below q are dropped, the others scaled by `scale`
struct RelDrop { unsigned q; float scale, keep; };      // keep: 1 / scale, exactly
static inline int rel_drop(float p, RelDrop* out) {
  if (!(p >= 0.f && p < 1.f)) return CNNK_ERR_SHAPE;
  out->q = (unsigned)((double)p * 65536.0 + 0.5);
  if (out->q >= 65536u) return CNNK_ERR_UNSUPPORTED;
  out->scale = (float)(65536.0 / (65536.0 - out->q));
  out->keep = (float)(65536 - out->q) / 65536.f;
  return CNNK_OK;
}

static inline bool rel_aligned(const void* p, size_t a) { return ((size_t)p & (a - 1)) == 0; }

// ---- bucket plan -----------------------------------------------------------------------------------------------
// Pairs in 32 x 32 blocks, block (t / 32, u / 32) row by row, in a block 64 lanes of 16 in the order in which a wavefront holds the accumulator of
// a 32 x 32 matrix product with one column a lane: lane (r / 4 % 2) * 32 + c, register (r / 8) * 4 + r % 4 for row r, column c.
//   by_query  a lane a query (column), its registers keys    u16 [NT][NT][64][16]
//   by_key    a lane a key, its registers queries, block (u / 32, t / 32)
// An entry is 4 x bucket, the byte offset into a head's table in LDS; 4 x buckets for masked pairs and for padding, where that table holds -infinity.
//   live_query, live_key   u64 [NT][4]: bit k of a block of queries (keys): its pairs with block k of the others are not all masked.  The walks
//             leave the others out.
//   about     int [2]: how many blocks that are; rel_plan_mark, so that a kernel can tell a plan of other sizes, and memory that holds none
// What reduces dx of the pairs, summed over images, to buckets.  These sums lie in blocks as in by_key, in a block registers in fours [4][64 lanes][4].
//   order     u16 [NT][NT][64][16]: a block's pairs sorted by bucket (masked ones last), sixteen to a lane: their bytes in the block
//   ends      u32 [NT][NT][64]: low half: which of a lane's sixteen end a run of one bucket; high half: runs of the lanes before
//             (a lane's runs go to the block's own place, one behind the other)
//   start     int [buckets + 1]: where a bucket's runs begin in
//   list      int [T * T at most]: places of its runs, in the order of the blocks
constexpr int kRelMaxT = 8192, kRelMaxBuckets = 16382;
// negative and odd: no two entries of a map or an order (multiples of 4), no word of ends, start or list (not negative)
__host__ __device__ static inline int rel_plan_mark(int T, int buckets) { return ~(T << 16 | buckets << 2); }
struct RelPlan { size_t by_query, by_key, order, ends, live_query, live_key, about, start, list, bytes; };
static inline RelPlan rel_plan_layout(int T, int buckets) {
  const size_t NT = (T + 31) / 32, map = NT * NT * 2048;
  RelPlan p;
  p.by_query = 0;
  p.by_key = map;
  p.order = 2 * map;
  p.ends = 3 * map;
  p.live_query = p.ends + NT * NT * 256;
  p.live_key = p.live_query + NT * 32;
  p.about = p.live_query + align_up(NT * 64, 256);
  p.start = p.about + 256;
  p.list = p.start + align_up((size_t)(buckets + 1) * 4, 256);
  p.bytes = p.list + align_up((size_t)T * T * 4, 256);
  return p;
}
// place of row r, column c of a block in its 1024 entries
__host__ __device__ __forceinline__ int rel_place(int r, int c) { return (((r >> 2 & 1) << 5 | c) << 4) | (r >> 3) << 2 | (r & 3); }
