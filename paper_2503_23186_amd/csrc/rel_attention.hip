// Entry points of self-attention with a learned relative position bias (include/cnnk_rel.h), and the sums behind its backward pass: dx of every pair over
// images to a sum for each bucket.
#include "rel_attention.h"

namespace {
// Sums of a block's pairs over the workgroups' slots, then of its runs of one bucket.  A wavefront to a block and a head; the block's sums go through LDS in the
// plan's order, sixteen to a lane, and its runs to the block's place in the first slot.  A grid's map leaves 100 to 200 runs of 1024 pairs, so that the
// gather behind this moves that much less (4096 tokens, 12 heads: 695 us for a gather of all pairs, 204 and 57 this way).  Memory bounds it.
__global__ void __launch_bounds__(256) rel_runs_kernel(RelArgs a, float* pairs, int units) {
  __shared__ __align__(16) float sm[4][1024];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blocks = a.NT * a.NT, block = blockIdx.x * 4 + wave, h = blockIdx.y;
  if (block >= blocks) return;
  const uint4* op = reinterpret_cast<const uint4*>(a.order + (size_t)block * 1024 + lane * 16);
  const uint4 o0 = op[0], o1 = op[1];
  const unsigned ends = a.ends[(size_t)block * 64 + lane];
  if (!rel_plan_fits(a, rel_about(a)) || !__any(ends & 0xffffu)) return;       // masked pairs only: no walk has been there
  float* m = pairs + ((size_t)h * blocks + block) * 1024;
  const size_t slot = (size_t)a.heads * blocks * 1024;
  const int slots = rel_groups(h, a.B, units);
  float4 s[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) s[k] = *reinterpret_cast<const float4*>(m + k * 256 + lane * 4);
  int x = 1;
  for (; x + 3 < slots; x += 4) {      // in flight together
    float4 v[4][4];
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[y][k] = *reinterpret_cast<const float4*>(m + (x + y) * slot + k * 256 + lane * 4);
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k].x += v[y][k].x, s[k].y += v[y][k].y, s[k].z += v[y][k].z, s[k].w += v[y][k].w;
  }
  for (; x < slots; ++x)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(m + x * slot + k * 256 + lane * 4);
      s[k].x += v.x, s[k].y += v.y, s[k].z += v.z, s[k].w += v.w;
    }
  const int runs = rel_block_runs(sm[wave], s, o0, o1, ends, lane);
  for (int k = lane; k < runs; k += 64) m[k] = sm[wave][k];
}

// `lanes` threads to a bucket and head, which take its runs by turns; a workgroup has neighbouring buckets, whose runs lie beside each other
// in maps by distance.
__global__ void __launch_bounds__(256) rel_buckets_kernel(RelArgs a, const float* __restrict__ pairs, int lanes, float* __restrict__ dtable) {
  __shared__ float sm[256];
  const int per = 256 / lanes, k = blockIdx.x * per + threadIdx.x / lanes, h = blockIdx.y, j = threadIdx.x & (lanes - 1);
  const float* m = pairs + (size_t)h * a.NT * a.NT * 1024;
  const bool fits = rel_plan_fits(a, rel_about(a));
  float s = fits ? 0.f : NAN;
  if (fits && k < a.buckets) {
    const int s1 = a.start[k + 1];
    int i = a.start[k] + j;
    for (; i + 3 * lanes < s1; i += 4 * lanes) {
      int at[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) at[e] = a.list[i + e * lanes];
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = m[at[e]];
      s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; i < s1; i += lanes) s += m[a.list[i]];
  }
  sm[threadIdx.x] = s;
  for (int w = lanes >> 1; w > 0; w >>= 1) {
    __syncthreads();
    if (j < w) sm[threadIdx.x] += sm[threadIdx.x + w];
  }
  if (j == 0 && k < a.buckets) dtable[(size_t)k * a.heads + h] = sm[threadIdx.x] * a.dr.scale;
}

int check(const cnnk_rel_desc* d, RelDrop* dr) {
  if (!d) return CNNK_ERR_NULL;
  if (d->B <= 0 || d->T <= 0 || d->heads <= 0 || d->dh <= 0 || d->buckets < 0) return CNNK_ERR_SHAPE;
  const int rc = rel_drop(d->p, dr);
  if (rc != CNNK_OK) return rc;
  if (d->dtype != CNNK_F32 && d->dtype != CNNK_BF16) return CNNK_ERR_UNSUPPORTED;
  if (d->dh != 16 && d->dh != 32 && d->dh != 64 && d->dh != 128) return CNNK_ERR_UNSUPPORTED;
  if (d->T > 2 * kRelMaxT || (d->buckets && (d->T > kRelMaxT || d->buckets > kRelMaxBuckets))) return CNNK_ERR_UNSUPPORTED;
  if (d->heads > 65535 || (double)d->T * 3 * d->heads * d->dh * elem_size(d->dtype) >= 2147483648.0) return CNNK_ERR_UNSUPPORTED;
  if (((double)d->B * d->heads + 8) * ((d->T + 31) / 32 + 7) >= 67108864.0) return CNNK_ERR_UNSUPPORTED;
  return CNNK_OK;
}
RelArgs args_of(const cnnk_rel_desc* d, RelDrop dr, const float* table, const void* plan, const int* lens, const unsigned long long* rng) {
  RelArgs a;
  a.B = d->B;
  a.T = d->T;
  a.Tp = (d->T + 63) / 64 * 64;
  a.heads = d->heads;
  a.by_heads = fast_div(d->heads);
  a.by_images = fast_div(d->B);
  a.dh = d->dh;
  a.NT = (d->T + 31) / 32;
  a.buckets = d->buckets;
  a.scale = (float)(1.0 / sqrt((double)d->dh));
  int down = d->dtype == CNNK_BF16 ? 8 : 0;
  while (1 << (down - (d->dtype == CNNK_BF16 ? 8 : 0)) < d->T) ++down;
  a.down = (float)down;
  a.up = (float)(1 << down);
  a.site = d->site;
  a.dr = dr;
  a.table = table;
  a.by_query = a.by_key = a.order = nullptr;
  a.ends = nullptr;
  a.live_query = a.live_key = nullptr;
  a.about = nullptr;
  a.start = a.list = nullptr;
  a.lens = lens;
  a.rng = rng;
  if (d->buckets) {
    const RelPlan at = rel_plan_layout(d->T, d->buckets);
    a.by_query = (const unsigned short*)((const char*)plan + at.by_query);
    a.by_key = (const unsigned short*)((const char*)plan + at.by_key);
    a.order = (const unsigned short*)((const char*)plan + at.order);
    a.ends = (const unsigned*)((const char*)plan + at.ends);
    a.about = (const RelAbout*)((const char*)plan + at.about);
    a.live_query = (const unsigned long long*)((const char*)plan + at.live_query);
    a.live_key = (const unsigned long long*)((const char*)plan + at.live_key);
    a.start = (const int*)((const char*)plan + at.start);
    a.list = (const int*)((const char*)plan + at.list);
  }
  return a;
}
// scratch of the backward pass: three floats for each row, and the sums of every pair, as often as a head's images lie in different workgroups
size_t rows_bytes(const cnnk_rel_desc* d) { return align_up((size_t)d->B * d->heads * 3 * ((d->T + 63) / 64 * 64) * 4, 256); }
// (head, image) pairs to a workgroup of the walk for dk and dv: as many as give every workgroup that the device holds (two to a CU, or one) the same number, so that there
// is one round of them and few sums to add up (64 images of 197 tokens, 12 heads of 64: the walk 77 us, 87 with one pair to a workgroup; 16 images of 4096 tokens, 3 heads
// of 64, 16129 buckets: backward 1990 us with the three that fill the device, 2440 with six; 9 images of 2601 tokens, 12 heads of 32 the other way, 2038 with five, 1957 with
// nine, whose sums lie in two slots instead of three).
int units_of(const cnnk_rel_desc* d) {
  const RelLaunch l = rel_launch(d->dtype == CNNK_BF16, d->dh, (d->T + 31) / 32, d->buckets, true);
  const long units = ((long)d->B * d->heads * l.parts + l.held - 1) / l.held;
  return (int)(units < d->B ? units : d->B);
}
// A head's images start at a multiple of g, the greatest divisor of B and units, behind a workgroup's start: units - g at most, so that they lie in (units - g + B) / units
// workgroups, rounded up.
size_t pairs_bytes(const cnnk_rel_desc* d) {
  const size_t NT = (d->T + 31) / 32;
  const int units = units_of(d);
  int g = d->B;
  for (int r = units; r;) {
    const int next = g % r;
    g = r, r = next;
  }
  return (size_t)(1 + (d->B - g + units - 1) / units) * d->heads * NT * NT * 4096;
}
size_t workspace_bytes(const cnnk_rel_desc* d, bool dtable) { return rows_bytes(d) + (d->buckets && dtable ? pairs_bytes(d) : 0); }
}  // namespace

extern "C" int cnnk_rel_attention_fwd(const cnnk_rel_desc* d, const void* qkv, const float* table, const void* plan, const int* lens, const unsigned long long* rng,
                                      void* o, float* stats, void* stream) {
  RelDrop dr;
  const int rc = check(d, &dr);
  if (rc != CNNK_OK) return rc;
  if (!qkv || !o || (d->buckets && (!table || !plan)) || (dr.q && !rng)) return CNNK_ERR_NULL;
  if (!rel_aligned(qkv, 16) || !rel_aligned(o, 16) || !rel_aligned(stats, 8) || !rel_aligned(table, 4) || !rel_aligned(plan, 256) ||
      !rel_aligned(lens, 4) || !rel_aligned(rng, 8))
    return CNNK_ERR_UNSUPPORTED;
  const RelArgs a = args_of(d, dr, table, plan, lens, rng);
  hipStream_t st = (hipStream_t)stream;
  return d->dtype == CNNK_BF16 ? rel_mfma_fwd(a, (const bf16_t*)qkv, (bf16_t*)o, stats, st) : rel_mfma_fwd(a, (const float*)qkv, (float*)o, stats, st);
}

extern "C" size_t cnnk_rel_attention_workspace_bytes(const cnnk_rel_desc* d) {
  RelDrop dr;
  if (check(d, &dr) != CNNK_OK) return 0;
  return workspace_bytes(d, true);
}

extern "C" int cnnk_rel_attention_bwd(const cnnk_rel_desc* d, const void* qkv, const void* o, const void* d_o, const float* table, const void* plan,
                                      const int* lens, const unsigned long long* rng, const float* stats, void* dqkv, float* dtable, void* ws, size_t ws_bytes,
                                      void* stream) {
  RelDrop dr;
  const int rc = check(d, &dr);
  if (rc != CNNK_OK) return rc;
  if (!qkv || !o || !d_o || !stats || !dqkv || (d->buckets && (!table || !plan)) || (dr.q && !rng)) return CNNK_ERR_NULL;
  if (!ws || ws_bytes < workspace_bytes(d, dtable != nullptr)) return CNNK_ERR_WORKSPACE;
  if (!rel_aligned(qkv, 16) || !rel_aligned(o, 16) || !rel_aligned(d_o, 16) || !rel_aligned(stats, 8) || !rel_aligned(table, 4) ||
      !rel_aligned(plan, 256) || !rel_aligned(lens, 4) || !rel_aligned(rng, 8) || !rel_aligned(dqkv, 16) || !rel_aligned(dtable, 4) || !rel_aligned(ws, 16))
    return CNNK_ERR_UNSUPPORTED;
  const RelArgs a = args_of(d, dr, table, plan, lens, rng);
  float *rows = (float*)ws, *pairs = d->buckets && dtable ? (float*)((char*)ws + rows_bytes(d)) : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const int units = units_of(d);
  bool runs = false;
  const int r = d->dtype == CNNK_BF16
                    ? rel_mfma_bwd(a, (const bf16_t*)qkv, (const bf16_t*)o, (const bf16_t*)d_o, stats, (bf16_t*)dqkv, rows, pairs, units, &runs, st)
                    : rel_mfma_bwd(a, (const float*)qkv, (const float*)o, (const float*)d_o, stats, (float*)dqkv, rows, pairs, units, &runs, st);
  if (r != CNNK_OK || !pairs) return r;
  const int blocks = a.NT * a.NT;
  if (!runs) rel_runs_kernel<<<dim3((blocks + 3) / 4, d->heads), 256, 0, st>>>(a, pairs, units);
  // enough threads to fill the device where buckets are few (732 buckets, 12 heads: 16 threads 3.9 us, 64 4.9)
  int lanes = 8;
  while (lanes < 256 && (long)d->buckets * d->heads * lanes < 131072) lanes *= 2;
  rel_buckets_kernel<<<dim3((d->buckets + 256 / lanes - 1) / (256 / lanes), d->heads), 256, 0, st>>>(a, pairs, lanes, dtable);
  return launch_status();
}
