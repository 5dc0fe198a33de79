// Self-attention with a learned relative position bias, dropout of the probabilities and padded batches (include/cnnk_rel.h): the kernels
// of fp32 storage, one wavefront to a row of scores (bf16: rel_attention_mfma.hip), and the entry points.
//
// Scores of 64 keys (queries) at a time, one a lane; the products with V, K, Q and dO that follow go over the same 64 with a feature a lane,
// the factors from LDS.  Probabilities are not stored: the forward pass keeps a row's largest score and the logarithm of its sum, apart, so that
// scores near the lowest finite value lose nothing.  dx = P (dP - delta), delta = do . o.
#include "rel_attention.h"

namespace {
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

template <typename T> __device__ __forceinline__ float dot_rows(const T* a, const T* b, int dh) {
  float s = 0.f;
  for (int k = 0; k < dh; k += 8) {
    float x[8], y[8];
    load8(a + k, x);
    load8(b + k, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  }
  return s;
}
// score of query t, key u, both within the image: -infinity if masked
__device__ __forceinline__ float score(const RelArgs& a, float qk, int t, int u, int h) {
  if (!a.buckets) return qk * a.scale;
  const int k = a.by_query[((size_t)(t >> 5) * a.NT + (u >> 5)) * 1024 + rel_place(u & 31, t & 31)] >> 2;
  return k < a.buckets ? fmaf(qk, a.scale, a.table[(size_t)k * a.heads + h]) : -INFINITY;
}
__device__ __forceinline__ float keep(const RelArgs& a, RelKey key, int bh, int t, int u) {      // 1 / (1 - p) or 0
  if (!a.dr.q) return 1.f;
  const RelWords r = rel_words((unsigned)u >> 1, (unsigned)t >> 2, (unsigned)bh, kDrawPairs, key);
  const int i = t & 3;
  const unsigned w = i < 2 ? (i ? r.w[1] : r.w[0]) : (i == 2 ? r.w[2] : r.w[3]);
  return (u & 1 ? w >> 16 : w & 0xffffu) < a.dr.q ? 0.f : a.dr.scale;
}
// sum over 64 rows from `row0` (at most n) of f[j] * m[row][c], for this lane's features lane and lane + 64
template <typename T> __device__ __forceinline__ void add_rows(const float* f, const T* m, size_t ld, int row0, int n, int dh, int lane, float acc[2]) {
  const int most = min(64, n - row0);
  for (int j = 0; j < most; ++j) {
    const float w = f[j];
    const T* r = m + (size_t)(row0 + j) * ld;
    if (lane < dh) acc[0] = fmaf(w, Elem<T>::ld(r + lane), acc[0]);
    if (lane + 64 < dh) acc[1] = fmaf(w, Elem<T>::ld(r + lane + 64), acc[1]);
  }
}

template <typename T>
__global__ void __launch_bounds__(64) rel_fwd_kernel(RelArgs a, const T* __restrict__ qkv, T* __restrict__ o, float* __restrict__ stats) {
  __shared__ float f[64];
  const int bh = blockIdx.x / a.T, b = bh / a.heads, h = bh - b * a.heads, t = blockIdx.x - bh * a.T, lane = threadIdx.x, d = a.heads * a.dh, n = rel_tokens(a, b);
  const size_t ld = 3 * (size_t)d;
  const T* base = qkv + (size_t)b * a.T * ld + h * a.dh;
  float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
  if (t < n) {
    RelKey key{0u, 0u};
    if (a.dr.q) key = rel_key(a.rng, a.site);
    for (int u0 = 0; u0 < n; u0 += 64) {
      const int u = u0 + lane;
      const float x = u < n ? score(a, dot_rows(base + (size_t)t * ld, base + (size_t)u * ld + d, a.dh), t, u, h) : -INFINITY;
      const float mn = fmaxf(m, wave_max(x));
      const float ref = mn > -INFINITY ? mn : 0.f;
      const float down = __builtin_amdgcn_exp2f((m - ref) * kLog2e), p = __builtin_amdgcn_exp2f((x - ref) * kLog2e);
      l = l * down + wave_sum(p);
      acc[0] *= down;
      acc[1] *= down;
      m = mn;
      f[lane] = p * keep(a, key, bh, t, u);
      __syncthreads();
      add_rows(f, base + 2 * d, ld, u0, n, a.dh, lane, acc);
      __syncthreads();
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = lane + 64 * i;
    if (c >= a.dh) break;
    const float v = t < n ? acc[i] * inv : 0.f;
    const size_t at = ((size_t)b * a.T + t) * d + h * a.dh + c;
    Elem<T>::st(o + at, v);
  }
  if (stats && lane == 0) {
    float* s = stats + ((size_t)bh * a.T + t) * 2;
    s[0] = l > 0.f ? m : -INFINITY;
    s[1] = l > 0.f ? kLn2 * __builtin_amdgcn_logf(l) : 0.f;
  }
}

// delta of every row: a wavefront to four rows, 16 lanes to one
template <typename T>
__global__ void __launch_bounds__(256) rel_delta_kernel(RelArgs a, const T* __restrict__ o, const T* __restrict__ d_o, float* __restrict__ delta) {
  const size_t row = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4);      // (b * heads + h) * T + t
  if (row >= (size_t)a.B * a.heads * a.T) return;
  const int t = (int)(row % (unsigned)a.T), bh = (int)(row / (unsigned)a.T), b = bh / a.heads, h = bh - b * a.heads;
  const size_t at = ((size_t)b * a.T + t) * a.heads * a.dh + h * a.dh;
  float s = 0.f;
  for (int c = threadIdx.x & 15; c < a.dh; c += 16)
    s = fmaf(Elem<T>::ld(d_o + at + c), Elem<T>::ld(o + at + c), s);
  s += row_rotated<8>(s);
  s += row_rotated<4>(s);
  s += row_rotated<2>(s);
  s += row_rotated<1>(s);
  if ((threadIdx.x & 15) == 0) delta[row] = s;
}

// P, and dx = P (dP - delta), of query t and key u, both within the image; g = do_t . v_u
__device__ __forceinline__ float prob(float x, const float* st) { return st[0] > -INFINITY ? __builtin_amdgcn_exp2f((x - st[0] - st[1]) * kLog2e) : 0.f; }

template <typename T>
__global__ void __launch_bounds__(64) rel_dq_kernel(RelArgs a, const T* __restrict__ qkv, const T* __restrict__ d_o, const float* __restrict__ stats,
                                                    const float* __restrict__ delta, T* __restrict__ dqkv) {
  __shared__ float f[64];
  const int bh = blockIdx.x / a.T, b = bh / a.heads, h = bh - b * a.heads, t = blockIdx.x - bh * a.T, lane = threadIdx.x, d = a.heads * a.dh, n = rel_tokens(a, b);
  const size_t ld = 3 * (size_t)d;
  const T *base = qkv + (size_t)b * a.T * ld + h * a.dh, *g = d_o + ((size_t)b * a.T + t) * d + h * a.dh;
  float acc[2] = {0.f, 0.f};
  if (t < n) {
    RelKey key{0u, 0u};
    if (a.dr.q) key = rel_key(a.rng, a.site);
    const size_t row = (size_t)bh * a.T + t;
    for (int u0 = 0; u0 < n; u0 += 64) {
      const int u = u0 + lane;
      float dx = 0.f;
      if (u < n) {
        const T* k = base + (size_t)u * ld + d;
        const float p = prob(score(a, dot_rows(base + (size_t)t * ld, k, a.dh), t, u, h), stats + row * 2);
        dx = p * (keep(a, key, bh, t, u) * dot_rows(g, k + d, a.dh) - delta[row]);
      }
      f[lane] = dx;
      __syncthreads();
      add_rows(f, base + d, ld, u0, n, a.dh, lane, acc);
      __syncthreads();
    }
  }
  T* out = dqkv + ((size_t)b * a.T + t) * ld + h * a.dh;
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < a.dh) Elem<T>::st(out + lane + 64 * i, acc[i] * a.scale);
}

template <typename T>
__global__ void __launch_bounds__(64) rel_dkv_kernel(RelArgs a, const T* __restrict__ qkv, const T* __restrict__ d_o, const float* __restrict__ stats,
                                                     const float* __restrict__ delta, T* __restrict__ dqkv) {
  __shared__ float f[64], e[64];
  const int bh = blockIdx.x / a.T, b = bh / a.heads, h = bh - b * a.heads, u = blockIdx.x - bh * a.T, lane = threadIdx.x, d = a.heads * a.dh, n = rel_tokens(a, b);
  const size_t ld = 3 * (size_t)d;
  const T *base = qkv + (size_t)b * a.T * ld + h * a.dh, *g = d_o + (size_t)b * a.T * d + h * a.dh, *k = base + (size_t)u * ld + d;
  float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
  if (u < n) {
    RelKey key{0u, 0u};
    if (a.dr.q) key = rel_key(a.rng, a.site);
    for (int t0 = 0; t0 < n; t0 += 64) {
      const int t = t0 + lane;
      float dx = 0.f, kept = 0.f;
      if (t < n) {
        const size_t row = (size_t)bh * a.T + t;
        const float p = prob(score(a, dot_rows(base + (size_t)t * ld, k, a.dh), t, u, h), stats + row * 2), w = keep(a, key, bh, t, u);
        kept = p * w;
        dx = p * (w * dot_rows(g + (size_t)t * d, k + d, a.dh) - delta[row]);
      }
      f[lane] = dx;
      e[lane] = kept;
      __syncthreads();
      add_rows(f, base, ld, t0, n, a.dh, lane, dk);
      add_rows(e, g, d, t0, n, a.dh, lane, dv);
      __syncthreads();
    }
  }
  T* out = dqkv + ((size_t)b * a.T + u) * ld + d + h * a.dh;
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < a.dh) {
      Elem<T>::st(out + lane + 64 * i, dk[i] * a.scale);
      Elem<T>::st(out + d + lane + 64 * i, dv[i]);
    }
}

// dx of every pair summed over the images, in the order of the plan's list: [heads][NT][NT][4][64][4]
template <typename T>
__global__ void __launch_bounds__(256) rel_pairs_kernel(RelArgs a, const T* __restrict__ qkv, const T* __restrict__ d_o, const float* __restrict__ stats,
                                                        const float* __restrict__ delta, float* __restrict__ pairs) {
  const int h = blockIdx.y, d = a.heads * a.dh;
  const size_t ld = 3 * (size_t)d, i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int block = (int)(i >> 10), t = block / a.NT * 32 + (int)(i >> 5 & 31), u = block % a.NT * 32 + (int)(i & 31);
  RelKey key{0u, 0u};
  if (a.dr.q) key = rel_key(a.rng, a.site);
  float sum = 0.f;
  for (int b = 0; b < a.B; ++b) {
    const int n = rel_tokens(a, b), bh = b * a.heads + h;
    if (t >= n || u >= n) continue;
    const T *base = qkv + (size_t)b * a.T * ld + h * a.dh, *k = base + (size_t)u * ld + d, *g = d_o + ((size_t)b * a.T + t) * d + h * a.dh;
    const size_t row = (size_t)bh * a.T + t;
    const float p = prob(score(a, dot_rows(base + (size_t)t * ld, k, a.dh), t, u, h), stats + row * 2);
    sum += p * (keep(a, key, bh, t, u) * dot_rows(g, k + d, a.dh) - delta[row]);
  }
  pairs[(size_t)h * a.NT * a.NT * 1024 + rel_sum_place(a.NT, t, u)] = sum;
}

// the splits' sums of the pairs into the first's place
__global__ void __launch_bounds__(256) rel_splits_kernel(float4* pairs, size_t n, int splits) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float4 s = pairs[i];
  for (int k = 1; k < splits; ++k) {
    const float4 v = pairs[k * n + i];
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  pairs[i] = s;
}

// `lanes` threads to a bucket and head, which take its pairs by turns; a workgroup has neighbouring buckets, whose pairs lie beside each other
// in maps by distance.
__global__ void __launch_bounds__(256) rel_buckets_kernel(RelArgs a, const float* __restrict__ pairs, int lanes, float* __restrict__ dtable) {
  __shared__ float sm[256];
  const int per = 256 / lanes, k = blockIdx.x * per + threadIdx.x / lanes, h = blockIdx.y, j = threadIdx.x & (lanes - 1);
  const float* m = pairs + (size_t)h * a.NT * a.NT * 1024;
  float s = 0.f;
  if (k < a.buckets) {
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
  if (j == 0 && k < a.buckets) dtable[(size_t)k * a.heads + h] = sm[threadIdx.x];
}

int check(const cnnk_rel_desc* d, RelDrop* dr) {
  if (!d) return CNNK_ERR_NULL;
  if (d->B <= 0 || d->T <= 0 || d->heads <= 0 || d->dh <= 0 || d->buckets < 0) return CNNK_ERR_SHAPE;
  const int rc = rel_drop(d->p, dr);
  if (rc != CNNK_OK) return rc;
  if (d->dtype != CNNK_F32 && d->dtype != CNNK_BF16) return CNNK_ERR_UNSUPPORTED;
  if (d->dh != 16 && d->dh != 32 && d->dh != 64 && d->dh != 128) return CNNK_ERR_UNSUPPORTED;
  if (d->T > 2 * kRelMaxT || (d->buckets && (d->T > kRelMaxT || d->buckets > kRelMaxBuckets))) return CNNK_ERR_UNSUPPORTED;
  if (d->heads > 65535 || (double)d->T * 3 * d->heads * d->dh * elem_size(d->dtype) >= 2147483648.0 || (double)d->B * d->heads * ((d->T + 31) / 32) > 2147483647.0 / 32) return CNNK_ERR_UNSUPPORTED;
  return CNNK_OK;
}
RelArgs args_of(const cnnk_rel_desc* d, RelDrop dr, const float* table, const void* plan, const int* lens, const unsigned long long* rng) {
  RelArgs a;
  a.B = d->B;
  a.T = d->T;
  a.Tp = (d->T + 63) / 64 * 64;
  a.heads = d->heads;
  a.dh = d->dh;
  a.NT = (d->T + 31) / 32;
  a.buckets = d->buckets;
  a.scale = (float)(1.0 / sqrt((double)d->dh));
  a.site = d->site;
  a.dr = dr;
  a.table = table;
  a.by_query = a.by_key = nullptr;
  a.start = a.list = nullptr;
  a.lens = lens;
  a.rng = rng;
  if (d->buckets) {
    const RelPlan at = rel_plan_layout(d->T, d->buckets);
    a.by_query = (const unsigned short*)((const char*)plan + at.by_query);
    a.by_key = (const unsigned short*)((const char*)plan + at.by_key);
    a.start = (const int*)((const char*)plan + at.start);
    a.list = (const int*)((const char*)plan + at.list);
  }
  return a;
}
// scratch of the backward pass: three floats for each row, and the sums of every pair, `splits` times over
size_t rows_bytes(const cnnk_rel_desc* d) { return align_up((size_t)d->B * d->heads * 3 * ((d->T + 63) / 64 * 64) * 4, 256); }
int splits_of(const cnnk_rel_desc* d) {
  if (d->dtype == CNNK_F32) return 1;
  const long NT = (d->T + 31) / 32, groups = d->heads * ((NT + 3) / 4), want = (512 + groups - 1) / groups;
  return (int)(want < d->B ? want : d->B);
}
size_t pairs_bytes(const cnnk_rel_desc* d) {
  const size_t NT = (d->T + 31) / 32;
  return (size_t)splits_of(d) * d->heads * NT * NT * 4096;
}

int fwd_f32(const RelArgs& a, const float* qkv, float* o, float* stats, hipStream_t st) {
  rel_fwd_kernel<float><<<(unsigned)(a.T * a.B * a.heads), 64, 0, st>>>(a, qkv, o, stats);
  return launch_status();
}
int bwd_f32(const RelArgs& a, const float* qkv, const float* o, const float* d_o, const float* stats, float* dqkv, float* rows, float* pairs, hipStream_t st) {
  const unsigned n = (unsigned)(a.T * a.B * a.heads);
  rel_delta_kernel<float><<<(n + 15) / 16, 256, 0, st>>>(a, o, d_o, rows);
  rel_dq_kernel<float><<<n, 64, 0, st>>>(a, qkv, d_o, stats, rows, dqkv);
  rel_dkv_kernel<float><<<n, 64, 0, st>>>(a, qkv, d_o, stats, rows, dqkv);
  if (pairs) rel_pairs_kernel<float><<<dim3(a.NT * a.NT * 4, a.heads), 256, 0, st>>>(a, qkv, d_o, stats, rows, pairs);
  return launch_status();
}
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
  return d->dtype == CNNK_BF16 ? rel_mfma_fwd(a, qkv, o, stats, st) : fwd_f32(a, (const float*)qkv, (float*)o, stats, st);
}

extern "C" size_t cnnk_rel_attention_workspace_bytes(const cnnk_rel_desc* d) {
  RelDrop dr;
  if (check(d, &dr) != CNNK_OK) return 0;
  return rows_bytes(d) + (d->buckets ? pairs_bytes(d) : 0);
}

extern "C" int cnnk_rel_attention_bwd(const cnnk_rel_desc* d, const void* qkv, const void* o, const void* d_o, const float* table, const void* plan,
                                      const int* lens, const unsigned long long* rng, const float* stats, void* dqkv, float* dtable, void* ws, size_t ws_bytes,
                                      void* stream) {
  RelDrop dr;
  const int rc = check(d, &dr);
  if (rc != CNNK_OK) return rc;
  if (!qkv || !o || !d_o || !stats || !dqkv || (d->buckets && (!table || !plan)) || (dr.q && !rng)) return CNNK_ERR_NULL;
  if (!ws || ws_bytes < cnnk_rel_attention_workspace_bytes(d)) return CNNK_ERR_WORKSPACE;
  if (!rel_aligned(qkv, 16) || !rel_aligned(o, 16) || !rel_aligned(d_o, 16) || !rel_aligned(stats, 8) || !rel_aligned(table, 4) ||
      !rel_aligned(plan, 256) || !rel_aligned(lens, 4) || !rel_aligned(rng, 8) || !rel_aligned(dqkv, 16) || !rel_aligned(dtable, 4) || !rel_aligned(ws, 256))
    return CNNK_ERR_UNSUPPORTED;
  const RelArgs a = args_of(d, dr, table, plan, lens, rng);
  float *rows = (float*)ws, *pairs = d->buckets && dtable ? (float*)((char*)ws + rows_bytes(d)) : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const int splits = splits_of(d);
  const int r = d->dtype == CNNK_BF16 ? rel_mfma_bwd(a, qkv, o, d_o, stats, dqkv, rows, pairs, splits, st)
                                      : bwd_f32(a, (const float*)qkv, (const float*)o, (const float*)d_o, stats, (float*)dqkv, rows, pairs, st);
  if (r != CNNK_OK || !pairs) return r;
  if (splits > 1) {
    const size_t n = (size_t)d->heads * a.NT * a.NT * 256;
    rel_splits_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>((float4*)pairs, n, splits);
  }
  // enough threads to fill the device where buckets are few
  int lanes = 8;
  while (lanes < 256 && (long)d->buckets * d->heads * lanes < 131072) lanes *= 2;
  rel_buckets_kernel<<<dim3((d->buckets + 256 / lanes - 1) / (256 / lanes), d->heads), 256, 0, st>>>(a, pairs, lanes, dtable);
  return launch_status();
}
