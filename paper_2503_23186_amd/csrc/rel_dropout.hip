// Dropout and stochastic depth from the counter-based generator of rel.h, with the bias in front and the residual sum behind.
// The mask is never stored: both directions form the draws of an octet of elements from its place, one call of the generator
// (four words, eight 16-bit draws) to 16 bytes of bf16.
#include "rel.h"
#include "vit.h"

namespace {
constexpr int kT = 256;

__global__ void rng_advance_kernel(unsigned long long* rng, unsigned long long by) { rng[1] += by; }

// Eight neighbours of row `row`, times keep / (1 - p).  There are fewer than 2^31 octets and rows, so that the counter's second word is 0 and
// divisions are multiplications (12608 x 768 bf16 with a residual sum 14.9 -> 14.5 us, the gradient with its sums 12.4 -> 11.3).
__device__ __forceinline__ void drop8(float* v, int octet, int row, FastDiv span, RelKey key, RelDrop dr) {
  if (span.d > 0) {
    const int i = span.div(row);
    const RelWords r = rel_words((unsigned)i >> 3, 0u, 0u, kDrawGroups, key);
    const unsigned k = (unsigned)i & 7u, w = k < 4 ? (k < 2 ? r.w[0] : r.w[1]) : (k < 6 ? r.w[2] : r.w[3]);
    const bool dropped = ((k & 1u ? w >> 16 : w & 0xffffu)) < dr.q;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = dropped ? 0.f : v[e] * dr.scale;
  } else {
    const RelWords r = rel_words((unsigned)octet, 0u, 0u, kDrawElements, key);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned draw = e & 1 ? r.w[e >> 1] >> 16 : r.w[e >> 1] & 0xffffu;
      v[e] = draw < dr.q ? 0.f : v[e] * dr.scale;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kT) dropout_kernel(const T* z, const float* __restrict__ bias, const T* res, const unsigned long long* __restrict__ rng,
                                                     T* y, int octets, FastDiv C8, FastDiv span, unsigned site, RelDrop dr) {
  RelKey key{0u, 0u};
  if (dr.q) key = rel_key(rng, site);
  for (long long at = (long long)blockIdx.x * kT + threadIdx.x; at < octets; at += (long long)gridDim.x * kT) {
    const int o = (int)at;
    int row, c;
    C8.divmod(o, &row, &c);
    float v[8];
    load8(z + at * 8, v);
    if (bias) {
      float b[8];
      load8(bias + c * 8, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += b[e];
    }
    if (dr.q) drop8(v, o, row, span, key, dr);
    if (res) {
      float r[8];
      load8(res + at * 8, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    store8(y + at * 8, v);
  }
}

// The backward pass with the sums over rows: 32 column octets x 8 row lanes per workgroup, blockIdx.x = slab of 256 columns, blockIdx.y = rows.
template <typename T>
__global__ void __launch_bounds__(kT) dropout_sum_kernel(const T* dy, const unsigned long long* __restrict__ rng, T* dz, float* __restrict__ part,
                                                         int rows, int C, int rows_per_chunk, FastDiv span, unsigned site, RelDrop dr) {
  __shared__ float sm[8][257];
  const int oc = threadIdx.x & 31, rl = threadIdx.x >> 5, c = blockIdx.x * 256 + oc * 8;
  const long long r0 = (long long)blockIdx.y * rows_per_chunk;
  const long long r1 = r0 + rows_per_chunk < rows ? r0 + rows_per_chunk : rows;
  RelKey key{0u, 0u};
  if (dr.q) key = rel_key(rng, site);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < C) {
    long long r = r0 + rl;
    for (; r + 8 < r1; r += 16) {          // two rows in flight
      float v[8], w[8];
      const size_t at = (size_t)r * C + c, bt = at + (size_t)8 * C;
      load8(dy + at, v);
      load8(dy + bt, w);
      if (dr.q) {
        drop8(v, (int)(at >> 3), (int)r, span, key, dr);
        drop8(w, (int)(bt >> 3), (int)r + 8, span, key, dr);
      }
      store8(dz + at, v);
      store8(dz + bt, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += w[e];
    }
    for (; r < r1; r += 8) {
      float v[8];
      const size_t at = (size_t)r * C + c;
      load8(dy + at, v);
      if (dr.q) drop8(v, (int)(at >> 3), (int)r, span, key, dr);
      store8(dz + at, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sm[rl][oc * 8 + e] = acc[e];
  __syncthreads();
  const int cc = blockIdx.x * 256 + threadIdx.x;
  if (cc < C) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += sm[k][threadIdx.x];
    part[(size_t)blockIdx.y * C + cc] = s;
  }
}

int check(const cnnk_dropout_desc* d, RelDrop* dr) {
  if (!d) return CNNK_ERR_NULL;
  if (d->rows <= 0 || d->C <= 0 || d->span < 0) return CNNK_ERR_SHAPE;
  const int rc = rel_drop(d->p, dr);
  if (rc != CNNK_OK) return rc;
  if (d->dtype != CNNK_F32 && d->dtype != CNNK_BF16) return CNNK_ERR_UNSUPPORTED;
  if (d->C % 8 != 0 || (double)d->rows * d->C > 2147483647.0 * 8) return CNNK_ERR_UNSUPPORTED;
  return CNNK_OK;
}
constexpr int kMaxSumC = 1 << 30;      // columns of sums: slabs of 256 are counted in 32 bits
int chunks_of(long long rows, int C) {
  const int slabs = (C + 255) / 256;
  long long want = 2048 / slabs, by_rows = (rows + 63) / 64;
  if (want < 1) want = 1;
  return (int)(want < by_rows ? want : by_rows);
}
FastDiv span_of(const cnnk_dropout_desc* d) {
  FastDiv f;
  f.init(d->span);
  f.d = d->span;
  return f;
}
void pass(const cnnk_dropout_desc* d, const void* z, const float* bias, const void* res, const unsigned long long* rng, void* y, RelDrop dr, hipStream_t st) {
  const long long octets = d->rows * d->C / 8, blocks = (octets + kT - 1) / kT;
  FastDiv C8;
  C8.init(d->C / 8);
  const unsigned grid = (unsigned)(blocks < 16384 ? blocks : 16384);
  if (d->dtype == CNNK_BF16)
    dropout_kernel<bf16_t><<<grid, kT, 0, st>>>((const bf16_t*)z, bias, (const bf16_t*)res, rng, (bf16_t*)y, (int)octets, C8, span_of(d), d->site, dr);
  else
    dropout_kernel<float><<<grid, kT, 0, st>>>((const float*)z, bias, (const float*)res, rng, (float*)y, (int)octets, C8, span_of(d), d->site, dr);
}
}  // namespace

extern "C" int cnnk_rng_advance(unsigned long long* rng, unsigned long long by, void* stream) {
  if (!rng) return CNNK_ERR_NULL;
  if (!rel_aligned(rng, 8)) return CNNK_ERR_UNSUPPORTED;
  rng_advance_kernel<<<1, 1, 0, (hipStream_t)stream>>>(rng, by);
  return launch_status();
}

extern "C" int cnnk_dropout_fwd(const cnnk_dropout_desc* d, const void* z, const float* bias, const void* res, const unsigned long long* rng, void* y,
                                void* stream) {
  RelDrop dr;
  const int rc = check(d, &dr);
  if (rc != CNNK_OK) return rc;
  if (!z || !y || (dr.q && !rng)) return CNNK_ERR_NULL;
  if (!rel_aligned(z, 16) || !rel_aligned(y, 16) || !rel_aligned(bias, 16) || !rel_aligned(res, 16) || !rel_aligned(rng, 8)) return CNNK_ERR_UNSUPPORTED;
  pass(d, z, bias, res, rng, y, dr, (hipStream_t)stream);
  return launch_status();
}

extern "C" size_t cnnk_dropout_workspace_bytes(const cnnk_dropout_desc* d) {
  RelDrop dr;
  if (check(d, &dr) != CNNK_OK || d->C > kMaxSumC) return 0;
  return align_up((size_t)chunks_of(d->rows, d->C) * d->C * sizeof(float), 256);
}

extern "C" int cnnk_dropout_bwd(const cnnk_dropout_desc* d, const void* dy, const unsigned long long* rng, void* dz, float* dbias, void* ws, size_t ws_bytes,
                                void* stream) {
  RelDrop dr;
  const int rc = check(d, &dr);
  if (rc != CNNK_OK) return rc;
  if (!dy || !dz || (dr.q && !rng)) return CNNK_ERR_NULL;
  if (dbias && d->C > kMaxSumC) return CNNK_ERR_UNSUPPORTED;
  if (dbias && (!ws || ws_bytes < cnnk_dropout_workspace_bytes(d))) return CNNK_ERR_WORKSPACE;
  if (!rel_aligned(dy, 16) || !rel_aligned(dz, 16) || !rel_aligned(rng, 8) || !rel_aligned(dbias, 4) || (dbias && !rel_aligned(ws, 16))) return CNNK_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  if (!dbias) {
    pass(d, dy, nullptr, nullptr, rng, dz, dr, st);
    return launch_status();
  }
  const int chunks = chunks_of(d->rows, d->C);
  const int rpc = (int)((d->rows + chunks - 1) / chunks);
  const dim3 grid((d->C + 255) / 256, chunks);
  float* part = (float*)ws;
  if (d->dtype == CNNK_BF16)
    dropout_sum_kernel<bf16_t><<<grid, kT, 0, st>>>((const bf16_t*)dy, rng, (bf16_t*)dz, part, (int)d->rows, d->C, rpc, span_of(d), d->site, dr);
  else
    dropout_sum_kernel<float><<<grid, kT, 0, st>>>((const float*)dy, rng, (float*)dz, part, (int)d->rows, d->C, rpc, span_of(d), d->site, dr);
  if (launch_status() != CNNK_OK) return CNNK_ERR_HIP;
  ColumnSums sums;
  sums.count = 1;
  sums.it[0] = {part, dbias, dbias + d->C / 2, chunks, d->C / 2};
  return column_sums_group(sums, st);
}
