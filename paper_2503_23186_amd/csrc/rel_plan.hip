// Bucket maps and their plans (rel.h has the layout).  A plan is made once for a map, so these kernels are plain: a sort of each block's pairs by
// bucket, then a counting sort of all blocks' runs, stable, so that a bucket's sum has one order.
#include "rel.h"

namespace {
constexpr int kParts = 256;              // of the places of runs
constexpr unsigned short kNoRun = 0xffff;

__global__ void __launch_bounds__(256) buckets_grid_kernel(int gw, int gh, int cls, int T, int* __restrict__ bucket) {
  const int n = (2 * gh - 1) * (2 * gw - 1);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)T * T; i += (size_t)gridDim.x * 256) {
    const int t = (int)(i / (unsigned)T) - cls, u = (int)(i % (unsigned)T) - cls;
    int k;
    if (t < 0) k = u < 0 ? n + 2 : n;
    else if (u < 0) k = n + 1;
    else k = (t / gw - u / gw + gh - 1) * (2 * gw - 1) + t % gw - u % gw + gw - 1;
    bucket[i] = k;
  }
}

__global__ void __launch_bounds__(256) plan_maps_kernel(int T, int NT, int buckets, const int* __restrict__ bucket, unsigned short* __restrict__ by_query,
                                                        unsigned short* __restrict__ by_key, int* __restrict__ about) {
  if (blockIdx.x == 0 && threadIdx.x == 0) about[0] = 0, about[1] = rel_plan_mark(T, buckets);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)NT * NT * 1024; i += (size_t)gridDim.x * 256) {
    const int block = (int)(i >> 10), t = block / NT * 32 + (int)(i >> 5 & 31), u = block % NT * 32 + (int)(i & 31);
    int k = buckets;
    if (t < T && u < T) {
      k = bucket[(size_t)t * T + u];
      if (k < 0 || k >= buckets) k = buckets;
    }
    by_query[((size_t)(t >> 5) * NT + (u >> 5)) * 1024 + rel_place(u & 31, t & 31)] = (unsigned short)(4 * k);
    by_key[((size_t)(u >> 5) * NT + (t >> 5)) * 1024 + rel_place(t & 31, u & 31)] = (unsigned short)(4 * k);
  }
}

// A workgroup to a block of queries (blockIdx.y 0) or keys (1): which blocks of the others it has pairs with that are not masked
__global__ void __launch_bounds__(256) plan_live_kernel(int NT, int buckets, const unsigned short* __restrict__ by_query, const unsigned short* __restrict__ by_key,
                                                        unsigned long long* __restrict__ live_query, unsigned long long* __restrict__ live_key,
                                                        int* __restrict__ dead) {
  __shared__ unsigned any[256];
  const unsigned short* map = (blockIdx.y ? by_key : by_query) + (size_t)blockIdx.x * NT * 1024;
  any[threadIdx.x] = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int k = threadIdx.x >> 6; k < NT; k += 4) {
    bool seen = false;
    for (int i = 0; i < 16; ++i) seen |= map[(size_t)k * 1024 + i * 64 + lane] != 4 * buckets;
    if (__any(seen) && lane == 0) any[k] = 1;
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    unsigned long long m = 0;
    for (int k = 0; k < 64; ++k) m |= (unsigned long long)any[threadIdx.x * 64 + k] << k;
    (blockIdx.y ? live_key : live_query)[(size_t)blockIdx.x * 4 + threadIdx.x] = m;
    const int here = min(64, max(0, NT - 64 * (int)threadIdx.x)) - __popcll(m);
    if (blockIdx.y == 0 && here) atomicAdd(dead, here);
  }
}

// A workgroup to a block of 32 keys x 32 queries: its pairs sorted by bucket and place (bitonic), runs within sixteen of them, each run's bucket.
__global__ void __launch_bounds__(256) plan_order_kernel(int T, int NT, int buckets, const int* __restrict__ bucket, unsigned short* __restrict__ order,
                                                         unsigned* __restrict__ ends, unsigned short* __restrict__ run_bucket) {
  __shared__ unsigned key[1024];
  __shared__ unsigned before[64];
  const int block = blockIdx.x, u0 = block / NT * 32, t0 = block % NT * 32;
  for (int i = threadIdx.x; i < 1024; i += 256) {
    const int lane = i >> 2 & 63, reg = (i >> 8) * 4 + (i & 3), t = t0 + (reg >> 2) * 8 + (lane >> 5) * 4 + (reg & 3), u = u0 + (lane & 31);
    int k = buckets;
    if (t < T && u < T) {
      k = bucket[(size_t)t * T + u];
      if (k < 0 || k >= buckets) k = buckets;
    }
    key[i] = (unsigned)k << 10 | i;
    run_bucket[(size_t)block * 1024 + i] = kNoRun;
  }
  for (int size = 2; size <= 1024; size *= 2)
    for (int step = size / 2; step > 0; step /= 2) {
      __syncthreads();
      for (int p = threadIdx.x; p < 512; p += 256) {
        const int i = (p / step) * 2 * step + p % step, j = i + step;
        const unsigned a = key[i], b = key[j];
        if ((a > b) == ((i & size) == 0)) key[i] = b, key[j] = a;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 1024; i += 256) order[(size_t)block * 1024 + i] = (unsigned short)((key[i] & 1023u) * 4);
  unsigned flags = 0;
  if (threadIdx.x < 64) {
    for (int e = 0; e < 16; ++e) {
      const int i = threadIdx.x * 16 + e;
      const unsigned k = key[i] >> 10;
      if (k < (unsigned)buckets && (e == 15 || key[i + 1] >> 10 != k)) flags |= 1u << e;
    }
    before[threadIdx.x] = __popc(flags);
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    unsigned at = 0;
    for (int l = 0; l < (int)threadIdx.x; ++l) at += before[l];
    ends[(size_t)block * 64 + threadIdx.x] = flags | at << 16;
    for (int e = 0; e < 16; ++e)
      if (flags >> e & 1) run_bucket[(size_t)block * 1024 + at++] = (unsigned short)(key[threadIdx.x * 16 + e] >> 10);
  }
}

// runs of each bucket in each part
__global__ void __launch_bounds__(256) plan_count_kernel(int places, int per, int buckets, const unsigned short* __restrict__ run_bucket, int* __restrict__ count) {
  extern __shared__ int cnt[];
  for (int k = threadIdx.x; k < buckets; k += 256) cnt[k] = 0;
  __syncthreads();
  const int end = min(places, ((int)blockIdx.x + 1) * per);
  for (int i = blockIdx.x * per + threadIdx.x; i < end; i += 256) {
    const int k = run_bucket[i];
    if (k < buckets) atomicAdd(cnt + k, 1);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < buckets; k += 256) count[(size_t)blockIdx.x * buckets + k] = cnt[k];
}

// a thread to a bucket: the counts become places within the bucket, its total goes to start
__global__ void __launch_bounds__(256) plan_parts_kernel(int buckets, int* __restrict__ count, int* __restrict__ start) {
  const int k = blockIdx.x * 256 + threadIdx.x;
  if (k >= buckets) return;
  int sum = 0;
  for (int p0 = 0; p0 < kParts; p0 += 32) {
    int c[32];
#pragma unroll
    for (int p = 0; p < 32; ++p) c[p] = count[(size_t)(p0 + p) * buckets + k];
#pragma unroll
    for (int p = 0; p < 32; ++p) {
      count[(size_t)(p0 + p) * buckets + k] = sum;
      sum += c[p];
    }
  }
  start[k] = sum;
}
// totals to starts, one workgroup: every thread a run of buckets
__global__ void __launch_bounds__(1024) plan_starts_kernel(int buckets, int* __restrict__ start) {
  __shared__ int sums[1024];
  const int per = (buckets + 1023) / 1024, k0 = min(buckets, (int)threadIdx.x * per), k1 = min(buckets, k0 + per);
  int s = 0;
  for (int k = k0; k < k1; ++k) s += start[k];
  sums[threadIdx.x] = s;
  __syncthreads();
  int at = 0;
  for (int j = 0; j < (int)threadIdx.x; ++j) at += sums[j];
  for (int k = k0; k < k1; ++k) {
    const int c = start[k];
    start[k] = at;
    at += c;
  }
  if (k0 < buckets && k1 == buckets) start[buckets] = at;
}

// one wavefront to a part, 64 places at a time; among them a run comes behind those before it in the same bucket
__global__ void __launch_bounds__(64) plan_list_kernel(int places, int per, int buckets, const unsigned short* __restrict__ run_bucket, const int* __restrict__ count,
                                                       const int* __restrict__ start, int* __restrict__ list) {
  extern __shared__ int at[];
  const int lane = threadIdx.x;
  for (int k = lane; k < buckets; k += 64) at[k] = start[k] + count[(size_t)blockIdx.x * buckets + k];
  __syncthreads();
  const int end = min(places, ((int)blockIdx.x + 1) * per);
  for (int i0 = blockIdx.x * per; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    int k = i < end ? run_bucket[i] : kNoRun;
    if (k >= buckets) k = -1;
    if (!__any(k >= 0)) continue;
    int before = 0, all = 0;
    for (int j = 0; j < 64; ++j) {
      const int same = __builtin_amdgcn_readlane(k, j) == k;
      all += same;
      before += j < lane ? same : 0;
    }
    const int place = k >= 0 ? at[k] + before : 0;
    __syncthreads();
    if (k >= 0) {
      list[place] = i;
      if (before == all - 1) at[k] = place + 1;
    }
    __syncthreads();
  }
}

size_t runs_bytes(int T) {
  const size_t NT = (T + 31) / 32;
  return NT * NT * 2048;
}
bool supported(int T, int buckets) { return T <= kRelMaxT && buckets <= kRelMaxBuckets; }
}  // namespace

extern "C" int cnnk_rel_buckets_grid(int gh, int gw, int cls, int* bucket, void* stream) {
  if (gh <= 0 || gw <= 0) return CNNK_ERR_SHAPE;
  const long long T = (long long)gh * gw + (cls != 0);
  if (T > kRelMaxT || (2LL * gh - 1) * (2LL * gw - 1) + 3 * (cls != 0) > kRelMaxBuckets) return CNNK_ERR_UNSUPPORTED;
  if (!bucket) return CNNK_ERR_NULL;
  if (!rel_aligned(bucket, 4)) return CNNK_ERR_UNSUPPORTED;
  const long long blocks = (T * T + 255) / 256;
  buckets_grid_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, (hipStream_t)stream>>>(gw, gh, cls != 0, (int)T, bucket);
  return launch_status();
}

extern "C" size_t cnnk_rel_plan_bytes(int T, int buckets) {
  return T > 0 && buckets > 0 && supported(T, buckets) ? rel_plan_layout(T, buckets).bytes : 0;
}
extern "C" size_t cnnk_rel_plan_workspace_bytes(int T, int buckets) {
  return T > 0 && buckets > 0 && supported(T, buckets) ? runs_bytes(T) + align_up((size_t)kParts * buckets * 4, 256) : 0;
}

extern "C" int cnnk_rel_plan(int T, int buckets, const int* bucket, void* plan, void* ws, size_t ws_bytes, void* stream) {
  if (T <= 0 || buckets <= 0) return CNNK_ERR_SHAPE;
  if (!supported(T, buckets)) return CNNK_ERR_UNSUPPORTED;
  if (!bucket || !plan) return CNNK_ERR_NULL;
  if (!ws || ws_bytes < cnnk_rel_plan_workspace_bytes(T, buckets)) return CNNK_ERR_WORKSPACE;
  if (!rel_aligned(bucket, 4) || !rel_aligned(plan, 256) || !rel_aligned(ws, 16)) return CNNK_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  const RelPlan at = rel_plan_layout(T, buckets);
  char* p = (char*)plan;
  unsigned short* runs = (unsigned short*)ws;
  int *count = (int*)((char*)ws + runs_bytes(T)), *start = (int*)(p + at.start), *list = (int*)(p + at.list);
  const int NT = (T + 31) / 32, places = NT * NT * 1024, per = ((places + kParts - 1) / kParts + 63) / 64 * 64;
  const size_t lds = (size_t)buckets * 4, blocks = ((size_t)places + 255) / 256;
  plan_maps_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, st>>>(T, NT, buckets, bucket, (unsigned short*)(p + at.by_query), (unsigned short*)(p + at.by_key),
                                                                                       (int*)(p + at.about));
  plan_live_kernel<<<dim3(NT, 2), 256, 0, st>>>(NT, buckets, (const unsigned short*)(p + at.by_query), (const unsigned short*)(p + at.by_key),
                                               (unsigned long long*)(p + at.live_query), (unsigned long long*)(p + at.live_key), (int*)(p + at.about));
  plan_order_kernel<<<NT * NT, 256, 0, st>>>(T, NT, buckets, bucket, (unsigned short*)(p + at.order), (unsigned*)(p + at.ends), runs);
  plan_count_kernel<<<kParts, 256, lds, st>>>(places, per, buckets, runs, count);
  plan_parts_kernel<<<(buckets + 255) / 256, 256, 0, st>>>(buckets, count, start);
  plan_starts_kernel<<<1, 1024, 0, st>>>(buckets, start);
  plan_list_kernel<<<kParts, 64, lds, st>>>(places, per, buckets, runs, count, start, list);
  return launch_status();
}
