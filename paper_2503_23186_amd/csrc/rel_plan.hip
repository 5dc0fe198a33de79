// Bucket maps and their plans (rel.h has the layout).  A plan is made once for a map, so these kernels are plain: a counting sort of the pairs
// by bucket in parts of the map, stable, so that a bucket's sum has one order.
#include "rel.h"

namespace {
constexpr int kParts = 256;      // of the T * T pairs

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
                                                        unsigned short* __restrict__ by_key) {
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

// pairs of each bucket in each part
__global__ void __launch_bounds__(256) plan_count_kernel(int pairs, int per, int buckets, const int* __restrict__ bucket, int* __restrict__ count) {
  extern __shared__ int cnt[];
  for (int k = threadIdx.x; k < buckets; k += 256) cnt[k] = 0;
  __syncthreads();
  const int end = min(pairs, ((int)blockIdx.x + 1) * per);
  for (int i = blockIdx.x * per + threadIdx.x; i < end; i += 256) {
    const int k = bucket[i];
    if (k >= 0 && k < buckets) atomicAdd(cnt + k, 1);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < buckets; k += 256) count[(size_t)blockIdx.x * buckets + k] = cnt[k];
}

// a thread to a bucket: the counts become places within the bucket, its total goes to start
__global__ void __launch_bounds__(256) plan_parts_kernel(int buckets, int* __restrict__ count, int* __restrict__ start) {
  const int k = blockIdx.x * 256 + threadIdx.x;
  if (k >= buckets) return;
  int sum = 0;
  for (int p = 0; p < kParts; ++p) {
    const int c = count[(size_t)p * buckets + k];
    count[(size_t)p * buckets + k] = sum;
    sum += c;
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

// one wavefront to a part, 64 pairs at a time; among them a pair comes behind those before it in the same bucket
__global__ void __launch_bounds__(64) plan_list_kernel(int T, int NT, int pairs, int per, int buckets, const int* __restrict__ bucket, const int* __restrict__ count,
                                                       const int* __restrict__ start, int* __restrict__ list) {
  extern __shared__ int at[];
  const int lane = threadIdx.x;
  for (int k = lane; k < buckets; k += 64) at[k] = start[k] + count[(size_t)blockIdx.x * buckets + k];
  __syncthreads();
  const int end = min(pairs, ((int)blockIdx.x + 1) * per);
  for (int i0 = blockIdx.x * per; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    int k = i < end ? bucket[i] : -1;
    if (k < 0 || k >= buckets) k = -1;
    int before = 0, all = 0;
    for (int j = 0; j < 64; ++j) {
      const int same = __builtin_amdgcn_readlane(k, j) == k;
      all += same;
      before += j < lane ? same : 0;
    }
    const int place = k >= 0 ? at[k] + before : 0;
    __syncthreads();
    if (k >= 0) {
      const int t = i / T, u = i - t * T;
      list[place] = rel_sum_place(NT, t, u);
      if (before == all - 1) at[k] = place + 1;
    }
    __syncthreads();
  }
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
  return T > 0 && buckets > 0 && supported(T, buckets) ? align_up((size_t)kParts * buckets * 4, 256) : 0;
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
  int *count = (int*)ws, *start = (int*)(p + at.start), *list = (int*)(p + at.list);
  const int NT = (T + 31) / 32, pairs = T * T, per = ((pairs + kParts - 1) / kParts + 63) / 64 * 64;
  const size_t lds = (size_t)buckets * 4, blocks = ((size_t)NT * NT * 1024 + 255) / 256;
  plan_maps_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, st>>>(T, NT, buckets, bucket, (unsigned short*)(p + at.by_query), (unsigned short*)(p + at.by_key));
  plan_count_kernel<<<kParts, 256, lds, st>>>(pairs, per, buckets, bucket, count);
  plan_parts_kernel<<<(buckets + 255) / 256, 256, 0, st>>>(buckets, count, start);
  plan_starts_kernel<<<1, 1024, 0, st>>>(buckets, start);
  plan_list_kernel<<<kParts, 64, lds, st>>>(T, NT, pairs, per, buckets, bucket, count, start, list);
  return launch_status();
}
