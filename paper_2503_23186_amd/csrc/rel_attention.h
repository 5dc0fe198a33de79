// What the attention kernels behind include/cnnk_rel.h get (rel_attention_mfma.h), and how the entry points (rel_attention.hip) reach them.
#pragma once
#include "rel.h"

static inline FastDiv fast_div(unsigned d) {
  FastDiv f;
  f.init(d);
  return f;
}
struct RelAbout { int dead, mark; };         // blocks that are masked as a whole, rel_plan_mark
struct RelArgs {
  int B, T, Tp, heads, dh, NT, buckets;      // Tp: T rounded up to 64, NT: blocks of 32
  FastDiv by_heads, by_images;
  float scale;                               // 1 / sqrt(dh)
  float down, up;                            // log2 of what probabilities are divided by while they are summed, and 2^down
  unsigned site;
  RelDrop dr;
  const float* table;
  const unsigned short *by_query, *by_key, *order;
  const unsigned* ends;
  const RelAbout* about;
  const unsigned long long *live_query, *live_key;
  const int *start, *list, *lens;
  const unsigned long long* rng;
};
// tokens of image b
__device__ __forceinline__ int rel_tokens(const RelArgs& a, int b) {
  if (!a.lens) return a.T;
  const int n = a.lens[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

// Whether the plan is one for the call's T and buckets, which a call cannot see before it is enqueued: with another its results are NaN, and nothing that the plan holds
// becomes an address of memory.  The walks load it with the rest and look at it when that is on its way, all five kernels with scalar loads (8 images of 197 tokens, 12 heads:
// forward 9.6 -> 9.7 us in evaluation, a training step's five kernels 53.4 -> 54.0; compared where it is loaded, 9.9 and 54.0).
__device__ __forceinline__ RelAbout rel_about(const RelArgs& a) {
  const auto p = (const __attribute__((address_space(4))) int*)(unsigned long long)a.about;      // constant while a kernel runs
  return RelAbout{p[0], p[1]};
}
__device__ __forceinline__ bool rel_plan_fits(const RelArgs& a, RelAbout about) { return about.mark == rel_plan_mark(a.T, a.buckets); }

// A block's sums by runs of one bucket (the plan's order): four quads of a lane in, the runs' sums out, one behind the other in the wavefront's 4 KB of LDS;
// returns their number.
__device__ __forceinline__ int rel_block_runs(float* mine, const float4 (&s)[4], uint4 o0, uint4 o1, unsigned ends, int lane) {
#pragma unroll
  for (int k = 0; k < 4; ++k) *reinterpret_cast<float4*>(mine + k * 256 + lane * 4) = s[k];
  __builtin_amdgcn_wave_barrier();      // the wavefront's own part of LDS, which it uses in order
  const unsigned w[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(mine) + (e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu));
  __builtin_amdgcn_wave_barrier();
  float* out = mine + (ends >> 16);
  float run = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    run += v[e];
    *out = run;       // over itself until the run ends: with a branch around the store the walk of 4096 tokens, 12 heads took 375 us instead of 349
    const unsigned last = ends >> e & 1;
    out += last;
    run = last ? 0.f : run;
  }
  __builtin_amdgcn_wave_barrier();
  return __builtin_amdgcn_readlane((int)((ends >> 16) + __popc(ends & 0xffffu)), 63);
}

// How a walk is launched: the LDS of its workgroup (two stages of 4 KB a plane of 32 features and matrix, the head's column of the table, which blocks are there, in the walk for
// dk and dv a stage's rows of statistics), its wavefronts, the parts of a (head, image) pair, and how many workgroups the device holds of the walk for dk and dv.
constexpr int kLiveBytes = 9 * 32;
constexpr size_t rel_stage_bytes(int dh) { return (size_t)(dh + 31) / 32 * 2 * 4096; }
struct RelLaunch { size_t lds; int waves, parts, held; };
static inline RelLaunch rel_launch(bool bf16, int dh, int NT, int buckets, bool backward) {
  RelLaunch l;
  l.lds = 2 * rel_stage_bytes(dh) + (buckets ? align_up((size_t)(buckets + 2) / 2 * 8 + kLiveBytes, 16) : 0) + (backward ? 2 * 3 * (bf16 ? 64 : 32) * 4 : 0);
  // Eight wavefronts where a CU's LDS holds one workgroup (and the registers are there: the backward walks of heads of 128 take those of a SIMD for one wavefront), otherwise
  // four (4096 tokens, 12 heads of 64, 16129 buckets: forward 241 us with four, 142 with eight, dq 280 and 179).
  const bool alone = l.lds > 81920, one = backward && dh > 64;
  const int most = alone && !one ? 8 : 4;
  l.waves = NT < most ? NT : most;
  l.parts = (NT + l.waves - 1) / l.waves;
  l.held = alone || one ? 256 : 512;
  return l;
}

// the first workgroup that has images of a head, and how many have them
__host__ __device__ __forceinline__ int rel_first_group(int head, int B, int units) { return (int)((long long)head * B / units); }
__host__ __device__ __forceinline__ int rel_groups(int head, int B, int units) {
  return (int)(((long long)head * B + B - 1) / units) - rel_first_group(head, B, units) + 1;
}
// rows: [B * heads][3][Tp] floats; pairs (NULL: no gradient of the table): [slots][heads][NT][NT][1024]; units: (head, image) pairs
// that a workgroup of the walk for dk and dv has; *runs: whether it has left runs instead of pairs.  T: bf16_t or float
template <typename T> int rel_mfma_fwd(const RelArgs& a, const T* qkv, T* o, float* stats, hipStream_t st);
template <typename T>
int rel_mfma_bwd(const RelArgs& a, const T* qkv, const T* o, const T* d_o, const float* stats, T* dqkv, float* rows, float* pairs, int units, bool* runs, hipStream_t st);
