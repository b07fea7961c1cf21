// Beam search's selection (swarm_beam_select): of all continuations (beam, token) of a prompt the n_keep with the largest
//   score[beam] + logit[beam][token] - log sum_v exp(logit[beam][v]),
// ties to the lowest beam * vocab + token.
//
// First kernel, a CTA per chunk of a beam's row: the chunk lives in registers, read once; its maximum and sum of
// exponentials, and its n_keep largest logits.  (Inside a row the order of the sums is the order of the logits.)  Second
// kernel, a CTA per prompt: log-sum-exp of every beam and the n_keep best of all chunks' candidates, in 64 bits, since
// candidates of different beams may differ by less than fp32 holds.
//
// The n_keep largest of a chunk: the n_keep-th largest of the threads' own maxima is a lower bound of the n_keep-th largest
// element, and only the n_keep threads above it can hold candidates; those few are gathered and ranked by counting.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "swarm_internal.cuh"

namespace swarm {
namespace {

constexpr int kBeamThreads = 256;
constexpr int kMergeThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;

typedef unsigned long long key_t;
// Order-preserving image of a float; with the complement of the index behind it, larger keys come first and no two are equal.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ key_t make_key(float x, uint32_t index) { return ((key_t)ordered(x) << 32) | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_index(key_t k) { return ~(uint32_t)k; }
__device__ __forceinline__ float key_value(key_t k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ float exp_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
  return y;
}

template <class T> struct Element;
template <> struct Element<float> {
  static __device__ __forceinline__ float one(const void* p, long long i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};
template <> struct Element<__nv_bfloat16> {
  static __device__ __forceinline__ float one(const void* p, long long i) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); }
  static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
};
template <> struct Element<__half> {
  static __device__ __forceinline__ float one(const void* p, long long i) { return __half2float(static_cast<const __half*>(p)[i]); }
  static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(h[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
};

// Per thread kPer elements of a chunk of kBeamThreads * kPer; `chunks` of them cover a row.
template <class T, int kPer>
__global__ void __launch_bounds__(kBeamThreads)
beam_chunk_kernel(const BeamCall c, int chunks, key_t* __restrict__ keys, float2* __restrict__ sums) {
  constexpr int kVec = 16 / (int)sizeof(T), kVecs = kPer / kVec;
  __shared__ key_t s_max[kBeamThreads];
  __shared__ key_t s_cand[64 * kPer];
  __shared__ float s_red[2][kBeamThreads / 32];
  __shared__ key_t s_bound;
  __shared__ int s_count;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / chunks, chunk = blockIdx.x - row * chunks;
  const int V = c.vocab, keep = c.n_keep;
  // Rows may start anywhere in a 16-byte line.  The tokens a thread has do not depend on that (equal rows give equal sums, and so
  // ties between beams stay ties): a vector across two lines is put together from both.
  const char* first = static_cast<const char*>(c.logits) + (long long)row * c.row_stride * (int)sizeof(T);
  const char* end = static_cast<const char*>(c.logits) + ((long long)(c.batch * c.n_beams - 1) * c.row_stride + V) * (int)sizeof(T);
  const int shift = (int)(reinterpret_cast<uintptr_t>(first) & 15u);
  float x[kPer];
  uint4 lo[kVecs], hi[kVecs];
  const int at0 = chunk * kBeamThreads * kPer;
  auto whole = [&](int at) { return at < V && first + (long long)at * (int)sizeof(T) + (shift ? 32 - shift : 16) <= end; };
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int at = at0 + (i * kBeamThreads + tid) * kVec;
    if (whole(at)) {
      const char* p = first + (long long)at * (int)sizeof(T) - shift;
      lo[i] = shift ? __ldg(reinterpret_cast<const uint4*>(p)) : ldg_nc_v4(p);
      if (shift) hi[i] = __ldg(reinterpret_cast<const uint4*>(p + 16));
    }
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int at = at0 + (i * kBeamThreads + tid) * kVec;
    const bool full = whole(at);
    if (full) {
      uint4 v = lo[i];
      if (shift) {
        uint32_t w[8] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w, hi[i].x, hi[i].y, hi[i].z, hi[i].w};
        if (shift & 4) {
#pragma unroll
          for (int z = 0; z < 7; ++z) w[z] = w[z + 1];
        }
        if (shift & 8) {
#pragma unroll
          for (int z = 0; z < 5; ++z) w[z] = w[z + 2];
        }
        const int bits = (shift & 3) * 8;
        v = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                       __funnelshift_r(w[3], w[4], bits));
      }
      Element<T>::unpack(v, x + i * kVec);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      float& f = x[i * kVec + e];
      if (at + e >= V) f = -INFINITY;
      else if (!full) f = Element<T>::one(first, at + e);
      if (!(f == f)) f = -INFINITY;                           // NaN: never chosen
    }
  }
  // the thread's largest, the first of equal ones
  float mine = -INFINITY;
  int where = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    if (x[e] > mine) { mine = x[e]; where = e; }
  auto token = [&](int e) { return at0 + ((e / kVec) * kBeamThreads + tid) * kVec + e % kVec; };
  s_max[tid] = make_key(mine, (uint32_t)token(where));
  float top = mine;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (lane == 0) s_red[0][warp] = top;
  if (tid == 0) s_count = 0;
  __syncthreads();
  top = s_red[0][0];
#pragma unroll
  for (int w = 1; w < kBeamThreads / 32; ++w) top = fmaxf(top, s_red[0][w]);
  const float ref = top == -INFINITY ? 0.f : top;
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < kPer; ++e) sum[e & 1] += exp_fast(x[e] - ref);
  float all = sum[0] + sum[1];
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  if (lane == 0) s_red[1][warp] = all;
  // the n_keep-th largest of the threads' maxima
  int above = 0;
  const key_t my_key = s_max[tid];
#pragma unroll 8
  for (int i = 0; i < kBeamThreads; i += 2) {
    const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(s_max + i);
    above += (two.x > my_key) + (two.y > my_key);
  }
  if (above == keep - 1) s_bound = my_key;
  __syncthreads();
  const key_t bound = s_bound;
  if (my_key >= bound) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const key_t k = make_key(x[e], (uint32_t)token(e));
      if (k >= bound && x[e] != -INFINITY) s_cand[atomicAdd(&s_count, 1)] = k;
    }
  }
  __syncthreads();
  const int n = s_count;
  key_t* out = keys + (long long)blockIdx.x * keep;
  for (int i = tid; i < n; i += kBeamThreads) {
    const key_t k = s_cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s_cand[j] > k;
    if (rank < keep) out[rank] = k;
  }
  for (int i = n + tid; i < keep; i += kBeamThreads) out[i] = 0;   // no such candidate (below the key of every logit)
  if (tid == 0) {
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kBeamThreads / 32; ++w) l += s_red[1][w];
    sums[blockIdx.x] = make_float2(top, l);
  }
}

__device__ __forceinline__ key_t ordered(double x) {
  const key_t b = (key_t)__double_as_longlong(x);
  return b >> 63 ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double unordered_d(key_t o) {
  return __longlong_as_double((long long)(o >> 63 ? o & ~(1ull << 63) : ~o));
}
struct Cand {
  key_t value;          // order-preserving image of the sum in 64 bits; 0: none
  uint32_t index;       // beam * vocab + token
};
__device__ __forceinline__ bool before(const Cand& a, const Cand& b) { return a.value > b.value || (a.value == b.value && a.index < b.index); }

__global__ void __launch_bounds__(kMergeThreads)
beam_merge_kernel(const BeamCall c, int chunks, int group, const key_t* __restrict__ keys, const float2* __restrict__ sums) {
  extern __shared__ __align__(16) unsigned char smem[];
  double* s_base = reinterpret_cast<double*>(smem);           // [n_beams] score - log sum exp
  Cand* s_max = reinterpret_cast<Cand*>(s_base + c.n_beams);
  Cand* s_cand = s_max + kMergeThreads;
  __shared__ Cand s_bound;
  __shared__ int s_count;
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int keep = c.n_keep, V = c.vocab;
  for (int k = warp; k < c.n_beams; k += kMergeThreads / 32) {
    const float2* mine = sums + ((long long)b * c.n_beams + k) * chunks;
    float m = -INFINITY;
    for (int i = lane; i < chunks; i += 32) m = fmaxf(m, mine[i].x);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    double l = 0.0;
    for (int i = lane; i < chunks; i += 32)
      if (mine[i].x != -INFINITY) l += (double)mine[i].y * exp((double)mine[i].x - (double)m);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    if (lane == 0) s_base[k] = (double)m + log(l);            // (a beam without a finite logit offers no candidate)
  }
  if (tid == 0) s_count = 0;
  __syncthreads();
  const int per_beam = chunks * keep, total = c.n_beams * per_beam;
  const key_t* list = keys + (long long)b * total;
  auto get = [&](int i) {
    const key_t k = list[i];
    const int beam = i / per_beam;
    Cand r;
    const double s = (double)c.score[b * c.n_beams + beam] + ((double)key_value(k) - s_base[beam]);
    r.value = k == 0 || !(s > -INFINITY) ? 0 : ordered(s);
    r.index = (uint32_t)beam * (uint32_t)V + key_index(k);
    return r;
  };
  Cand mine{0, 0xFFFFFFFFu - (uint32_t)tid};                  // (indices of their own, so that no two are equal)
  for (int i = tid; i < total; i += kMergeThreads) {
    const Cand r = get(i);
    if (r.value != 0 && before(r, mine)) mine = r;
  }
  // maxima of groups of threads, where the candidates above their n_keep-th largest fit: ranking costs the square of their number
  for (int o = 1; o < group; o <<= 1) {
    const Cand other{__shfl_xor_sync(0xFFFFFFFFu, mine.value, o), __shfl_xor_sync(0xFFFFFFFFu, mine.index, o)};
    if (before(other, mine)) mine = other;
  }
  if (tid % group == 0) s_max[tid / group] = mine;
  __syncthreads();
  if (tid < kMergeThreads / group) {
    const Cand max = s_max[tid];
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < kMergeThreads / group; ++i) above += before(s_max[i], max);
    if (above == keep - 1) s_bound = max;
  }
  __syncthreads();
  const Cand bound = s_bound;
  if (mine.value != 0 && !before(bound, mine)) {
    for (int i = tid; i < total; i += kMergeThreads) {
      const Cand r = get(i);
      if (r.value != 0 && !before(bound, r)) s_cand[atomicAdd(&s_count, 1)] = r;
    }
  }
  __syncthreads();
  const int n = s_count;
  for (int i = tid; i < max(n, keep); i += kMergeThreads) {
    int rank = i;
    Cand r{0, 0};
    if (i < n) {
      r = s_cand[i];
      rank = 0;
      for (int j = 0; j < n; ++j) rank += before(s_cand[j], r);
    }
    if (rank < keep) {
      const long long at = (long long)b * keep + rank;
      const bool some = r.value != 0;
      c.new_score[at] = some ? (float)unordered_d(r.value) : -INFINITY;
      c.parent[at] = some ? b * c.n_beams + (int)(r.index / (uint32_t)V) : -1;
      c.token[at] = some ? (int)(r.index % (uint32_t)V) : -1;
    }
  }
}

// Elements per thread: a chunk is kBeamThreads times as many.  16 for few rows of small vocabularies (more CTAs, shorter
// ones), 32 otherwise.
int per_thread(long long rows, int vocab) { return rows * ((vocab + 8191) / 8192) < 296 ? 16 : 32; }
int chunks_of(int vocab, int per) { return (vocab + kBeamThreads * per - 1) / (kBeamThreads * per); }
constexpr int kMergeSmemMax = 200 * 1024;
// Shared memory of the second kernel: every thread of the n_keep groups above the bound may bring all of its candidates.
long long merge_smem(int beams, int chunks, int keep, int group) {
  const long long total = (long long)beams * chunks * keep, per = (total + kMergeThreads - 1) / kMergeThreads;
  return beams * 8LL + (kMergeThreads + std::min(keep * per * group, total)) * (long long)sizeof(Cand);
}
int merge_group(int beams, int chunks, int keep) { return merge_smem(beams, chunks, keep, 4) <= kMergeSmemMax ? 4 : 1; }

template <class T>
cudaError_t launch_chunks(const BeamCall& c, int per, int chunks, key_t* keys, float2* sums, cudaStream_t st) {
  const dim3 grid((unsigned)((long long)c.batch * c.n_beams * chunks));
  return per == 16 ? launch_pdl(beam_chunk_kernel<T, 16>, grid, dim3(kBeamThreads), 0, st, true, c, chunks, keys, sums)
                   : launch_pdl(beam_chunk_kernel<T, 32>, grid, dim3(kBeamThreads), 0, st, true, c, chunks, keys, sums);
}

constexpr int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

}  // namespace

bool beam_supported(int batch, int n_beams, int vocab, int n_keep) {
  const long long rows = (long long)batch * n_beams;
  const int per = per_thread(rows, vocab), chunks = chunks_of(vocab, per);
  return (long long)n_beams * vocab < (1LL << 31) && rows * chunks < (1LL << 31) && (long long)n_beams * chunks * n_keep < (1LL << 30) &&
         merge_smem(n_beams, chunks, n_keep, 1) <= kMergeSmemMax;
}

long long beam_select_workspace_bytes(int batch, int n_beams, int vocab, int n_keep) {
  const long long rows = (long long)batch * n_beams, chunks = chunks_of(vocab, per_thread(rows, vocab));
  return align256(rows * chunks * n_keep * 8) + align256(rows * chunks * 8);
}

cudaError_t launch_beam_select(const BeamCall& c, void* workspace, cudaStream_t st) {
  const long long rows = (long long)c.batch * c.n_beams;
  const int per = per_thread(rows, c.vocab), chunks = chunks_of(c.vocab, per);
  key_t* keys = static_cast<key_t*>(workspace);
  float2* sums = reinterpret_cast<float2*>(static_cast<unsigned char*>(workspace) + align256(rows * chunks * c.n_keep * 8));
  const int group = merge_group(c.n_beams, chunks, c.n_keep);
  const size_t smem = (size_t)merge_smem(c.n_beams, chunks, c.n_keep, group);
  cudaError_t e = cudaFuncSetAttribute(beam_merge_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMergeSmemMax);
  if (e != cudaSuccess) return e;
  e = c.dtype == SWARM_DTYPE_F32    ? launch_chunks<float>(c, per, chunks, keys, sums, st)
      : c.dtype == SWARM_DTYPE_BF16 ? launch_chunks<__nv_bfloat16>(c, per, chunks, keys, sums, st)
                                    : launch_chunks<__half>(c, per, chunks, keys, sums, st);
  if (e != cudaSuccess) return e;
  return launch_pdl(beam_merge_kernel, dim3((unsigned)c.batch), dim3(kMergeThreads), smem, st, true, c, chunks, group, keys, sums);
}

}  // namespace swarm
