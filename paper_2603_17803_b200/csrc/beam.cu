// Beam search's selection (swarm_beam_select): of all continuations (beam, token) of a prompt the n_keep with the largest
//   score[beam] + logit[beam][token] - log sum_v exp(logit[beam][v]),
// ties to the lowest beam * vocab + token.
//
// First kernel, a CTA per stretch of a beam's row, which it reads once, a chunk in registers at a time: a running maximum and sum
// of exponentials per thread, joined at the end, and the n_keep largest logits so far.  (Inside a row the order of the sums is the
// order of the logits.)  Second kernel, a CTA per prompt: log-sum-exp of every beam and the n_keep best of all stretches'
// candidates, in 64 bits, since candidates of different beams may differ by less than fp32 holds.
//
// The n_keep largest: once n_keep logits are held, only those above the least of them matter, and soon hardly any thread has
// one.  In a chunk where many threads do (the first one), the n_keep-th largest of the maxima of groups of threads is a lower
// bound of what can be chosen, and only the n_keep groups above it can hold candidates; those few are gathered and ranked
// by counting.
//
// Bound by HBM while the rows are read: 32 x 16 rows of 131072 fp32 (268 MB) take 62 us, of which 46 at 5.8 TB/s, 9 while only the
// SMs with a fourth row still read (512 rows on 148 SMs; shorter stretches balance them but pay a first chunk each: 72 us with
// two per row), 7 the second kernel, a chain of barriers.  A prompt of 4 x 32000 takes 9: two launches, and those chains.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "swarm_internal.cuh"

namespace swarm {
namespace {

constexpr int kBeamThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

typedef unsigned long long key_t;
// Order-preserving image of a float; with the complement of the index behind it, larger keys come first and no two are equal.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ key_t make_key(float x, uint32_t index) { return ((key_t)ordered(x + 0.f) << 32) | (uint32_t)~index; }   // (-0 as 0)
__device__ __forceinline__ uint32_t key_index(key_t k) { return ~(uint32_t)k; }
__device__ __forceinline__ float key_value(key_t k) { return unordered((uint32_t)(k >> 32)); }

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

constexpr float kLog2eLow = 1.9259629911e-8f;               // log2 e - kLog2e: sums of different beams are compared far below 2^-24
__device__ __forceinline__ float exp2_fast(float y) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {   // NaN is passed over
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Two floats in a register pair: one instruction for both.
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t pair_of(float lo, float hi) {
  pair_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(pair_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
  pair_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
  pair_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
  pair_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp_fast(float t) { return exp2_fast(fmaf(t, kLog2eLow, t * kLog2e)); }   // e^t for t <= 0
// sum of e^(x - ref) over the logits, none far above ref (the difference first: logits of the type's lowest value mask, too)
template <int n>
__device__ __forceinline__ float sum_exp(const float (&x)[n], float ref) {
  const pair_t l = pair_of(kLog2e, kLog2e), low = pair_of(kLog2eLow, kLog2eLow), r = pair_of(-ref, -ref);
  pair_t part[2] = {0ull, 0ull};
#pragma unroll
  for (int e = 0; e < n; e += 2) {
    const pair_t t = add2(pair_of(x[e], x[e + 1]), r);
    float y0, y1;
    unpair(fma2(t, low, mul2(t, l)), y0, y1);
    part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], pair_of(exp2_fast(y0), exp2_fast(y1)));
  }
  float a, b;
  unpair(add2(part[0], part[1]), a, b);
  return a + b;
}

// out(i, rank) for every i < n, rank = how many j < n have greater(j, i).  All threads take part; entered behind a barrier.  Where
// there are more threads than entries, several share an entry's comparisons.
template <int kThreads, class Greater, class Out>
__device__ __forceinline__ void rank_all(int n, int* s_rank, Greater&& greater, Out&& out) {
  const int tid = threadIdx.x;
  if (2 * n > kThreads) {
    for (int i = tid; i < n; i += kThreads) {
      int r = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) r += greater(j, i);
      out(i, r);
    }
    return;
  }
  const int width = n <= 32 ? 32 : 1 << (32 - __clz(n - 1)), parts = kThreads / width, i = tid & (width - 1);
  if (tid < n) s_rank[tid] = 0;
  __syncthreads();
  if (i < n) {
    int r = 0;
#pragma unroll 4
    for (int j = tid / width; j < n; j += parts) r += greater(j, i);
    if (r != 0) atomicAdd(s_rank + i, r);
  }
  __syncthreads();
  if (tid < n) out(tid, s_rank[tid]);
}

// (three stages leave room for three CTAs per SM in place of four: 32 x 16 x 131072 fp32 73 -> 93 us)
constexpr int kStages = 2, kLineBytes = 33 * 16;
__device__ __forceinline__ void copy_line(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// A chunk is kPer tokens for each of kBeamThreads threads; a CTA takes `span` chunks of a row one after the other.
template <class T, int kPer>
__global__ void __launch_bounds__(kBeamThreads, kPer == 32 ? 3 : 4)
beam_chunk_kernel(const BeamCall c, int stretches, int span, key_t* __restrict__ keys, float2* __restrict__ sums) {
  constexpr int kVec = 16 / (int)sizeof(T), kVecs = kPer / kVec, kChunk = kBeamThreads * kPer;
  constexpr int kMany = 64;                                   // threads with a candidate that are gathered as they are
  constexpr int kRoom = kMaxBeamKeep + 128 * kPer;
  extern __shared__ __align__(16) unsigned char s_raw[];      // [kStages][warp][kVecs][33] 16-byte lines, then the candidates
  key_t* s_cand = reinterpret_cast<key_t*>(s_raw + kStages * kBeamThreads / 32 * kVecs * kLineBytes);
  __shared__ key_t s_max[128];
  __shared__ key_t s_top[kMaxBeamKeep];
  __shared__ float2 s_red[kBeamThreads / 32];
  __shared__ key_t s_bound;
  __shared__ int s_count;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / stretches, stretch = blockIdx.x - row * stretches;
  const int V = c.vocab, keep = c.n_keep;
  const int gather = max(64, 2 * keep);                       // candidates that are ranked together (by comparing all with all)
  // Rows may start anywhere in a 16-byte line.  The tokens a thread has do not depend on that (equal rows give equal sums, and so
  // ties between beams stay ties): a vector across two lines is put together from both.
  const char* first = static_cast<const char*>(c.logits) + (long long)row * c.row_stride * (int)sizeof(T);
  const char* end = static_cast<const char*>(c.logits) + ((long long)(c.batch * c.n_beams - 1) * c.row_stride + V) * (int)sizeof(T);
  const int shift = (int)(reinterpret_cast<uintptr_t>(first) & 15u);
  const int begin = stretch * span * kChunk, stop = min(V, begin + span * kChunk);
  // chunks of this stretch whose vectors (with the line behind, where they are put together) lie inside the row and the tensor
  const int n_whole = max(0, (int)min((long long)(stop - begin), (long long)(end - 32 - first) / (int)sizeof(T) - begin) / kChunk);
  const char* const start = first + ((long long)begin + tid * kVec) * (int)sizeof(T) - shift;
  const char* next = start;
  // Chunks travel through shared memory by 16-byte asynchronous copies, kStages ahead; a warp reads only what its own lanes have
  // copied (and, of a row that starts inside a line, the line behind).
  auto line = [&](int stage, int i) { return s_raw + ((stage * (kBeamThreads / 32) + warp) * kVecs + i) * kLineBytes + lane * 16; };
  auto fetch = [&](int stage, bool some) {
    if (some) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) copy_line(line(stage, i), next + i * kBeamThreads * 16);
      if (shift != 0 && lane == 31) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) copy_line(line(stage, i) + 16, next + i * kBeamThreads * 16 + 16);
      }
      next += kChunk * (int)sizeof(T);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto chunk_of = [&](int stage, uint4 (&raw)[kVecs]) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) raw[i] = *reinterpret_cast<const uint4*>(line(stage, i));
    if (shift != 0) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const uint4 lo = raw[i], hi = *reinterpret_cast<const uint4*>(line(stage, i) + 16);
        uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        if (shift & 4) {
#pragma unroll
          for (int z = 0; z < 7; ++z) w[z] = w[z + 1];
        }
        if (shift & 8) {
#pragma unroll
          for (int z = 0; z < 5; ++z) w[z] = w[z + 2];
        }
        const int bits = (shift & 3) * 8;
        raw[i] = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                            __funnelshift_r(w[3], w[4], bits));
      }
    }
    __syncwarp();                                             // all lanes have read: the stage may be written again
  };
  if (tid == 0) s_count = 0;
  // Sum of e^(x - top) over this thread's logits so far.  top is raised only by logits that pass it by more than kSlack: the
  // exponentials stay below e^kSlack.
  constexpr float kSlack = 8.f;
  float top = -INFINITY, sum = 0.f;
  float floor_ = -INFINITY;                                   // the least of the n_keep largest at the last ranking
  // Ranks the gathered candidates and keeps the n_keep largest.  Entered behind a barrier, left in front of one.
  auto rank = [&] {
    const int n = s_count;
    if (n >= keep) {
      for (int i = tid; i < n; i += kBeamThreads) {
        const key_t k = s_cand[i];
        int r = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) r += s_cand[j] > k;
        if (r < keep) s_top[r] = k;
      }
      __syncthreads();
      if (tid < keep) s_cand[tid] = s_top[tid];
      if (tid == 0) s_count = keep;
      floor_ = key_value(s_top[keep - 1]);
    }
  };
  // Behind the first chunk candidates are rare, and no barrier is spent on them: a thread appends what lies above the floor it knows,
  // and the gathered ones are ranked after 1, 2, 4, 8, 16, 24 ... chunks, each time about as many again as are kept.
  // Where more come than there is room for (logits that rise along the row), the stretch is done again with a look at every chunk.
  bool over = false;
  for (bool careful = false;; careful = true) {
#pragma unroll
    for (int i = 0; i < kStages; ++i) fetch(i, i < n_whole);
    int stage = 0;
    bool more = false;                                          // this thread has appended since the last ranking
    for (int at0 = begin, chunk = 0; at0 < stop; at0 += kChunk, ++chunk) {
      float x[kPer];
      if (chunk < n_whole) {
        uint4 raw[kVecs];
        chunk_of(stage, raw);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) Element<T>::unpack(raw[i], x + i * kVec);
        fetch(stage, chunk + kStages < n_whole);
        if (++stage == kStages) stage = 0;
      } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int at = at0 + (i * kBeamThreads + tid) * kVec;
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[i * kVec + e] = at + e < V ? Element<T>::one(first, at + e) : -INFINITY;
        }
      }
      float best4[4];                                           // of quarters of the thread's logits
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        best4[z] = fmaxf(x[z * kPer / 4], x[z * kPer / 4 + 1]);
#pragma unroll
        for (int e = 2; e < kPer / 4; e += 2) best4[z] = max3(best4[z], x[z * kPer / 4 + e], x[z * kPer / 4 + e + 1]);
      }
      float mine = fmaxf(max3(best4[0], best4[1], best4[2]), best4[3]);
      if (mine > top + kSlack) {                                // (-inf: any finite value)
        sum *= exp_fast(top - mine);                            // (0 * 2^-inf the first time)
        top = mine;
      }
      const float ref = top == -INFINITY ? 0.f : top;
      const float part = sum_exp(x, ref);
      if (part == part) {
        sum += part;
      } else {                                                  // NaN among them: never chosen, counted as nothing
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = fmaxf(x[e], -INFINITY);
        mine = fmaxf(mine, -INFINITY);                          // (nothing but NaN: its key must not stand above a logit's)
        sum += sum_exp(x, ref);
      }

      // Candidates: logits above the floor.
      auto token = [&](int e) { return (uint32_t)(at0 + ((e / kVec) * kBeamThreads + tid) * kVec + e % kVec); };
      if (!careful && chunk > 0) {
        if (__any_sync(0xFFFFFFFFu, mine > floor_)) {
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            if (!__any_sync(0xFFFFFFFFu, best4[z] > floor_)) continue;
#pragma unroll
            for (int e = z * kPer / 4; e < (z + 1) * kPer / 4; ++e) {
              if (x[e] > floor_) {
                const int at = atomicAdd(&s_count, 1);
                if (at < kRoom) s_cand[at] = make_key(x[e], token(e));
                else over = true;
                more = true;
              }
            }
          }
        }
        if ((chunk & (chunk + 1)) == 0 || (chunk & 7) == 7) {
          if (__syncthreads_or(more)) {
            if (__syncthreads_or(over)) break;
            rank();
            __syncthreads();
            more = false;
          }
        }
        continue;
      }
      const int hits = __syncthreads_count(mine > floor_);
      if (hits == 0) continue;
      const int held = s_count;
      __syncthreads();
      if (held >= (hits > kMany ? keep + 1 : gather)) {         // (many hits: the bound below may bring as many as fit beside n_keep)
        rank();
        __syncthreads();
      }
      key_t bound = 0;
      float bound_value = -INFINITY;
      if (hits > kMany) {
        const int group = keep > 32 ? 2 : 4, groups = kBeamThreads / group;
        int where = 0;
#pragma unroll
        for (int e = kPer - 1; e >= 0; --e)
          if (x[e] == mine) where = e;                          // the first of equal ones
        key_t best = make_key(mine, token(where));
        for (int o = 1; o < group; o <<= 1) {
          const key_t other = __shfl_xor_sync(0xFFFFFFFFu, best, o);
          if (other > best) best = other;
        }
        if (tid % group == 0) s_max[tid / group] = best;
        __syncthreads();
        if (tid < groups) {
          const key_t my_key = s_max[tid];
          int above = 0;
#pragma unroll 8
          for (int i = 0; i < groups; i += 2) {
            const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(s_max + i);
            above += (two.x > my_key) + (two.y > my_key);
          }
          if (above == keep - 1) s_bound = my_key;
        }
        __syncthreads();
        bound = s_bound;
        bound_value = key_value(bound);
      }
      if (__any_sync(0xFFFFFFFFu, mine > floor_ && mine >= bound_value)) {
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          if (!__any_sync(0xFFFFFFFFu, best4[z] > floor_ && best4[z] >= bound_value)) continue;
#pragma unroll
          for (int e = z * kPer / 4; e < (z + 1) * kPer / 4; ++e) {
            if (x[e] > floor_ && x[e] >= bound_value) {
              const key_t k = make_key(x[e], token(e));
              if (k >= bound) s_cand[atomicAdd(&s_count, 1)] = k;
            }
          }
        }
      }
      if (!careful) {                                           // (the first chunk: a floor for the others)
        __syncthreads();
        rank();
        __syncthreads();
      }
    }
    if (!__syncthreads_or(over)) break;
    // once more, from the start (copies under way would still write to the ring)
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    over = false;
    if (tid == 0) s_count = 0;
    top = floor_ = -INFINITY;
    sum = 0.f;
    next = start;
  }
  if (s_count > keep) rank();
  __syncthreads();
  // the threads' sums
  float m = top;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  float l = top == -INFINITY ? 0.f : sum * exp_fast(top - m);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
  if (lane == 0) s_red[warp] = make_float2(m, l);
  __syncthreads();
  key_t* out = keys + (long long)blockIdx.x * keep;
  const int n = s_count;                                      // at most n_keep, in no order while fewer
  if (tid < keep) {
    if (tid < n) {
      const key_t k = s_cand[tid];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += s_cand[j] > k;
      out[rank] = k;
    } else {
      out[tid] = 0;                                           // no such candidate (below the key of every logit)
    }
  }
  if (tid == 0) {
    float M = -INFINITY, all = 0.f;
#pragma unroll
    for (int w = 0; w < kBeamThreads / 32; ++w) M = fmaxf(M, s_red[w].x);
#pragma unroll
    for (int w = 0; w < kBeamThreads / 32; ++w)
      if (s_red[w].x != -INFINITY) all += s_red[w].y * exp_fast(s_red[w].x - M);
    sums[blockIdx.x] = make_float2(M, all);
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

constexpr int kHold = 4;                                    // candidates that a thread keeps in registers

// The candidates' sums are compared as ordered images with the index behind; what a thread cannot hold it reads again.
template <int kThreads, int kGroups>
__global__ void __launch_bounds__(kThreads)
beam_merge_kernel(const BeamCall c, int chunks, const key_t* __restrict__ keys, const float2* __restrict__ sums) {
  extern __shared__ __align__(16) unsigned char smem[];
  double* s_base = reinterpret_cast<double*>(smem);           // [n_beams] log sum exp, then [n_beams] scores
  double* s_score = s_base + c.n_beams;
  Cand* s_max = reinterpret_cast<Cand*>(s_score + c.n_beams);
  Cand* s_cand = s_max + kGroups;
  __shared__ Cand s_bound;
  __shared__ int s_count, s_rank[kThreads];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int keep = c.n_keep, V = c.vocab;
  const int per_beam = chunks * keep, total = c.n_beams * per_beam;
  const key_t* list = keys + (long long)b * total;
  pdl_wait();
  pdl_launch_dependents();
  // Place p of the candidates belongs to group p % kGroups of neighbouring threads; the candidates of a list stand in as many groups,
  // and lists turned against one another, since few lists may hold most of what is chosen: then the n_keep-th largest of the
  // groups' maxima is a bound that few others pass (32 x 16 lists of 32: this kernel 16 us with the places in order, 7 so).
  constexpr int kGroup = kThreads / kGroups;
  auto place = [&](int i) { return i * kThreads + tid % kGroup * kGroups + tid / kGroup; };
  auto entry = [&](int p) {                                   // list * n_keep + rank of a place
    const int l = p / keep;
    return l * keep + (p - l * keep + l % keep * 11) % keep;
  };
  key_t held[kHold];
#pragma unroll
  for (int i = 0; i < kHold; ++i) held[i] = place(i) < total ? list[entry(place(i))] : 0;
  for (int k = tid; k < c.n_beams; k += kThreads) s_score[k] = (double)c.score[b * c.n_beams + k];
  const float2* const all_sums = sums + (long long)b * c.n_beams * chunks;
  auto sum_of = [&](int k) { return k < c.n_beams && lane < chunks ? all_sums[(long long)k * chunks + lane] : make_float2(-INFINITY, 0.f); };
  float2 ahead = sum_of(warp);
  for (int k = warp; k < c.n_beams; k += kThreads / 32) {
    const float2* mine = all_sums + (long long)k * chunks;
    const float2 first = ahead;
    ahead = sum_of(k + kThreads / 32);
    float m = first.x;
    for (int i = lane + 32; i < chunks; i += 32) m = fmaxf(m, mine[i].x);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    double l = first.x == -INFINITY ? 0.0 : (double)(first.y * exp_fast(first.x - m));
    for (int i = lane + 32; i < chunks; i += 32)
      if (mine[i].x != -INFINITY) l += (double)(mine[i].y * exp_fast(mine[i].x - m));
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    if (lane == 0) s_base[k] = (double)m + log(l);            // (a beam without a finite logit offers no candidate)
  }
  if (tid == 0) s_count = 0;
  __syncthreads();
  auto cand = [&](int i, key_t k) {
    const int beam = i / per_beam;
    Cand r;
    const double s = s_score[beam] + ((double)key_value(k) - s_base[beam]);
    r.value = k == 0 || !(s > -INFINITY) ? 0 : ordered(s + 0.0);
    r.index = (uint32_t)beam * (uint32_t)V + key_index(k);
    return r;
  };
  Cand mine[kHold], best{0, 0xFFFFFFFFu - (uint32_t)tid};     // (indices of their own, so that no two are equal)
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    mine[i].value = 0;
    if (place(i) < total) mine[i] = cand(place(i), held[i]);
    if (mine[i].value != 0 && before(mine[i], best)) best = mine[i];
  }
  for (int p = place(kHold); p < total; p += kThreads) {
    const Cand r = cand(p, list[entry(p)]);
    if (r.value != 0 && before(r, best)) best = r;
  }
  // maxima of groups of threads, where the candidates above their n_keep-th largest fit: ranking costs the square of their number
  for (int o = 1; o < kGroup; o <<= 1) {
    const Cand other{__shfl_xor_sync(0xFFFFFFFFu, best.value, o), __shfl_xor_sync(0xFFFFFFFFu, best.index, o)};
    if (before(other, best)) best = other;
  }
  if (tid % kGroup == 0) s_max[tid / kGroup] = best;
  __syncthreads();
  rank_all<kThreads>(kGroups, s_rank, [&](int j, int i) { return before(s_max[j], s_max[i]); }, [&](int i, int r) { if (r == keep - 1) s_bound = s_max[i]; });
  __syncthreads();
  const Cand bound = s_bound;
#pragma unroll
  for (int i = 0; i < kHold; ++i)
    if (mine[i].value != 0 && !before(bound, mine[i])) s_cand[atomicAdd(&s_count, 1)] = mine[i];
  for (int p = place(kHold); p < total; p += kThreads) {
    const Cand r = cand(p, list[entry(p)]);
    if (r.value != 0 && !before(bound, r)) s_cand[atomicAdd(&s_count, 1)] = r;
  }
  __syncthreads();
  const int n = s_count;
  auto write = [&](const Cand& r, int rank) {
    const long long at = (long long)b * keep + rank;
    const bool some = r.value != 0;
    c.new_score[at] = some ? (float)unordered_d(r.value) : -INFINITY;
    c.parent[at] = some ? b * c.n_beams + (int)(r.index / (uint32_t)V) : -1;
    c.token[at] = some ? (int)(r.index % (uint32_t)V) : -1;
  };
  if (tid >= n && tid < keep) write(Cand{0, 0}, tid);
  rank_all<kThreads>(n, s_rank, [&](int j, int i) { return before(s_cand[j], s_cand[i]); }, [&](int i, int r) { if (r < keep) write(s_cand[i], r); });
}

// How a row is cut.  Elements per thread: 64 bytes of them, of 16-bit types 32 bytes where that leaves SMs without a chunk.
// Stretches: as many as the device holds CTAs at a time, since candidates grow rare with the length of a stretch and each pays for a
// first chunk (fp32, 32 x 16 x 131072: 62 us with whole rows, 72 with halves, 83 with quarters; bf16, 5 x 16 x 119450: 25 us with 5
// stretches in one wave, 40 with 8 in two).
struct Cut {
  int per, span, stretches;
};
Cut cut_of(long long rows, int vocab, int dtype) {
  Cut c;
  auto chunks = [&](int per) { return (vocab + kBeamThreads * per - 1) / (kBeamThreads * per); };
  c.per = dtype == SWARM_DTYPE_F32 || rows * chunks(32) < kSms ? 16 : 32;
  const long long at_once = kSms * (c.per == 32 ? 3 : 4);
  const int most = (int)std::max<long long>(1, std::min<long long>(chunks(c.per), at_once / rows));
  c.span = (chunks(c.per) + most - 1) / most;
  c.stretches = (chunks(c.per) + c.span - 1) / c.span;
  return c;
}
// The second kernel: 64 groups of candidates where all of the n_keep best groups' candidates fit in shared memory, else 256; four
// candidates per thread of 256 threads, or, of more, of 1024 (bf16, 5 x 16 x 119450, 2560 candidates: 7 us of this kernel, 11 with 256).
constexpr int kMergeSmemMax = 200 * 1024;
long long candidates(int beams, int stretches, int keep) { return (long long)beams * stretches * keep; }
long long merge_smem(int beams, int stretches, int keep, int groups) {
  const long long total = candidates(beams, stretches, keep);
  return beams * 16LL + (groups + std::min(keep * ((total + groups - 1) / groups), total)) * (long long)sizeof(Cand);
}
int merge_groups(int beams, int stretches, int keep) { return merge_smem(beams, stretches, keep, 64) <= kMergeSmemMax ? 64 : 256; }

template <class T, int kPer>
constexpr int chunk_smem() {
  return kStages * kBeamThreads / 32 * (kPer * (int)sizeof(T) / 16) * kLineBytes + (kMaxBeamKeep + 128 * kPer) * (int)sizeof(key_t);
}
template <class T, int kPer>
cudaError_t launch_chunks_of(const BeamCall& c, const Cut& cut, key_t* keys, float2* sums, cudaStream_t st) {
  const dim3 grid((unsigned)((long long)c.batch * c.n_beams * cut.stretches));
  return launch_pdl(beam_chunk_kernel<T, kPer>, grid, dim3(kBeamThreads), (size_t)chunk_smem<T, kPer>(), st, true, c, cut.stretches,
                    cut.span, keys, sums);
}
// The kernels' room in shared memory, once per device (each of these calls takes the host a microsecond or two).
template <class T, int kPer>
cudaError_t configure_chunks() {
  return cudaFuncSetAttribute(beam_chunk_kernel<T, kPer>, cudaFuncAttributeMaxDynamicSharedMemorySize, chunk_smem<T, kPer>());
}
cudaError_t configure_beam() {
  static std::atomic<unsigned long long> configured{0};       // a bit per device
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = device < 64 ? 1ull << device : 0ull;
  if (configured.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(beam_merge_kernel<256, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMergeSmemMax);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(beam_merge_kernel<1024, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMergeSmemMax);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(beam_merge_kernel<1024, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMergeSmemMax);
  if (e == cudaSuccess) e = configure_chunks<float, 16>();
  if (e == cudaSuccess) e = configure_chunks<__nv_bfloat16, 16>();
  if (e == cudaSuccess) e = configure_chunks<__nv_bfloat16, 32>();
  if (e == cudaSuccess) e = configure_chunks<__half, 16>();
  if (e == cudaSuccess) e = configure_chunks<__half, 32>();
  if (e == cudaSuccess) configured.fetch_or(bit, std::memory_order_release);
  return e;
}
template <class T>
cudaError_t launch_chunks(const BeamCall& c, const Cut& cut, key_t* keys, float2* sums, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (cut.per == 32) return launch_chunks_of<T, 32>(c, cut, keys, sums, st);
  return launch_chunks_of<T, 16>(c, cut, keys, sums, st);
}

constexpr int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

// (Whatever the type of the logits: 16 elements per thread give the most stretches.)
int most_stretches(long long rows, int vocab) {
  return std::max(cut_of(rows, vocab, SWARM_DTYPE_F32).stretches, cut_of(rows, vocab, SWARM_DTYPE_BF16).stretches);
}
}  // namespace

bool beam_supported(int batch, int n_beams, int vocab, int n_keep) {
  if (vocab >= (1 << 30)) return false;                       // (tokens are counted in 32 bits up to the end of a row's last stretch)
  const long long rows = (long long)batch * n_beams;
  const int parts = most_stretches(rows, vocab);
  return (long long)n_beams * vocab < (1LL << 31) && rows * parts < (1LL << 31) && (long long)n_beams * parts * n_keep < (1LL << 30) &&
         merge_smem(n_beams, parts, n_keep, 256) <= kMergeSmemMax;
}

long long beam_select_workspace_bytes(int batch, int n_beams, int vocab, int n_keep) {
  const long long rows = (long long)batch * n_beams, parts = most_stretches(rows, vocab);
  return align256(rows * parts * n_keep * 8) + align256(rows * parts * 8);
}

cudaError_t launch_beam_select(const BeamCall& c, void* workspace, cudaStream_t st) {
  const long long rows = (long long)c.batch * c.n_beams;
  const Cut cut = cut_of(rows, c.vocab, c.dtype);
  key_t* keys = static_cast<key_t*>(workspace);
  float2* sums = reinterpret_cast<float2*>(static_cast<unsigned char*>(workspace) + align256(rows * cut.stretches * c.n_keep * 8));
  const int groups = merge_groups(c.n_beams, cut.stretches, c.n_keep);
  const size_t smem = (size_t)merge_smem(c.n_beams, cut.stretches, c.n_keep, groups);
  cudaError_t e = configure_beam();
  if (e != cudaSuccess) return e;
  e = c.dtype == SWARM_DTYPE_F32    ? launch_chunks<float>(c, cut, keys, sums, st)
      : c.dtype == SWARM_DTYPE_BF16 ? launch_chunks<__nv_bfloat16>(c, cut, keys, sums, st)
                                    : launch_chunks<__half>(c, cut, keys, sums, st);
  if (e != cudaSuccess) return e;
  const bool many = groups > 64 || candidates(c.n_beams, cut.stretches, c.n_keep) > kHold * 256;
  auto* merge = !many ? beam_merge_kernel<256, 64> : groups == 64 ? beam_merge_kernel<1024, 64> : beam_merge_kernel<1024, 256>;
  return launch_pdl(merge, dim3((unsigned)c.batch), dim3(many ? 1024 : 256), smem, st, true, c, cut.stretches, keys, sums);
}

}  // namespace swarm
