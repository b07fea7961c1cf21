// Commit of new tokens to the cache (swarm_append_tokens): the keys and values of a prompt, of a decoded token or of the
// accepted path of a drafted tree go behind the tokens a request has, and the min/max summaries of the pages they reach
// are brought up to date.
#include "swarm_internal.cuh"

namespace swarm {
namespace {

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A warp per (page that may receive tokens, KV head): lanes 0-15 take the even tokens, lanes 16-31 the odd ones, 16 bytes of
// K and of V each; the page's minima and maxima are taken on the way, so that the new rows are read once and written once.
// Bound by HBM for prompts (444 MB in 74 us, 6.0 TB/s: eight 16-byte loads a lane are in flight, and a page's rows are one stretch of
// 4 KB), by the launch for a few tokens a request (64 requests, 1 to 8 of 16 tokens: 3.6 us in a graph, 4.8 from the host).
constexpr int kThreads = 256, kBatch = 4;
__global__ void __launch_bounds__(kThreads)
append_kernel(const Geometry geo, const AppendCall c, int ctas, unsigned* __restrict__ tickets, uint32_t* __restrict__ status) {
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x / ctas, cta = blockIdx.x - b * ctas, lane = threadIdx.x & 31;
  const int S = geo.S, Hkv = geo.Hkv;
  const int len = c.ctx_len[b], n = c.n_new[b];
  const long long base = c.page_base[b], owned = c.page_base[b + 1] - base;
  // (a range that is not inside the pool would be written to all the same)
  const bool bad = len < 0 || n < 0 || n > c.n_places || (long long)len + n > min(owned, (long long)geo.Pmax) * S || base < 0 ||
                   base + owned > geo.n_pool_pages;
  const bool in_place = c.ctx_len_out == c.ctx_len;
  if (in_place) __syncthreads();                             // every thread has its length before this CTA counts as having read it
  if (threadIdx.x == 0) {
    // the new length may take the old one's place: then the request's last CTA to have read it writes it
    bool mine = cta == 0;
    if (in_place) {
      mine = atom_acq_rel_add(tickets + b, 1u) == (unsigned)ctas - 1u;
      if (mine) tickets[b] = 0u;
    }
    if (mine) c.ctx_len_out[b] = bad ? len : len + n;
    if (bad && cta == 0) atomicOr(status, SWARM_DEV_BAD_LENGTH);
  }
  if (bad || n == 0) return;
  const int unit = cta * (kThreads / 32) + (threadIdx.x >> 5);
  const int p = len / S + unit / Hkv, kv = unit % Hkv;
  const int lo = max(len, p * S), hi = min(len + n, (p + 1) * S);
  if (lo >= hi) return;
  const int half = lane >> 4, col = (lane & 15) * 8;
  const long long blk = (long long)S * kHeadDim;
  uint16_t* to = c.kv_pool + ((base + p) * Hkv + kv) * 2 * blk + col;
  uint32_t least[4], most[4];                                // pairs of bf16
#pragma unroll
  for (int e = 0; e < 4; ++e) { least[e] = 0x7F807F80u; most[e] = 0xFF80FF80u; }   // +inf, -inf
  for (int t0 = lo; t0 < hi; t0 += 2 * kBatch) {
    uint4 k[kBatch], v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + 2 * i + half;
      k[i] = v[i] = make_uint4(0, 0, 0, 0);
      if (t < hi) {
        int from = t - len;
        if (c.path != nullptr) from = c.path[(long long)b * c.n_places + from];
        if (from >= 0 && from < c.T) {
          const long long row = (((long long)b * c.T + from) * Hkv + kv) * kHeadDim + col;
          k[i] = ldg_nc_v4(c.k + row);
          v[i] = ldg_nc_v4(c.v + row);
        } else if (col == 0) {
          atomicOr(status, SWARM_DEV_BAD_TOKEN);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + 2 * i + half;
      if (t < hi) {
        uint16_t* row = to + (long long)(t - p * S) * kHeadDim;
        *reinterpret_cast<uint4*>(row) = k[i];
        *reinterpret_cast<uint4*>(row + blk) = v[i];
        const uint32_t words[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) { least[e] = min2(least[e], words[e]); most[e] = max2(most[e], words[e]); }
      }
    }
  }
  if (c.ksum == nullptr) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    least[e] = min2(least[e], __shfl_xor_sync(0xFFFFFFFFu, least[e], 16));
    most[e] = max2(most[e], __shfl_xor_sync(0xFFFFFFFFu, most[e], 16));
  }
  uint4* sum = reinterpret_cast<uint4*>(c.ksum + (((base + p) * Hkv + kv) * 2 + half) * (long long)kHeadDim + col);
  uint32_t r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = half ? most[e] : least[e];
  if (lo > p * S) {                                          // the page held tokens: their summary takes part
    const uint4 old = *sum;
    const uint32_t words[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = half ? max2(r[e], words[e]) : min2(r[e], words[e]);
  }
  *sum = make_uint4(r[0], r[1], r[2], r[3]);
}

long long ctas_per_request(const Geometry& geo, int n_places) {
  const long long pages = ((long long)n_places + 2 * geo.S - 2) / geo.S;   // touched, wherever in its page the request ends
  return (pages * geo.Hkv + kThreads / 32 - 1) / (kThreads / 32);
}

}  // namespace

bool append_supported(const Geometry& geo, int n_places) { return ctas_per_request(geo, n_places) * geo.B < (1LL << 31); }

cudaError_t launch_append(const Geometry& geo, const AppendCall& c, unsigned* tickets, uint32_t* status, cudaStream_t st) {
  const int ctas = (int)ctas_per_request(geo, c.n_places);
  return launch_pdl(append_kernel, dim3((unsigned)(ctas * geo.B)), dim3(kThreads), 0, st, true, geo, c, ctas, tickets, status);
}

}  // namespace swarm
