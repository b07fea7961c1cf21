// Re-layout of the cache (swarm_plan_pages, swarm_move_pages).  Every request owns one contiguous range of the pool, so
// freeing, thinning out, forking, reordering and growing requests are all one thing: a new list of ranges and pages to move.
//
// The plan: new request j continues old request parent[j] with the pages that `keep` holds, in order, and has reserve[j]
// spare pages behind them.  One kernel, a CTA per request: each sums the counts of all requests for itself (a byte a page),
// which is cheaper than a second launch (24 requests of 1024 pages: 5 us, bound by three trips to memory one after the other).
//
// The move: pairs (src, dst) of pages.  Between two pools they are independent.  Inside one pool a page may be read by one
// pair and overwritten by another; the pairs are taken in an order in which every reader of a page comes before its writer
// (downward moves first to last, then upward moves last to first: right for every plan that keeps the requests' order), and a
// CTA that has READ its page waits before it writes until the readers of its destination have read theirs.  Those were taken
// earlier and do not wait in front of their reads, so the waits end.  Pairs that break the order are found beforehand.
#include "swarm_internal.cuh"

#include <algorithm>

namespace swarm {
namespace {

constexpr int kPlanThreads = 512;

__device__ __forceinline__ int warp_sum(int v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// `keep` of 16 pages from page x on, as bits (x need not be aligned; pages from `end` on count as not kept)
__device__ __forceinline__ unsigned keep_bits(const uint8_t* keep, long long x, long long end) {
  unsigned bits = 0u;
  if (keep == nullptr) {
    bits = 0xFFFFu;
  } else if ((reinterpret_cast<uintptr_t>(keep + x) & 15u) == 0 && x + 16 <= end) {
    const uint4 v = *reinterpret_cast<const uint4*>(keep + x);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) bits |= ((w[i >> 2] >> (8 * (i & 3))) & 0xFFu) != 0u ? 1u << i : 0u;
  } else {
    for (int i = 0; i < 16; ++i)
      if (x + i < end && keep[x + i] != 0) bits |= 1u << i;
  }
  return x + 16 <= end ? bits : x >= end ? 0u : bits & ((1u << (end - x)) - 1u);
}

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const Geometry geo, const PlanCall c, uint32_t* __restrict__ status) {
  __shared__ long long s_before[2], s_all[2];
  __shared__ unsigned s_bad;
  __shared__ int s_warp[kPlanThreads / 32 + 1];
  pdl_wait();
  pdl_launch_dependents();
  const int j = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, S = geo.S, B = geo.B;
  if (tid == 0) { s_before[0] = s_before[1] = s_all[0] = s_all[1] = 0; s_bad = 0u; }
  __syncthreads();

  // a warp per request: what it owns and moves; `fine` says that its tables can be read
  long long before[2] = {0, 0}, all[2] = {0, 0};
  unsigned bad = 0u;
  for (int r = warp; r < B; r += kPlanThreads / 32) {
    const int from = c.parent[r];
    const int spare = c.reserve != nullptr ? c.reserve[r] : 0;
    if (spare < 0) bad |= SWARM_DEV_BAD_LENGTH;
    if (from < -1 || from >= B) { bad |= SWARM_DEV_BAD_PAGE; continue; }
    int n = 0;
    if (from >= 0) {
      const long long base = c.page_base[from], owned = c.page_base[from + 1] - base;
      const int len = c.ctx_len[from];
      if (len < 0 || pages_of(len, S) > owned || base < 0 || base + owned > geo.n_pool_pages) { bad |= SWARM_DEV_BAD_LENGTH; continue; }
      const int P = pages_of(len, S);
      if (c.keep == nullptr) {
        n = P;
      } else {
        const long long lo = base & ~15LL;                  // aligned blocks of 16; those in front of the range are cut off
        for (long long x = lo + lane * 16; x < base + P; x += 512) {
          unsigned bits = keep_bits(c.keep, x, base + P);
          if (x < base) bits &= ~((1u << (base - x)) - 1u);
          n += __popc(bits);
        }
        n = warp_sum(n);
      }
      if (c.in_place && lane == 0) {                        // the order of the requests has to stay: the parent before this one
        for (int r2 = r - 1; r2 >= 0; --r2)
          if (c.parent[r2] >= 0) {
            if (c.parent[r2] >= from) bad |= SWARM_DEV_BAD_PAGE;
            break;
          }
      }
    }
    all[0] += n + max(spare, 0);
    all[1] += n;
    if (r < j) { before[0] += n + max(spare, 0); before[1] += n; }
  }
  if (lane == 0) {
    for (int i = 0; i < 2; ++i) {
      atomicAdd(reinterpret_cast<unsigned long long*>(s_before + i), (unsigned long long)before[i]);
      atomicAdd(reinterpret_cast<unsigned long long*>(s_all + i), (unsigned long long)all[i]);
    }
    if (bad) atomicOr(&s_bad, bad);
  }
  __syncthreads();
  unsigned refused = s_bad;
  if (s_all[0] > geo.n_pool_pages || s_all[1] > c.max_moves) refused |= SWARM_DEV_BAD_LENGTH;
  if (refused != 0u) {                                       // every CTA sees the same: the layout stays what it was
    if (tid == 0) {
      c.new_page_base[j] = c.page_base[j];
      c.new_ctx_len[j] = c.ctx_len[j];
      if (j == B - 1) {
        c.new_page_base[B] = c.page_base[B];
        *c.n_moves = -1;
        atomicOr(status, refused);
      }
    }
    return;
  }
  const long long to = s_before[0];
  long long at = s_before[1];
  if (tid == 0) {
    c.new_page_base[j] = to;
    if (j == B - 1) {
      c.new_page_base[B] = s_all[0];
      *c.n_moves = (int)s_all[1];
    }
  }
  const int from = c.parent[j];
  if (from < 0) {
    if (tid == 0) c.new_ctx_len[j] = 0;
    return;
  }
  const long long base = c.page_base[from];
  const int len = c.ctx_len[from], P = pages_of(len, S);
  const long long lo = base & ~15LL, end = base + P;
  const long long first = at;
  for (long long x0 = lo; x0 < end; x0 += kPlanThreads * 16) {
    const long long x = x0 + tid * 16;
    unsigned bits = x < end ? keep_bits(c.keep, x, end) : 0u;
    if (x < base) bits &= base - x >= 16 ? 0u : ~((1u << (base - x)) - 1u);
    const int mine = __popc(bits);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int ahead = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
      if (w < warp) ahead += s_warp[w];
      total += s_warp[w];
    }
    long long m = at + ahead + incl - mine;
    for (; bits != 0u; bits &= bits - 1u, ++m) {
      c.src[m] = (int)(x + __ffs(bits) - 1);
      c.dst[m] = (int)(to + (m - first));
    }
    at += total;
    __syncthreads();
  }
  if (tid == 0) {
    // a partial last page that is kept stays the last; without it every page is full
    const bool ends = P > 0 && (c.keep == nullptr || c.keep[end - 1] != 0);
    c.new_ctx_len[j] = (int)((at - first) * S - (ends ? P * S - len : 0));
  }
}

// ---- moves ----------------------------------------------------------------------------------------------------------------
constexpr int kChunk = 32 * 1024;                          // bytes of K/V that a CTA moves at a time
constexpr int kTail = 8 * 1024;                            // room for the page's summaries beside its last chunk
constexpr int kMoveSmem = kChunk + kTail + 64;
constexpr int kMoveCtasPerSm = 5;
constexpr int kSetupThreads = 1024, kSetupCtas = 8;
constexpr unsigned kMoveWait = 1u << 22;

struct MoveTables {
  int32_t* reader;     // [n_pool_pages] 1 + place in the order of the last pair that reads the page
  int32_t* pending;    // [n_pool_pages] chunks of the page still to be read
  int32_t* writer;     // [n_pool_pages] place in the order of the first pair that writes the page
  unsigned* ctl;       // [0] next item, [1] pairs that move upward, [2] pairs that move downward (or to another pool)
};
struct MoveShape {
  long long kv_bytes, sum_bytes;   // of a page
  int kv_chunks, sum_chunks;       // sum_chunks: summaries moved as items of their own (0: beside the last chunk, or none)
  int items;                       // of a pair
  bool in_place;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int order_of(int i, int n, int src, int dst, bool in_place) { return in_place && dst > src ? 2 * n - 1 - i : i; }

// Entries of the tables that the pairs touch are cleared, then filled.  One cluster of CTAs, so that a barrier lies between.
__global__ void __launch_bounds__(kSetupThreads)
move_setup_kernel(const Geometry geo, const MoveCall c, const MoveShape m, const MoveTables t, uint32_t* __restrict__ status) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = max(0, min(*c.n_moves, c.max_moves));
  const int first = blockIdx.x * kSetupThreads + threadIdx.x;
  if (first == 0) {
    t.ctl[0] = t.ctl[1] = t.ctl[2] = 0u;
    if (*c.n_moves > c.max_moves) atomicOr(status, SWARM_DEV_BAD_LENGTH);
  }
  auto each = [&](auto&& f) {
    for (int i = first; i < n; i += kSetupThreads * kSetupCtas) {
      const int src = c.src[i], dst = c.dst[i];
      if (src >= 0 && dst >= 0 && src < geo.n_pool_pages && dst < geo.n_pool_pages) f(i, src, dst);
      else f(i, -1, -1);
    }
  };
  each([&](int, int src, int dst) {
    if (src < 0) { atomicOr(status, SWARM_DEV_BAD_PAGE); return; }
    t.writer[dst] = 0x7FFFFFFF;
    if (m.in_place) t.reader[src] = t.pending[src] = t.reader[dst] = t.pending[dst] = 0;
  });
  __threadfence();
  __syncwarp();
  cluster_sync();
  unsigned up = 0u, down = 0u;
  each([&](int i, int src, int dst) {
    if (src < 0) return;
    const int order = order_of(i, n, src, dst, m.in_place);
    if (m.in_place && src == dst) {                          // stays where it is: no item below looks at it unless some pair moves down
      if (atomicMin(t.writer + dst, order) != 0x7FFFFFFF) atomicOr(status, SWARM_DEV_BAD_PAGE);
      return;
    }
    atomicMin(t.writer + dst, order);
    if (!m.in_place) { ++down; return; }
    atomicMax(t.reader + src, order + 1);
    atomicAdd(t.pending + src, m.items);
    if (dst > src) ++up; else ++down;
  });
  if (up) atomicAdd(t.ctl + 1, up);
  if (down) atomicAdd(t.ctl + 2, down);
}

// A warp per CTA; lane 0 copies: page -> shared memory -> page by bulk copies, 32 KB at a time, several CTAs per SM.  Bound by HBM:
// 602 MB inside one pool, pages read once and written once, in 92 us (6.5 TB/s).  Between two pools 766 MB take 100 us (with the plan
// and the tables 115), of which DRAM carries 630 (6.1 TB/s): pages that several requests continue are read from it less than once per
// copy (306 of 383 MB), and 59 MB of the writes are still in L2 at the end.  Five CTAs with 32 KB each are what an SM's shared memory holds; while one waits for readers of its
// destination, the others copy.  Items go to whoever is free, in the order of the moves, which the waits need anyway.
__global__ void __launch_bounds__(32)
move_kernel(const Geometry geo, const MoveCall c, const MoveShape m, const MoveTables t, uint32_t* __restrict__ status) {
  extern __shared__ __align__(128) unsigned char smem[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kChunk + kTail);
  const uint32_t bar_at = smem_addr(bar), buf = smem_addr(smem);
  if (threadIdx.x != 0) return;
  asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar_at));
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_wait();
  pdl_launch_dependents();
  const int n = max(0, min(*c.n_moves, c.max_moves));
  const unsigned up = t.ctl[1], down = t.ctl[2];
  // the order's places: [0, n) downward moves (all moves between two pools), [n, 2n) upward moves
  const long long begin = down ? 0 : n, end = up ? 2LL * n : n;
  const long long items = (end - begin) * m.items;
  unsigned parity = 0u;
  long long next = atomicAdd(t.ctl, 1u);
  while (next < items) {
    const long long item = next;
    const long long place = begin + item / m.items;
    const int part = (int)(item % m.items);
    const int i = (int)(place < n ? place : 2LL * n - 1 - place);
    const int src = c.src[i], dst = c.dst[i];
    const bool there = src >= 0 && dst >= 0 && src < geo.n_pool_pages && dst < geo.n_pool_pages;
    const bool mine = there && !(m.in_place && src == dst) && (!m.in_place || (dst > src) == (place >= n));
    next = atomicAdd(t.ctl, 1u);                              // (asked for before the copy, needed behind it)
    if (m.in_place && there && src == dst && place < n && part == 0 && t.writer[dst] != (int)place)
      atomicOr(status, SWARM_DEV_BAD_PAGE);
    if (!mine) continue;
    // the first pair to write a page writes it, and no pair that comes later may read it
    const bool fine = t.writer[dst] == (int)place && (!m.in_place || t.reader[dst] <= (int)place + 1);
    if (!fine) {
      if (part == 0) atomicOr(status, SWARM_DEV_BAD_PAGE);
      if (m.in_place) red_release_add(reinterpret_cast<unsigned*>(t.pending + src), 0xFFFFFFFFu);
      continue;
    }
    const bool is_sum = part >= m.kv_chunks;
    const long long off = is_sum ? (long long)(part - m.kv_chunks) * kChunk : (long long)part * kChunk;
    const unsigned bytes = (unsigned)min((long long)kChunk, (is_sum ? m.sum_bytes : m.kv_bytes) - off);
    const bool beside = part == m.kv_chunks - 1 && m.sum_bytes > 0 && m.sum_chunks == 0;   // the summaries go along
    const unsigned char* from = is_sum ? reinterpret_cast<const unsigned char*>(c.from_ksum) + src * m.sum_bytes + off
                                       : reinterpret_cast<const unsigned char*>(c.from_pool) + src * m.kv_bytes + off;
    unsigned char* to = is_sum ? reinterpret_cast<unsigned char*>(c.to_ksum) + dst * m.sum_bytes + off
                               : reinterpret_cast<unsigned char*>(c.to_pool) + dst * m.kv_bytes + off;
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // the buffer's last contents are on their way out
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_at), "r"(bytes + (beside ? (unsigned)m.sum_bytes : 0u)) : "memory");
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(buf), "l"(from), "r"(bytes), "r"(bar_at) : "memory");
    if (beside)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(buf + kChunk),
                   "l"(reinterpret_cast<const unsigned char*>(c.from_ksum) + src * m.sum_bytes), "r"((unsigned)m.sum_bytes), "r"(bar_at)
                   : "memory");
    const bool table = part == 0 && c.from_p2c != nullptr;
    int cluster = 0;
    if (table) cluster = __ldcg(c.from_p2c + src);
    unsigned done = 0u;
    for (unsigned polls = 0; polls < kMoveWait && !done; ++polls)
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(done)
          : "r"(bar_at), "r"(parity)
          : "memory");
    parity ^= 1u;
    bool ready = done != 0u;
    if (m.in_place) {
      red_release_add(reinterpret_cast<unsigned*>(t.pending + src), 0xFFFFFFFFu);
      if (ready) ready = wait_zero(reinterpret_cast<const unsigned*>(t.pending + dst));
    }
    if (!ready) {
      atomicOr(status, SWARM_DEV_TIMEOUT);
      if (!done) break;                                      // the copy never came: nothing more through this buffer
      continue;
    }
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(buf), "r"(bytes) : "memory");
    if (beside)
      asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<unsigned char*>(c.to_ksum) + dst * m.sum_bytes),
                   "r"(buf + kChunk), "r"((unsigned)m.sum_bytes)
                   : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    if (table) c.to_p2c[dst] = cluster;
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

constexpr int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

}  // namespace

cudaError_t configure_pages() { return cudaFuncSetAttribute(move_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMoveSmem); }

bool pages_supported(const Geometry& geo) { return geo.n_pool_pages < (1LL << 30); }

// The queue of items (both directions of every pair) is counted in 32 bits, and every CTA counts once more at its end.
bool moves_supported(const Geometry& geo, int max_moves) {
  const long long page = (long long)geo.Hkv * 2 * geo.S * kHeadDim * 2, sums = (long long)geo.Hkv * 2 * kHeadDim * 2;
  const long long items = (page + kChunk - 1) / kChunk + (sums + kChunk - 1) / kChunk;
  return max_moves < (1 << 30) && 2 * items * max_moves < (1LL << 32) - (1 << 20);
}

long long move_pages_workspace_bytes(const Geometry& geo) { return 256 + 3 * align256(geo.n_pool_pages * 4); }

cudaError_t launch_plan_pages(const Geometry& geo, const PlanCall& c, uint32_t* status, cudaStream_t st) {
  return launch_pdl(plan_kernel, dim3((unsigned)geo.B), dim3(kPlanThreads), 0, st, true, geo, c, status);
}

cudaError_t launch_move_pages(const Geometry& geo, const MoveCall& c, void* workspace, uint32_t* status, cudaStream_t st) {
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const int64_t table = align256(geo.n_pool_pages * 4);
  const MoveTables t{reinterpret_cast<int32_t*>(ws + 256), reinterpret_cast<int32_t*>(ws + 256 + table),
                     reinterpret_cast<int32_t*>(ws + 256 + 2 * table), reinterpret_cast<unsigned*>(ws)};
  MoveShape m;
  m.kv_bytes = (long long)geo.Hkv * 2 * geo.S * kHeadDim * 2;
  m.sum_bytes = c.from_ksum != nullptr ? (long long)geo.Hkv * 2 * kHeadDim * 2 : 0;
  m.kv_chunks = (int)((m.kv_bytes + kChunk - 1) / kChunk);
  m.sum_chunks = m.sum_bytes > kTail ? (int)((m.sum_bytes + kChunk - 1) / kChunk) : 0;
  m.items = m.kv_chunks + m.sum_chunks;
  m.in_place = c.in_place;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kSetupCtas);
  cfg.blockDim = dim3(kSetupThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSetupCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, move_setup_kernel, geo, c, m, t, status);
  if (e != cudaSuccess) return e;
  const long long most = (long long)c.max_moves * m.items;
  const unsigned grid = (unsigned)std::max<long long>(1, std::min<long long>(most, (long long)sm_count() * kMoveCtasPerSm));
  return launch_pdl(move_kernel, dim3(grid), dim3(32), (size_t)kMoveSmem, st, true, geo, c, m, t, status);
}

}  // namespace swarm
