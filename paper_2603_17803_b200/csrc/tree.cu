// Attention of a tree of drafted tokens over the paged cache (swarm_tree_attn).
//
// Row (t, h) of request b, t < n_draft[b]:  s_j = q . k_j / sqrt(d) over the context's tokens (of all pages, or of the
// pages selected for head h) and over the drafted tokens j that the mask shows row t;
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  lse = m + log sum_j exp(s_j - m),  in one pass over K and V.
// The g query heads of a KV head and the drafted tokens of a request see the same keys: they are the up to 256 rows of one
// matrix product with every tile of 128 tokens, so K and V are read once for all of them.
//
//   warps 0-3, 4-7   two softmax streams, a thread per row of 128 (tcgen05.ld: lane = row), which holds the 128 scores of a tile in
//                    registers (setmaxnreg: two threads per row, with 64 each, gained nothing and spilled)
//   warp 8           copies: K and V tiles of 32 KB by TMA into a ring, 128-byte swizzle
//   warp 9           matrix products: S = Q K^T (operands in shared memory), O += P V (P from tensor memory)
//   warp 10          copies of the units' queries, each as soon as the last product with the one before is done
//   warp 11          lists the CTA's share of the work
// Tensor memory: S0, S1 (128 columns each; P, in bf16, takes the place of S), O0, O1.  While one stream is in its softmax
// the tensor core works for the other.  Up to 128 rows: the streams take alternate tiles of the same rows, and their
// sums are joined at the end through tensor memory; beyond (kWide), each has 128 rows of its own and both use every tile.
//
// The tiles of all (request, KV head) units form one list that is cut evenly over the CTAs, whatever the lengths
// are; a unit that is cut leaves partial (m, l, O) per CTA, joined by a second kernel with a lane per row.
//
// What bounds it.  Up to 128 rows, HBM: 16 tokens x 4 heads over 128K tokens (537 MB) take 90 us, 6.0 TB/s.  More rows, the chain of a
// tile: product, scores to registers, maximum, exponentials, P back, product.  Two streams overlap theirs, and the tensor pipe is
// active in 48 % of the cycles (64K tokens): 64 tokens x 8 heads over 256K tokens (550 GFLOP) take 495 us, 1.11 PFLOP/s at full
// clocks (570-590 us where the power limit holds the clock at 1.45 GHz).  Leaving out half of the scores' products gained 7 % there,
// of O's products 3 %, the exponentials 8 %: no unit by itself.  Selected pages: 8 x 16 tokens over 256 pages a head (338 MB) take
// 76 us, of which 6 build the lists; the copies are of 2 KB (K) and 4 KB (V), with larger ones it would be 71.  A short prompt (777
// tokens) takes 10 us: two launches, a first tile from DRAM, the chain of two tiles, and the joining.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "swarm_internal.cuh"

namespace swarm {
namespace {

constexpr int kTile = 128;                                 // tokens of a tile, rows of a stream
constexpr int kTileBytes = kTile * kHeadDim * 2;           // K or V of a tile: two halves of 64 coordinates
constexpr int kHalfBytes = kTileBytes / 2;
constexpr int kSoftWarps = 8;
constexpr int kThreads = (kSoftWarps + 4) * 32;
constexpr int kLoadWarp = kSoftWarps, kMmaWarp = kSoftWarps + 1, kQueryWarp = kSoftWarps + 2,
              kListWarp = kSoftWarps + 3;
constexpr int kSegs = 32;                                  // segments of a CTA listed at a time
constexpr int kMaxTreeCtas = kSms;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr unsigned kWaitLimit = 1u << 22;                  // polls of a try_wait that itself blocks briefly
// The running maximum is raised only when a tile exceeds it by more than 2^8: until then the exponentials stay below
// 2^8 * 128 terms, far from any limit of fp32 or bf16, and O needs no rescaling (the final division cancels the reference).
constexpr float kMaxSlack = 8.f;

struct Seg {                                               // tiles [t0, t1) of one unit
  int b, kv;
  int t0, t1;
  int ctx_tiles, ctx_tokens;
  int nd;                                                  // drafted tokens
  int last;                                                // t1 ends the unit
  int base;                                                // first pool page of the request
};

template <bool kWide>
struct Layout {
  static constexpr int kQTiles = kWide ? 2 : 1;
  static constexpr int kSlots = 4;                           // 128 KB in flight; more leave too little L1 (6 and 5: up to 5 % slower)
  static constexpr int kRows = kQTiles * kTile;
  static constexpr int kRing = kQTiles * kTileBytes;
  static constexpr int kBars = kRing + kSlots * kTileBytes;
  static constexpr int kList = kBars + 256;
  static constexpr int kMl = kList + kSegs * (int)sizeof(Seg);   // (m, l) of [stream][row]
  static constexpr int kScan = kMl + 2 * kTile * 8;
  static constexpr int kBytes = kScan + 256;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count));
}
__device__ __forceinline__ void bar_expect(uint64_t* bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait of a whole warp, in step: branches that the lanes take together cost a fraction of diverging ones.  When it runs
// out, `stop` tells the other warps of the CTA, whose waits then end as well.
__device__ __forceinline__ bool bar_wait(uint64_t* bar, unsigned parity, volatile int* stop) {
  for (unsigned polls = 0; polls < kWaitLimit; ++polls) {
    if (__all_sync(0xFFFFFFFFu, bar_try(bar, parity))) return true;
    if (__any_sync(0xFFFFFFFFu, *stop != 0)) return false;
  }
  *stop = 1;
  return false;
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, int c4, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(smem_addr(bar))
      : "memory");
}

// ---- tensor memory and tcgen05 ------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t (&r)[16], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Products and their commits are issued by one lane (`lead` = 1 there, else 0), as predicated instructions of a warp in step: in
// a branch of its own for that lane their operands would not be known to be uniform, and each would take 100 cycles to issue.
__device__ __forceinline__ uint32_t lead_lane() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p;
}
__device__ __forceinline__ void tc_commit(uint64_t* bar, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_addr(bar)),
      "r"(lead)
      : "memory");
}
// Shared-memory operand with the 128-byte swizzle: `lead` and `stride` in bytes.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// bf16 x bf16 -> fp32, 128 x 128; `transposed`: the second operand is stored with its rows along the products' sum
__host__ __device__ constexpr uint32_t mma_shape(bool transposed) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (transposed ? 1u << 16 : 0u) | ((uint32_t)(kTile / 8) << 17) | ((uint32_t)(kTile / 16) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(shape), "r"((uint32_t)add), "r"(lead)
      : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {      // 2^x, relative error about 2^-22; 0 for x = -inf
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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
// 2^y of both for y > -126: y = n + f with n whole and |f| <= 1/2, 2^f by a polynomial of degree 5 (fitted to the least largest
// relative error, 2.1e-7 in fp32), n added to the exponent.  It runs on the multiply-add units, beside the exponentials of the
// special function unit (kByFma: which pairs of eight; a quarter of them is best by 2 % among none to all), which a tile of 256
// rows would keep busy for longer than its K and V take to arrive.
constexpr unsigned kByFma = 0x11u;
__device__ __forceinline__ void exp2_pair(pair_t y, float& lo, float& hi) {
  float y0, y1;
  unpair(y, y0, y1);
  y = pair_of(fmaxf(y0, -125.f), fmaxf(y1, -125.f));
  const pair_t magic = pair_of(12582912.f, 12582912.f), n = add2(y, magic);   // 1.5 * 2^23: the whole part ends in the low bits
  const pair_t f = fma2(add2(n, pair_of(-12582912.f, -12582912.f)), pair_of(-1.f, -1.f), y);
  pair_t r = pair_of(0.0013276466634124517f, 0.0013276466634124517f);
  r = fma2(r, f, pair_of(0.009675540961325169f, 0.009675540961325169f));
  r = fma2(r, f, pair_of(0.05550713464617729f, 0.05550713464617729f));
  r = fma2(r, f, pair_of(0.24022120237350464f, 0.24022120237350464f));
  r = fma2(r, f, pair_of(0.6931469440460205f, 0.6931469440460205f));
  r = fma2(r, f, pair_of(1.0000001192092896f, 1.0000001192092896f));
  float r0, r1, n0, n1;
  unpair(r, r0, r1);
  unpair(n, n0, n1);
  lo = __uint_as_float(__float_as_uint(r0) + (__float_as_uint(n0) << 23));
  hi = __uint_as_float(__float_as_uint(r1) + (__float_as_uint(n1) << 23));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

struct TreeArgs {
  Geometry geo;
  const uint16_t* q;
  const int64_t* page_base;
  const int32_t* ctx_len;
  const int32_t* n_draft;
  const uint32_t* mask;       // [B][T][words] or null: a chain
  const int2* list;           // selected pages: [B*Hkv][list_cap] {page, heads}; null: all pages
  const int32_t* list_tokens; // [B*Hkv] context tokens among them
  int list_cap;
  int T, words, row_blocks, chunks;
  int tile_tokens;            // drafted tokens of a tile of rows: row r of a tile is token r / g of it, head r % g
  float4* part_o;             // [CTA][2][32 groups of four coordinates][rows]
  float2* part_ml;            // [CTA][2][rows]
  int32_t* unit_first;        // [B*Hkv] 2 * chunk + place of the unit's first partial
  int32_t* unit_last;         // [B*Hkv] its last chunk
  uint16_t* out;
  float* lse;
  uint32_t* status;
};

// A length fits the request's pages, and, where pages are selected, the lists of at most Pmax pages that the selection makes.
__device__ __forceinline__ bool length_fits(const TreeArgs& a, int len, long long owned) {
  const int P = pages_of(len, a.geo.S);
  return len >= 0 && P <= owned && (a.list == nullptr || P <= a.geo.Pmax);
}
// Context tokens (those of the selected pages, if there is a selection), drafted tokens and first pool page of a unit; no drafted
// tokens where the request's length does not fit its pages.
__device__ __forceinline__ void unit_lengths(const TreeArgs& a, int u, int& ctx, int& nd, int& base, bool& bad) {
  const int b = u / a.geo.Hkv;
  const int len = a.ctx_len[b];
  base = (int)a.page_base[b];
  const long long owned = a.page_base[b + 1] - a.page_base[b];
  nd = a.n_draft[b];
  bad = nd < 0 || nd > a.T;
  nd = max(0, min(nd, a.T));
  if (!length_fits(a, len, owned)) {
    bad = true;
    nd = 0;
  }
  ctx = a.list != nullptr ? a.list_tokens[u] : len;
}
__device__ __forceinline__ int tiles_of(int ctx, int nd) {
  return nd == 0 ? 0 : (ctx + kTile - 1) / kTile + (nd + kTile - 1) / kTile;
}

template <bool kWide>
__global__ void __launch_bounds__(kThreads, 1)
tree_attn_kernel(const __grid_constant__ CUtensorMap pool_tile, const __grid_constant__ CUtensorMap pool_page,
                 const __grid_constant__ CUtensorMap pool_page_half,
                 const __grid_constant__ CUtensorMap draft_k, const __grid_constant__ CUtensorMap draft_v,
                 const __grid_constant__ CUtensorMap queries, const TreeArgs a) {
  using L = Layout<kWide>;
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t *full = bars, *empty = bars + 6, *s_full = bars + 12, *p_full = bars + 14, *q_full = bars + 16, *joined = bars + 17,
           *drained = bars + 18, *q_empty = bars + 19, *o_full = bars + 20;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(bars + 22);
  volatile int* stop = reinterpret_cast<volatile int*>(bars + 23);
  int* n_segs = reinterpret_cast<int*>(bars + 24);
  Seg* list = reinterpret_cast<Seg*>(smem + L::kList);
  float2* ml = reinterpret_cast<float2*>(smem + L::kMl);
  int* scan = reinterpret_cast<int*>(smem + L::kScan);

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);    // (known to be the same for the whole warp: see lead_lane)
  const int rb = blockIdx.x % a.row_blocks, chunk = blockIdx.x / a.row_blocks;
  const int g = a.geo.g, Hkv = a.geo.Hkv, S = a.geo.S;
  const int units = a.geo.B * Hkv;
  const int first_tile = rb * L::kQTiles;                    // of rows
  const auto row_tiles = [&](int nd) { return (nd + a.tile_tokens - 1) / a.tile_tokens - first_tile; };   // <= 0: none for this CTA

  if (tid == 0) {
    for (int i = 0; i < L::kSlots; ++i) { bar_init(full + i, 1); bar_init(empty + i, 1); }
    for (int i = 0; i < 2; ++i) { bar_init(s_full + i, 1); bar_init(o_full + i, 1); bar_init(p_full + i, kSoftWarps / 2); }
    bar_init(q_full, 1);
    bar_init(q_empty, 1);
    bar_init(joined, kSoftWarps);
    bar_init(drained, 1);
    *stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tc_fence_before();
  }
  pdl_wait();
  pdl_launch_dependents();

  // ---- this CTA's share of all tiles: the list of units is summed by the whole CTA, the unit of its first tile found.  Up to a
  // unit per thread, their lengths stay in shared memory (the ring is still empty) for the first list of segments.
  int4* lengths = reinterpret_cast<int4*>(smem + L::kRing);
  const bool cached = units <= kThreads;
  const int per = (units + kThreads - 1) / kThreads;
  const int u_lo = min(units, tid * per), u_hi = min(units, u_lo + per);
  int mine = 0;
  for (int u = u_lo; u < u_hi; ++u) {
    int ctx, nd, base;
    bool bad;
    unit_lengths(a, u, ctx, nd, base, bad);
    if (bad && blockIdx.x == 0 && u % Hkv == 0) atomicOr(a.status, SWARM_DEV_BAD_LENGTH);
    if (cached) lengths[u] = make_int4(ctx, nd, base, 0);
    mine += tiles_of(ctx, nd);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (in front of the copies that go there)
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  tc_fence_after();
  int before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const int v = scan[w];
    if (w < warp) before += v;
    total += v;
  }
  const int each = total / a.chunks, more = total - each * a.chunks;   // the first `more` CTAs take one tile more
  const int w0 = chunk * each + min(chunk, more), w1 = w0 + each + (chunk < more ? 1 : 0);
  if (w0 < w1 && before <= w0 && w0 < before + mine) {       // one thread: its units hold the first tile
    int u = u_lo, at = before;
    for (; u + 1 < u_hi; ++u) {
      int ctx, nd, base;
      bool bad;
      unit_lengths(a, u, ctx, nd, base, bad);
      const int n = tiles_of(ctx, nd);
      if (at + n > w0) break;
      at += n;
    }
    scan[kThreads / 32] = u;
    scan[kThreads / 32 + 1] = at;
  }
  __syncthreads();
  const uint32_t tmem = *tmem_at;

  // state of the roles, carried from one list of segments to the next
  int slot = 0;
  unsigned ring_phase = 0u;                                  // parity of the current round through the ring
  unsigned s_phase = 0u, p_phase = 0u, q_phase = 0u, j_phase = 0u;   // (p_phase: a bit per stream)
  int issued = 0, asked = 0;                                 // copies started of tiles, of queries
  bool ok = true;
  bool first_list = true;
  int u_next = w0 < w1 ? scan[kThreads / 32] : units;
  int at_next = w0 < w1 ? scan[kThreads / 32 + 1] : 0;

  int count = 0;
  // Calls `work` for one list of segments after the other; every warp of the CTA goes through the same lists.
  auto lists = [&](auto&& work) {
    while (u_next < units && at_next < w1) {
      __syncthreads();                                       // the previous list has been worked through
      if (*stop != 0) break;
      if (warp == kListWarp) {                                   // the next (up to 32) units with tiles in this CTA's share
        const int u = u_next + lane;
        int ctx = 0, nd = 0, base = 0, n = 0;
        bool bad;
        if (u < units) {
          if (cached && first_list) {
            const int4 v = lengths[u];
            ctx = v.x;
            nd = v.y;
            base = v.z;
          } else {
            unit_lengths(a, u, ctx, nd, base, bad);
          }
          n = tiles_of(ctx, nd);
        }
        int end = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, end, o);
          if (lane >= o) end += v;
        }
        end += at_next;
        const int begin = end - n;
        const bool here = n > 0 && begin < w1 && end > w0;
        const unsigned all = __ballot_sync(0xFFFFFFFFu, here);
        if (here) {
          Seg s;
          s.b = u / Hkv;
          s.kv = u - s.b * Hkv;
          s.t0 = max(w0, begin) - begin;
          s.t1 = min(w1, end) - begin;
          s.ctx_tiles = (ctx + kTile - 1) / kTile;
          s.ctx_tokens = ctx;
          s.nd = nd;
          s.last = s.t1 == n;
          s.base = base;
          list[__popc(all & ((1u << lane) - 1u))] = s;
          if (rb == 0) {
            if (s.t0 == 0) a.unit_first[u] = 2 * chunk + (begin == w0 ? 0 : 1);
            if (s.last) a.unit_last[u] = chunk;
          }
        }
        if (lane == 31) scan[kThreads / 32 + 2] = end;
        if (lane == 0) *n_segs = __popc(all);
      }
      __syncthreads();
      count = *n_segs;
      u_next += 32;
      at_next = scan[kThreads / 32 + 2];
      work();
      first_list = false;
    }
  };

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");     // 128 * 72 + 256 * 216 = 384 * 168, what the CTA was launched with
    if (warp == kLoadWarp) {
      // ---- copies, in the order the matrix products use them
      // which: 0 = K, 1 = V; `page`: the lane's page of the tile, where pages are selected
      auto load_tile = [&](const Seg& s, int t, int which, int page) -> bool {
        if (issued >= L::kSlots && !bar_wait(empty + slot, ring_phase ^ 1u, stop)) return false;
        const uint32_t dst = smem_addr(smem + L::kRing + slot * kTileBytes);
        uint64_t* bar = full + slot;
        if (t >= s.ctx_tiles) {                              // drafted tokens; rows behind the last are filled with zeros
          if (lane == 0) {
            bar_expect(bar, kTileBytes);
            tma_load(dst, which == 0 ? &draft_k : &draft_v, 0, (t - s.ctx_tiles) * kTile, 0, s.kv, s.b, bar);
          }
        } else if (a.list == nullptr) {
          if (lane == 0) {
            bar_expect(bar, kTileBytes);
            tma_load(dst, &pool_tile, 0, 0, s.base + t * (kTile / S), 0, s.kv * 2 + which, bar);
          }
        } else {                                             // the tile's pages one by one, a lane each
          const int per_tile = kTile / S, pages = min(per_tile, (s.ctx_tokens + S - 1) / S - t * per_tile);
          if (lane == 0) bar_expect(bar, (unsigned)(pages * S * kHeadDim * 2));
          __syncwarp();
          // K's rows have to lie at one distance through the whole tile, a half of the coordinates at a time; V enters the product 16
          // tokens at a time, so that a page's V may stay together: fewer and larger copies (selected pages 80.0 -> 76.4 us)
          if (lane < pages && which == 0)
            for (int h = 0; h < 2; ++h)
              tma_load(dst + h * kHalfBytes + lane * S * 128, &pool_page_half, 0, 0, s.base + page, h, s.kv * 2, bar);
          else if (lane < pages)
            tma_load(dst + lane * S * 256, &pool_page, 0, 0, s.base + page, 0, s.kv * 2 + 1, bar);
        }
        __syncwarp();
        ++issued;
        if (++slot == L::kSlots) { slot = 0; ring_phase ^= 1u; }
        return true;
      };
      lists([&] {
      for (int i = 0; ok && i < count; ++i) {
        const Seg s = list[i];
        if (row_tiles(s.nd) <= 0) continue;
        const int n = s.t1 - s.t0;
        // K of a tile, and V of the one that many tiles earlier whose softmax is done by then
        const int behind = kWide && row_tiles(s.nd) > 1 ? 1 : 2;
        // the list of pages is read a tile ahead: its latency would lie in front of every copy
        const int per_tile = kTile / S, listed = a.list != nullptr ? (s.ctx_tokens + S - 1) / S : 0;
        const int2* pages = a.list + (long long)(s.b * Hkv + s.kv) * a.list_cap + lane;
        auto page_of = [&](int t) { return lane < per_tile && t * per_tile + lane < listed ? pages[t * per_tile].x : 0; };
        int now = page_of(s.t0), next = 0, before = 0, before2 = 0;
        for (int k = 0; ok && k < 2 * (n + behind); ++k) {
          const int which = (k & 1) ^ 1, t = (k >> 1) - which * behind;
          if (which == 1) next = page_of(s.t0 + (k >> 1) + 1);
          if (t >= 0 && t < n) ok = load_tile(s, s.t0 + t, which, which == 0 ? now : behind == 1 ? before : before2);
          if (which == 0) { before2 = before; before = now; now = next; }
        }
      }
      });
    } else if (warp == kMmaWarp) {
      // ---- matrix products
      const uint32_t q_at = smem_addr(smem);
      auto advance = [&](int n) {
        slot += n;
        if (slot >= L::kSlots) { slot -= L::kSlots; ring_phase ^= 1u; }
      };
      // place of the ring `ahead` copies further on
      auto place = [&](int ahead, int& sl, unsigned& ph) {
        sl = slot + ahead;
        ph = ring_phase;
        if (sl >= L::kSlots) { sl -= L::kSlots; ph ^= 1u; }
      };
      const uint32_t lead = lead_lane();
      auto scores = [&](int st, int sl, int q_tile) {        // S = Q K^T
        const uint64_t qd = operand(q_at + q_tile * kTileBytes, 16, 1024);
        const uint64_t kd = operand(smem_addr(smem + L::kRing + sl * kTileBytes), 16, 1024);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = (uint32_t)((k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2);
          mma_ss(tmem + st * kTile, qd + off, kd + off, mma_shape(false), k > 0, lead);
        }
      };
      // O += P V.  V's halves lie apart through the whole tile, or, of selected pages, through a page; the offsets of 16 tokens are
      // those of odd and even places.
      auto values = [&](int st, int sl, bool by_page, bool add) {
        const uint64_t vd = operand(smem_addr(smem + L::kRing + sl * kTileBytes), by_page ? S * 128 : kHalfBytes, 1024);
        const uint32_t odd = by_page && S == 16 ? 4096 >> 4 : 2048 >> 4, even = by_page ? 8192 >> 4 : 4096 >> 4;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          mma_ts(tmem + 256 + st * kTile, tmem + st * kTile + k * 8, vd + (uint64_t)((k >> 1) * even + (k & 1) * odd), mma_shape(true),
                 add || k > 0, lead);
      };
      auto commit = [&](uint64_t* bar) { tc_commit(bar, lead); };
      // V rows behind the tile's last token may hold anything, and 0 * NaN must not reach the sums
      auto clear_tail = [&](const Seg& s, int t, int sl) {
        const int left = t < s.ctx_tiles ? s.ctx_tokens - t * kTile : s.nd - (t - s.ctx_tiles) * kTile;
        if (left >= kTile) return;
        unsigned char* v = smem + L::kRing + sl * kTileBytes;
        const int rows = a.list != nullptr && t < s.ctx_tiles ? S : kTile;   // (16, 32 or 128) of a block whose halves lie apart
        for (int i = lane; i < (kTile - left) * 16; i += 32) {
          const int token = left + (i >> 4);
          *reinterpret_cast<uint4*>(v + (token & -rows) * 256 + ((i >> 3) & 1) * rows * 128 + (token & (rows - 1)) * 128 + (i & 7) * 16) =
              make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      };
      lists([&] {
      for (int i = 0; ok && i < count; ++i) {
        const Seg s = list[i];
        if (row_tiles(s.nd) <= 0) continue;
        const bool wide = kWide && row_tiles(s.nd) > 1;
        const int n = s.t1 - s.t0;
        ok = bar_wait(q_full, q_phase, stop);
        q_phase ^= 1u;
        if (!ok) break;
        tc_fence_after();
        // Wide: both streams use every tile, step by step in turn: O += P V of a tile, then S of the next.  Else the streams take
        // alternate tiles: O += P V of a tile, then S of the one after the next.
        const int steps = wide ? 2 * n + 2 : n + 2;
#pragma unroll 1
        for (int j = 0; j < steps; ++j) {
          const int st = j & 1, tv = wide ? (j >> 1) - 1 : j - 2, tk = wide ? j >> 1 : j;
          const bool has_v = tv >= 0 && tv < n, has_k = tk < n;
          const bool opens = !wide || st == 0, closes = !wide || st == 1;   // the first and the last use of the tiles
          int sv, sk;
          unsigned pv, pk;
          place(0, sv, pv);
          place(has_v ? 1 : 0, sk, pk);
          if (has_v) {
            if (opens) {
              if (!(ok = bar_wait(full + sv, pv, stop))) break;
              clear_tail(s, s.t0 + tv, sv);
            }
            ok = bar_wait(p_full + st, (p_phase >> st) & 1u, stop);
            p_phase ^= 1u << st;
            if (!ok) break;
            tc_fence_after();
            values(st, sv, a.list != nullptr && s.t0 + tv < s.ctx_tiles, tv >= (wide ? 1 : 2));
            if (closes) commit(empty + sv);
          }
          if (has_k) {
            if (opens && !(ok = bar_wait(full + sk, pk, stop))) break;
            scores(st, sk, wide ? st : 0);
            commit(s_full + st);
            if (closes) {
              commit(empty + sk);
              if (tk == n - 1) commit(q_empty);
            }
          } else if (has_v) {
            commit(o_full + st);
          }
          if (closes) advance((has_v ? 1 : 0) + (has_k ? 1 : 0));
        }
      }
      });
    } else if (warp == kQueryWarp) {
      lists([&] {
        for (int i = 0; ok && i < count; ++i) {
          const Seg s = list[i];
          if (row_tiles(s.nd) <= 0) continue;
          if (asked > 0 && !(ok = bar_wait(q_empty, q_phase, stop))) break;
          if (asked > 0) q_phase ^= 1u;
          const int tiles = min(L::kQTiles, row_tiles(s.nd));
          if (lane == 0) {
            bar_expect(q_full, (unsigned)(tiles * a.tile_tokens * g * kHeadDim * 2));
            for (int j = 0; j < 2 * tiles; ++j)              // a tile's halves of 64 coordinates; tokens behind the last are zeros
              tma_load(smem_addr(smem + (j >> 1) * kTileBytes + (j & 1) * kHalfBytes), &queries, (j & 1) * 64, 0,
                       (first_tile + (j >> 1)) * a.tile_tokens, s.kv, s.b, q_full);
          }
          __syncwarp();
          ++asked;
        }
      });
    } else {
      lists([] {});
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---- softmax
    const int st = warp >> 2, lane_row = (warp & 3) * 32 + lane;
    const uint32_t lane_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_at = lane_at + st * kTile, o_at = lane_at + 256 + st * kTile;
    unsigned o_phase = 0u;
    const float scale = 0.08838834764831845f * kLog2e;       // 1 / sqrt(128), in the log2 domain
    lists([&] {
      for (int i = 0; ok && i < count; ++i) {
        const Seg& s = list[i];                              // (read where it is needed: registers are short here)
        if (row_tiles(s.nd) <= 0) continue;
        const bool wide = kWide && row_tiles(s.nd) > 1;
        const int tile_first = (first_tile + (wide ? st : 0)) * a.tile_tokens;   // first token of this stream's rows
        const int t_row = tile_first + lane_row / g, h_row = lane_row % g;       // this thread's row
        const int rows = min(a.tile_tokens, s.nd - tile_first) * g;              // of the stream
        const bool there = lane_row < rows, busy = lane_row - lane < rows;       // busy: some row of the warp exists
        const int n = s.t1 - s.t0;
        const int my_n = wide ? n : (n + 1 - st) >> 1;
        float m = -INFINITY, l = 0.f;
        // the heads that have selected the lane's page of a tile
        auto heads_of = [&](int t) {
          const int at = t * (kTile / S) + lane;
          return lane < kTile / S && at * S < s.ctx_tokens && t < s.ctx_tiles ? a.list[(long long)(s.b * Hkv + s.kv) * a.list_cap + at].y : 0;
        };
        int heads_ahead = a.list != nullptr ? heads_of(s.t0 + (wide ? 0 : st)) : 0;
        for (int k = 0; k < my_n; ++k) {
          const int t = s.t0 + (wide ? k : 2 * k + st);
          // Which of the tile's tokens the row sees: all; or whole pages, a bit per 16 tokens; or token by token.
          const bool of_ctx = t < s.ctx_tiles;
          const int first = (of_ctx ? t : t - s.ctx_tiles) * kTile, left = (of_ctx ? s.ctx_tokens : s.nd) - first;
          const bool by_token = !of_ctx || left < kTile, by_page = a.list != nullptr && of_ctx;
          uint32_t see[4] = {0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu}, on = 0xFFu;
          if (by_page) {
            const int heads = heads_ahead;                   // of the lane's page; the next tile's are on their way meanwhile
            heads_ahead = heads_of(t + (wide ? 1 : 2));
            uint32_t bits = 0u;
#pragma unroll
            for (int p = 0; p < 8; ++p) bits |= ((uint32_t)__shfl_sync(0xFFFFFFFFu, heads, S == 16 ? p : p >> 1) >> h_row & 1u) << p;
            on = bits;
          }
          if (busy && by_token) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              see[w] = left >= 32 * w + 32 ? 0xFFFFFFFFu : left > 32 * w ? (1u << (left - 32 * w)) - 1u : 0u;
              const int at = first + 32 * w;
              if (of_ctx)
                see[w] &= ((on >> 2 * w) & 1u ? 0xFFFFu : 0u) | ((on >> 2 * w) & 2u ? 0xFFFF0000u : 0u);
              else if (a.mask == nullptr)
                see[w] &= t_row >= at + 31 ? 0xFFFFFFFFu : t_row >= at ? (2u << (t_row - at)) - 1u : 0u;
              else if (t_row < s.nd)
                see[w] &= at / 32 < a.words ? a.mask[((long long)s.b * a.T + t_row) * a.words + at / 32] : 0u;
            }
          }
          if (!(ok = bar_wait(s_full + st, s_phase, stop))) break;
          s_phase ^= 1u;
          tc_fence_after();
          if (busy) {
            uint32_t x[4][32];
#pragma unroll
            for (int w = 0; w < 4; ++w) tmem_ld32(x[w], s_at + 32 * w);
            tmem_wait_ld();
            if (by_token) {
#pragma unroll
              for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (!((see[w] >> e) & 1u)) x[w][e] = 0xFF800000u;   // -inf, whatever the padding held
            }
            float top = -INFINITY;
#pragma unroll
            for (int p = 0; p < 8; ++p) {
              float mx = -INFINITY;
#pragma unroll
              for (int e = 0; e < 16; e += 2) mx = max3(mx, __uint_as_float(x[p >> 1][16 * (p & 1) + e]), __uint_as_float(x[p >> 1][16 * (p & 1) + e + 1]));
              top = fmaxf(top, (on >> p) & 1u ? mx : -INFINITY);
            }
            top *= scale;
            if (k == 0) {
              m = top;
            } else {
              const bool raise = top > m + kMaxSlack;        // (m = -inf: any finite value)
              if (__any_sync(0xFFFFFFFFu, raise)) {
                const float factor = raise ? exp2_fast(m - top) : 1.f;
                if (raise) m = top;
                l *= factor;
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                  uint32_t o[16];
                  tmem_ld16(o, o_at + 16 * w);
                  tmem_wait_ld();
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                  tmem_st16(o_at + 16 * w, o);
                }
                tmem_wait_st();
              }
            }
            const float ref = m == -INFINITY ? 0.f : -m;
            // P is rounded to bf16 for the matrix product with V (half a step, 2^-8 of each weight at most); the sum keeps fp32
            pair_t sum[2] = {0ull, 0ull};
            const pair_t scale2 = pair_of(scale, scale);
            auto weigh = [&](auto mixed) {
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                uint32_t p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  // (a page that the row's head has not selected: -inf in place of -m)
                  const float r = decltype(mixed)::value || ((on >> (2 * w + (e >> 3))) & 1u) ? ref : -INFINITY;
                  const pair_t y = fma2(pair_of(__uint_as_float(x[w][2 * e]), __uint_as_float(x[w][2 * e + 1])), scale2, pair_of(r, r));
                  float p0, p1;
                  if (decltype(mixed)::value && kByFma >> (e & 7) & 1) {
                    exp2_pair(y, p0, p1);
                  } else {
                    unpair(y, p0, p1);
                    p0 = exp2_fast(p0);
                    p1 = exp2_fast(p1);
                  }
                  sum[e & 1] = add2(sum[e & 1], pair_of(p0, p1));
                  const __nv_bfloat162 pair = __floats2bfloat162_rn(p0, p1);
                  p[e] = *reinterpret_cast<const uint32_t*>(&pair);
                }
                tmem_st16(s_at + 16 * w, p);
              }
            };
            if (by_token || by_page) weigh(std::false_type());   // (-inf has to give 0)
            else weigh(std::true_type());
            float s0, s1;
            unpair(add2(sum[0], sum[1]), s0, s1);
            l += s0 + s1;
            tmem_wait_st();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(p_full + st);
        }
        if (!ok) break;
        if (my_n > 0) {
          if (!(ok = bar_wait(o_full + st, o_phase, stop))) break;   // the last product with V is complete
          o_phase ^= 1u;
        }
        // up to 128 rows both streams hold sums of the same rows; each thread joins half of the coordinates
        float a_own = 1.f, a_other = 0.f;
        if (!wide) {
          ml[st * kTile + lane_row] = make_float2(m, l);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(joined);
          if (!(ok = bar_wait(joined, j_phase, stop))) break;
          j_phase ^= 1u;
          tc_fence_after();
          const float2 other = ml[(st ^ 1) * kTile + lane_row];
          const float both = fmaxf(m, other.x);
          a_own = m == -INFINITY ? 0.f : exp2_fast(m - both);
          a_other = other.x == -INFINITY ? 0.f : exp2_fast(other.x - both);
          l = l * a_own + other.y * a_other;
          m = both;
        } else {
          tc_fence_after();
        }
        if (busy) {
          const bool whole = s.t0 == 0 && s.last;
          const float inv = l > 0.f ? 1.f / l : 0.f;
          const long long part = blockIdx.x * 2 + (i == 0 && first_list ? 0 : 1);
          const int r = (wide ? st * kTile : 0) + lane_row;  // row of the block
          const long long at = ((long long)s.b * a.T + t_row) * a.geo.Hq + s.kv * g + h_row;
          const bool own_on = my_n > 0, other_on = !wide && (st == 1 || n > 1);   // (a stream without a tile has written no O)
          const int width = wide ? 128 : 64, col0 = wide ? 0 : st * 64;
          for (int col = col0; col < col0 + width; col += 16) {
            uint32_t o[16], o2[16];
            tmem_ld16(o, lane_at + 256 + st * kTile + col);
            if (!wide) tmem_ld16(o2, lane_at + 256 + (st ^ 1) * kTile + col);
            tmem_wait_ld();
            float f[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              f[e] = own_on ? __uint_as_float(o[e]) * a_own : 0.f;
              if (other_on) f[e] += __uint_as_float(o2[e]) * a_other;
            }
            if (there) {
              if (whole) {
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                  uint4 v;
                  uint32_t* pv = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                  for (int z = 0; z < 4; ++z) {
                    const __nv_bfloat162 pair = __floats2bfloat162_rn(f[e + 2 * z] * inv, f[e + 2 * z + 1] * inv);
                    pv[z] = *reinterpret_cast<const uint32_t*>(&pair);
                  }
                  *reinterpret_cast<uint4*>(a.out + at * kHeadDim + col + e) = v;
                }
              } else {
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                  __stcg(a.part_o + (part * 32 + (col + e) / 4) * L::kRows + r, make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]));
              }
            }
          }
          if (there && col0 == 0) {
            if (whole) a.lse[at] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
            else __stcg(a.part_ml + part * L::kRows + r, make_float2(m, l));
          }
        }
        // the rows' sums and O may be written again once all warps are here
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(joined);
        if (!(ok = bar_wait(joined, j_phase, stop))) break;
        j_phase ^= 1u;
      }
    });
  }
  __syncthreads();

  if (*stop != 0) {
    // a wait ran out: copies and products under way still write to this CTA's memory
    if (tid == 0) atomicOr(a.status, SWARM_DEV_TIMEOUT);
    if (warp == kLoadWarp) {
      for (int i = 0; i < min(issued, L::kSlots); ++i) {
        if (--slot < 0) { slot = L::kSlots - 1; ring_phase ^= 1u; }
        for (unsigned polls = 0; polls < kWaitLimit && !bar_try(full + slot, ring_phase); ++polls) { }
      }
    }
    if (warp == kQueryWarp && asked > 0)
      for (unsigned polls = 0; polls < kWaitLimit && !bar_try(q_full, (unsigned)(asked - 1) & 1u); ++polls) { }
    if (warp == kMmaWarp) {
      tc_commit(drained, lead_lane());
      for (unsigned polls = 0; polls < kWaitLimit && !bar_try(drained, 0u); ++polls) { }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

// Joins the partial sums of the units that were cut: a lane per row, 16 coordinates per warp, and kSplit warps that share a unit's
// partials (few units are cut into many).  The partials lie with the rows innermost, so that both kernels touch whole lines.
template <int kQTiles, int kSplit>
__global__ void __launch_bounds__(256)
tree_merge_kernel(const TreeArgs a, int groups, int tiles) {
  constexpr int kRows = kQTiles * kTile, kCols = 8 / kSplit;  // kCols groups of 16 coordinates per CTA
  __shared__ float s_ml[kSplit > 1 ? kSplit * 64 : 1];
  __shared__ float s_o[kSplit > 1 ? kSplit * 16 * 32 : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, split = warp / kCols;
  int id = blockIdx.x;
  const int col = (id % kSplit) * kCols + warp % kCols;
  id /= kSplit;
  const int group = id % groups;
  id /= groups;
  const int tile = id % tiles, u = id / tiles;
  const int b = u / a.geo.Hkv, kv = u - b * a.geo.Hkv, g = a.geo.g;
  const int in_tile = group * 32 + lane, t = tile * a.tile_tokens + in_tile / g, h = in_tile % g;
  // (the caller's tables: nothing between the wait of the kernel in front and here writes them; read past L1, since this kernel
  // has not waited for anything yet)
  const int len = __ldcg(a.ctx_len + b);
  const long long owned = __ldcg(a.page_base + b + 1) - __ldcg(a.page_base + b);
  const int nd = !length_fits(a, len, owned) ? 0 : max(0, min(__ldcg(a.n_draft + b), a.T));
  pdl_wait();
  const int first = a.unit_first[u], last = a.unit_last[u];  // (not written where nd is 0)
  pdl_launch_dependents();
  if (tile * a.tile_tokens >= nd) return;
  const int c0 = first >> 1, n = last - c0 + 1;
  if (n <= 1) return;                                        // written by the CTA that had the whole unit
  if (first < 0 || last >= a.chunks) return;                 // (a wait ran out and the unit was not listed: reported)
  const bool here = in_tile < a.tile_tokens * g && t < nd;
  const int rb = tile / kQTiles, r = tile % kQTiles * kTile + min(in_tile, kTile - 1);
  float M = -INFINITY, sum = 0.f;
  float4 o[4];
#pragma unroll
  for (int z = 0; z < 4; ++z) o[z] = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kAhead = 3;
  for (int i0 = split; here && i0 < n; i0 += kSplit * kAhead) {
    float2 ml[kAhead];
    float4 v[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int c = i0 + i * kSplit;
      ml[i] = make_float2(-INFINITY, 0.f);
      if (c < n) {
        const long long p = (long long)((c0 + c) * a.row_blocks + rb) * 2 + (c == 0 ? first & 1 : 0);
        ml[i] = __ldcg(a.part_ml + p * kRows + r);
#pragma unroll
        for (int z = 0; z < 4; ++z) v[i][z] = __ldcg(a.part_o + (p * 32 + col * 4 + z) * kRows + r);
      }
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == -INFINITY ? 0.f : top, keep = exp2_fast(M - ref);
    M = top;
    sum *= keep;
#pragma unroll
    for (int z = 0; z < 4; ++z) { o[z].x *= keep; o[z].y *= keep; o[z].z *= keep; o[z].w *= keep; }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i * kSplit >= n) break;
      const float w = exp2_fast(ml[i].x - ref);
      sum = fmaf(ml[i].y, w, sum);
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        o[z].x = fmaf(v[i][z].x, w, o[z].x); o[z].y = fmaf(v[i][z].y, w, o[z].y);
        o[z].z = fmaf(v[i][z].z, w, o[z].z); o[z].w = fmaf(v[i][z].w, w, o[z].w);
      }
    }
  }
  if constexpr (kSplit > 1) {
    s_ml[split * 64 + lane] = M;
    s_ml[split * 64 + 32 + lane] = sum;
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      s_o[(split * 16 + 4 * z) * 32 + lane] = o[z].x;
      s_o[(split * 16 + 4 * z + 1) * 32 + lane] = o[z].y;
      s_o[(split * 16 + 4 * z + 2) * 32 + lane] = o[z].z;
      s_o[(split * 16 + 4 * z + 3) * 32 + lane] = o[z].w;
    }
    __syncthreads();
    // two coordinates per warp
    static_assert(kSplit == 8, "16 coordinates over 8 warps");
    M = s_ml[lane];
#pragma unroll
    for (int i = 1; i < kSplit; ++i) M = fmaxf(M, s_ml[i * 64 + lane]);
    const float ref = M == -INFINITY ? 0.f : M;
    sum = 0.f;
    float o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int i = 0; i < kSplit; ++i) {
      const float w = exp2_fast(s_ml[i * 64 + lane] - ref);
      sum = fmaf(s_ml[i * 64 + 32 + lane], w, sum);
      o0 = fmaf(s_o[(i * 16 + 2 * warp) * 32 + lane], w, o0);
      o1 = fmaf(s_o[(i * 16 + 2 * warp + 1) * 32 + lane], w, o1);
    }
    if (!here) return;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const long long at = ((long long)b * a.T + t) * a.geo.Hq + kv * g + h;
    *reinterpret_cast<__nv_bfloat162*>(a.out + at * kHeadDim + col * 16 + 2 * warp) = __floats2bfloat162_rn(o0 * inv, o1 * inv);
    if (warp == 0 && col == 0) a.lse[at] = sum > 0.f ? (M + log2f(sum)) * kLn2 : -INFINITY;
  } else {
    if (!here) return;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const long long at = ((long long)b * a.T + t) * a.geo.Hq + kv * g + h;
#pragma unroll
    for (int z = 0; z < 4; z += 2) {
      const __nv_bfloat162 w[4] = {__floats2bfloat162_rn(o[z].x * inv, o[z].y * inv), __floats2bfloat162_rn(o[z].z * inv, o[z].w * inv),
                                   __floats2bfloat162_rn(o[z + 1].x * inv, o[z + 1].y * inv), __floats2bfloat162_rn(o[z + 1].z * inv, o[z + 1].w * inv)};
      *reinterpret_cast<uint4*>(a.out + at * kHeadDim + col * 16 + z * 4) = *reinterpret_cast<const uint4*>(w);
    }
    if (col == 0) a.lse[at] = sum > 0.f ? (M + log2f(sum)) * kLn2 : -INFINITY;
  }
}

// The pages that the heads of a KV head have selected, ascending, each with the heads that did: a CTA per unit.  The
// union is a bitmap in shared memory; a page's place in the list is the number of set bits below it.
__global__ void __launch_bounds__(256)
tree_list_kernel(const TreeArgs a, const int32_t* __restrict__ sel, const int32_t* __restrict__ n_sel, int2* __restrict__ list,
                 int32_t* __restrict__ list_tokens) {
  extern __shared__ uint32_t s_map[];                        // [words] bits, then [words] set bits in front
  __shared__ int s_sum[8];
  const int u = blockIdx.x, b = u / a.geo.Hkv, kv = u - b * a.geo.Hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words = (a.geo.Pmax + 31) / 32;
  int* s_before = reinterpret_cast<int*>(s_map + words);
  for (int i = tid; i < words; i += 256) s_map[i] = 0u;
  pdl_wait();
  pdl_launch_dependents();
  __syncthreads();
  const int S = a.geo.S, len = a.ctx_len[b];
  const long long owned = a.page_base[b + 1] - a.page_base[b];
  const int P = length_fits(a, len, owned) ? pages_of(len, S) : 0;
  // every selected page of the group's heads: kHold entries of a thread at a time, all loads ahead of their uses (4 heads with 256
  // pages: 6.1 us, one after the other 8.3); the first ones are kept for the second look
  const int k = a.geo.k, entries = a.geo.g * k;
  constexpr int kHold = 8, kNone = -1;
  auto pages_at = [&](int j0, int (&p)[kHold]) {
    int n[kHold];
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int j = j0 + i * 256 + tid, hh = j / k;
      const long long bh = (long long)b * a.geo.Hq + kv * a.geo.g + hh;
      n[i] = j < entries ? n_sel[bh] - (j - hh * k) : 0;      // > 0: the entry counts
      p[i] = j < entries ? sel[bh * k + (j - hh * k)] : kNone;
    }
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (n[i] <= 0) p[i] = kNone;
      else if (p[i] < 0 || p[i] >= P) { atomicOr(a.status, SWARM_DEV_BAD_PAGE); p[i] = kNone; }
  };
  auto mark = [&](const int (&p)[kHold]) {
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (p[i] != kNone) atomicOr(s_map + (p[i] >> 5), 1u << (p[i] & 31));
  };
  int held[kHold];
  pages_at(0, held);
  mark(held);
  for (int j0 = kHold * 256; j0 < entries; j0 += kHold * 256) {
    int p[kHold];
    pages_at(j0, p);
    mark(p);
  }
  __syncthreads();
  const int per = (words + 255) / 256, lo = min(words, tid * per), hi = min(words, lo + per);
  int mine = 0;
  for (int w = lo; w < hi; ++w) mine += __popc(s_map[w]);
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) s_sum[warp] = incl;
  __syncthreads();
  int at = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (w < warp) at += s_sum[w];
    total += s_sum[w];
  }
  int2* row = list + (long long)u * a.list_cap;
  for (int w = lo; w < hi; ++w) {
    s_before[w] = at;
    for (uint32_t bits = s_map[w]; bits != 0u; bits &= bits - 1u) row[at++] = make_int2(32 * w + __ffs(bits) - 1, 0);
  }
  __syncthreads();
  auto add_heads = [&](int j0, const int (&p)[kHold]) {
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (p[i] != kNone)
        atomicOr(reinterpret_cast<unsigned*>(&row[s_before[p[i] >> 5] + __popc(s_map[p[i] >> 5] & ((1u << (p[i] & 31)) - 1u))].y),
                 1u << ((j0 + i * 256 + tid) / k));
  };
  add_heads(0, held);
  for (int j0 = kHold * 256; j0 < entries; j0 += kHold * 256) {
    int p[kHold];
    pages_at(j0, p);
    add_heads(j0, p);
  }
  if (tid == 0) {
    const bool ends = P > 0 && ((s_map[(P - 1) >> 5] >> ((P - 1) & 31)) & 1u);
    list_tokens[u] = total * S - (ends ? max(0, P * S - len) : 0);
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn g_encode = nullptr;

// bf16 tensor of five dimensions, boxes of 64 coordinates with the 128-byte swizzle.  Strides in bytes.
cudaError_t make_map(CUtensorMap* map, const void* base, const cuuint64_t (&dims)[5], const cuuint64_t (&strides)[4], const cuuint32_t (&box)[5]) {
  if (g_encode == nullptr) return cudaErrorNotSupported;
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  const CUresult r = g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

constexpr int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct TreeLayout {
  int64_t part_o, part_ml, unit_first, unit_last, list, list_tokens, total;
  int list_cap;
};
int tile_tokens_of(const Geometry& geo) { return kTile / geo.g; }
int row_tiles_of(const Geometry& geo, int T) { return (T + tile_tokens_of(geo) - 1) / tile_tokens_of(geo); }
TreeLayout tree_layout(const Geometry& geo, int T) {
  TreeLayout l;
  const int64_t units = (int64_t)geo.B * geo.Hkv, tiles = row_tiles_of(geo, T);
  const int64_t rows = tiles > 1 ? 2 * kTile : kTile;
  const int64_t ctas = std::max<int64_t>(kMaxTreeCtas, (tiles + 1) / 2);
  l.list_cap = (int)std::min<int64_t>((int64_t)geo.g * geo.k, geo.Pmax);
  l.part_o = 0;
  l.part_ml = align256(l.part_o + ctas * 2 * rows * kHeadDim * 4);
  l.unit_first = align256(l.part_ml + ctas * 2 * rows * 8);
  l.unit_last = align256(l.unit_first + units * 4);
  l.list_tokens = align256(l.unit_last + units * 4);
  l.list = align256(l.list_tokens + units * 4);
  l.total = align256(l.list + units * l.list_cap * 8);
  return l;
}

}  // namespace

bool tree_supported(const Geometry& geo, int T, bool selected) {
  if (geo.g > kTile || (int64_t)T * geo.g >= (int64_t(1) << 30) || geo.n_pool_pages >= (int64_t(1) << 31) || (int64_t)geo.B * geo.Hkv * row_tiles_of(geo, T) * 32 >= (int64_t(1) << 31) ||
      (geo.n_pool_pages * geo.S / kTile + (int64_t)geo.B * (T / kTile + 2)) * geo.Hkv >= (int64_t(1) << 31))
    return false;
  return !selected || (geo.g <= 32 && (geo.Pmax + 31) / 32 * 8 <= kMaxTreeMapBytes);
}

long long tree_attn_workspace_bytes(const Geometry& geo, int T) { return tree_layout(geo, T).total; }

cudaError_t configure_tree() {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q);
  if (e != cudaSuccess || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  g_encode = reinterpret_cast<EncodeTiledFn>(p);
  e = cudaFuncSetAttribute(tree_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<false>::kBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_attn_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<true>::kBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(tree_list_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxTreeMapBytes);
  return e;
}

cudaError_t launch_tree_attn(const Geometry& geo, const TreeCall& c, void* workspace, uint32_t* status, cudaStream_t st) {
  const TreeLayout lay = tree_layout(geo, c.T);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  TreeArgs a{};
  a.geo = geo;
  a.q = c.q;
  a.page_base = c.page_base;
  a.ctx_len = c.ctx_len;
  a.n_draft = c.n_draft;
  a.mask = c.mask;
  a.T = c.T;
  a.words = (c.T + 31) / 32;
  a.part_o = reinterpret_cast<float4*>(ws + lay.part_o);
  a.tile_tokens = tile_tokens_of(geo);
  a.part_ml = reinterpret_cast<float2*>(ws + lay.part_ml);
  a.unit_first = reinterpret_cast<int32_t*>(ws + lay.unit_first);
  a.unit_last = reinterpret_cast<int32_t*>(ws + lay.unit_last);
  a.list_cap = lay.list_cap;
  a.out = c.out;
  a.lse = c.lse;
  a.status = status;

  const cuuint64_t row = kHeadDim * 2, S = (cuuint64_t)geo.S, Hkv = (cuuint64_t)geo.Hkv, T = (cuuint64_t)c.T;
  // pool: (64 coordinates, token of the page, page, half of the coordinates, KV head and K or V)
  CUtensorMap tile{}, page{}, half{}, dk, dv, dq;
  const cuuint64_t pool_dims[5] = {64, S, (cuuint64_t)geo.n_pool_pages, 2, Hkv * 2};
  const cuuint64_t pool_strides[4] = {row, Hkv * 2 * S * row, 128, S * row};
  const cuuint32_t tile_box[5] = {64, (cuuint32_t)S, (cuuint32_t)(kTile / S), 2, 1}, page_box[5] = {64, (cuuint32_t)S, 1, 2, 1},
                   half_box[5] = {64, (cuuint32_t)S, 1, 1, 1};
  cudaError_t e = cudaSuccess;                               // (each of these calls is host time in front of the launch)
  if (c.sel == nullptr) {
    e = make_map(&tile, c.kv_pool, pool_dims, pool_strides, tile_box);
  } else {
    e = make_map(&page, c.kv_pool, pool_dims, pool_strides, page_box);
    if (e == cudaSuccess) e = make_map(&half, c.kv_pool, pool_dims, pool_strides, half_box);
  }
  // drafted tokens: (64 coordinates, token, half of the coordinates, KV head, request)
  const cuuint64_t draft_dims[5] = {64, T, 2, Hkv, (cuuint64_t)geo.B};
  const cuuint64_t draft_strides[4] = {Hkv * row, 128, row, T * Hkv * row};
  const cuuint32_t draft_box[5] = {64, (cuuint32_t)kTile, 2, 1, 1};
  if (e == cudaSuccess) e = make_map(&dk, c.k, draft_dims, draft_strides, draft_box);
  if (e == cudaSuccess) e = make_map(&dv, c.v, draft_dims, draft_strides, draft_box);
  // queries: (128 coordinates, head of the group, token, KV head, request)
  const cuuint64_t q_dims[5] = {kHeadDim, (cuuint64_t)geo.g, T, Hkv, (cuuint64_t)geo.B};
  const cuuint64_t q_strides[4] = {row, (cuuint64_t)geo.Hq * row, (cuuint64_t)geo.g * row, T * (cuuint64_t)geo.Hq * row};
  const cuuint32_t q_box[5] = {64, (cuuint32_t)geo.g, (cuuint32_t)a.tile_tokens, 1, 1};
  if (e == cudaSuccess) e = make_map(&dq, c.q, q_dims, q_strides, q_box);
  if (e != cudaSuccess) return e;

  if (c.sel != nullptr) {
    int2* list = reinterpret_cast<int2*>(ws + lay.list);
    int32_t* tokens = reinterpret_cast<int32_t*>(ws + lay.list_tokens);
    a.list = list;
    a.list_tokens = tokens;
    e = launch_pdl(tree_list_kernel, dim3((unsigned)(geo.B * geo.Hkv)), dim3(256), (size_t)((geo.Pmax + 31) / 32) * 8, st, true, a, c.sel,
                   c.n_sel, list, tokens);
    if (e != cudaSuccess) return e;
  }
  const int tiles = row_tiles_of(geo, c.T);
  const bool wide = tiles > 1;
  a.row_blocks = (tiles + 1) / 2;
  const int64_t most = (int64_t)geo.B * geo.Hkv * (((int64_t)geo.Pmax * geo.S + kTile - 1) / kTile + (c.T + kTile - 1) / kTile);
  a.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(kMaxTreeCtas, sm_count()) / a.row_blocks, most));
  const unsigned grid = (unsigned)(a.chunks * a.row_blocks);
  e = wide ? launch_pdl(tree_attn_kernel<true>, dim3(grid), dim3(kThreads), (size_t)Layout<true>::kBytes, st, true, tile, page, half, dk, dv, dq, a)
           : launch_pdl(tree_attn_kernel<false>, dim3(grid), dim3(kThreads), (size_t)Layout<false>::kBytes, st, true, tile, page, half, dk, dv, dq, a);
  if (e != cudaSuccess) return e;
  const int groups = (std::min(c.T, a.tile_tokens) * geo.g + 31) / 32;
  // few units are cut into many parts: their partials are shared by the warps of a CTA
  const bool many = (int64_t)geo.B * geo.Hkv * 4 <= a.chunks;
  const dim3 merge_grid((unsigned)((int64_t)geo.B * geo.Hkv * tiles * groups * (many ? 8 : 1)));
  auto* merge = wide ? (many ? tree_merge_kernel<2, 8> : tree_merge_kernel<2, 1>) : (many ? tree_merge_kernel<1, 8> : tree_merge_kernel<1, 1>);
  return launch_pdl(merge, merge_grid, dim3(256), 0, st, true, a, groups, tiles);
}

}  // namespace swarm
