// Attention of a chunk of new tokens of every sequence over the paged, segmented (prompt | beacons | window) store.
//
// Item i of the batch brings m_i = cu_q[i + 1] - cu_q[i] query rows; row r sees the first first_i + r + 1 live entries
// of its sequence in logical order (all of them where there are fewer):
//     out[r, h] = softmax_j(sm_scale <q[r, h], K_j>) V_j,   j < min(first_i + r + 1, live_i),
// zeros where that is nothing.  That is the attention of a prompt chunk behind the entries stored before it, and of
// the last m_i entries of a window (several guessed tokens checked at once).
//
// k_chunk_attn runs on the tcgen05 tensor cores.  A thread block (one per SM) works on units of 256 query rows, two
// groups of floor(128 / G) tokens times the G query heads of a KV head, against tiles of 64 keys that both groups share:
// S = Q K^T into tensor memory, softmax by one thread per row, P as bf16 back into tensor memory, O += P V.  S of a group
// has two places, used in turn, so that the next tile's S is there when the rows have finished one.  Sharing K and V halves
// what a block reads: with a block per group the reads' latency was the bound (4 x 2048 rows over 8192 entries, 32 / 8 heads:
// 1.07 ms).  A unit with rows for one group only ("solo") belongs to one of the groups, taken in turn, so that one writes
// its results while the other begins.
//   * Keys come from pages.  The live entries lie in a virtual row space, prompt from 0, beacons and window each from
//     the next multiple of the copy height (of 8 at least), so that (row & 7) equals the entry's position in its segment modulo 8:
//     the store's chunk permutation IS the 128-byte swizzle of the product's operand layout, and unswizzled tensor
//     copies of up to 32 entries of one page (64 of the head's coordinates each) put a tile together, K and V alike.
//     The copy height R is the largest power of two up to that which divides the page size, so no copy crosses a page.
//   * The key tiles of all (sequence, KV head, query tile) units form one line that is cut into equal spans, one per
//     thread block, of at least 8 tiles, so that a large prompt chunk ends everywhere at the same time; where there are fewer
//     units than blocks, each unit is cut into equal pieces instead, of at least 8 tiles (joining pieces takes about as long as four
//     to eight tiles) and as many as its share of the blocks that are left over, at least one.  So equal units have a second piece
//     only while they are at most a third of the blocks, 49 on 148 SMs: calls of 50 to 147 equal units leave blocks without work, and
//     so do sequences that are much shorter than 8 tiles (20 prompts of 60 tokens, 8 KV heads: 20 blocks).  A unit that is cut
//     leaves unnormalised partial results (m, l, O) per row in the workspace, and the block that takes its last ticket joins them in
//     the order of the keys, sixteen at a time, so results do not depend on which block that is.
//   * Every block works the line out from the lengths on the device by itself: no host copy of a length, no plan
//     kernel, and the call can be captured.
//   * The copies, the products and the rows' softmax each have warps of their own, and the stream of tiles goes on across
//     units.
// Bounds.  At many rows per key: the round S -> softmax -> P -> product -> next S of each group, 1.1 us per pair of tiles, of which
// the tensor pipe is busy for 41 %, the exponential unit for 47 % and the issue slots for 43 % (4 x 1024 rows over 3024
// entries); with half the products left out the kernel gains 7 %, without exponentials 3 %.  At few rows: the reads of the cache (a tile is 32 KB of K
// and V for 4.2 MFLOP per group) and, below some 20 us, the steps from the launch to the first tile and from the last one to
// the joined result.  Measured, 32 / 8 heads of 128, pages of 16: 4 x 2048 rows over 8192 entries 0.88 ms in a short replay (1090
// TFLOP/s, 0.66 of the measured product rate), 1.05 ms per call in a run of a second, at lower clocks (920 TFLOP/s); 64 x 5 rows over
// 585 entries 46 us (3.3 TB/s); 64 single rows over 2000 99 us (5.3 TB/s).
// 12 / 2 heads: one row over 100,000 entries 38 us (2.7 TB/s), 13 rows over 512 15 us.  Tried on the large chunk (0.88 ms): a
// quarter of the exponentials as polynomials on the ordinary pipes 0.93; one lane that waits and issues by itself, without votes,
// 0.99 (its operands are no longer uniform over the warp); a warp of its own for each of the two products 0.94; the rows' loop
// rehearsed before the first tile, so that its instructions are there, 0.97.
//
// Entries that no row of a query tile can see are not read into a product: their scores are overwritten with -inf, and
// V rows that are past the last visible entry of the tile are cleared in shared memory, so that whatever the
// pool holds there (it is never initialised) cannot reach a result.  Every wait is bounded; on expiry the block
// records BC_ERR_TIMEOUT, waits for what it has in flight, releases its tensor memory and returns.
//
// k_chunk_reference is the simple form behind BC_FLAG_ATTN_REFERENCE: one warp per query row and head.
#include <cuda.h>

#include "bc_common.cuh"

namespace {

#include "bc_tc.cuh"
#include "bc_book_device.cuh"

constexpr int kGroup = 128;                    // rows, and row threads, of a group
constexpr int kThreads = 2 * kGroup + 128;     // two groups, a product warp for each and two copy warps
constexpr int kKeys = 64;                      // keys per tile
constexpr int kMaxItems = BC_MAX_ATTN_BATCH;
constexpr int kTmemColumns = 512;              // S and O; what is allocated and what is given back

// ---- the simple form -----------------------------------------------------------------------------------------------
// item of packed row `row`: the largest i with cu[i] <= row; false if the row belongs to none
__device__ __forceinline__ bool find_item(const int32_t* cu, int n, int row, int* item) {
  int lo = 0, hi = n;
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (cu[mid] <= row) lo = mid; else hi = mid; }
  *item = lo;
  return cu[lo] <= row && row < cu[lo + 1];
}

__global__ void k_chunk_reference(BcMeta m, BcGeom g, BcChunkArgs a) {
  const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  const int D = g.head_dim, per = D / 32, kvh = h / (g.q_heads / g.kv_heads);
  int i;
  if (!find_item(a.cu_q, a.n, row, &i)) return;
  const int slot = a.slots[i], len = a.cu_q[i + 1] - a.cu_q[i];
  int P = 0, nb = 0, w = 0;
  if (slot >= 0 && slot < m.max_seqs && m.open[slot]) { P = m.prompt_len[slot]; nb = m.n_beacons[slot]; w = m.window_len[slot]; }
  const int live = P + nb + w;
  const long long first = a.first != nullptr ? a.first[i] : live - len;
  const long long vis = min((long long)live, max(0ll, first + (row - a.cu_q[i]) + 1));
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q) + ((int64_t)row * g.q_heads + h) * D;
  float qv[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int e = 0; e < per; ++e) qv[e] = __bfloat162float(q[lane * per + e]);
  float mrun = -INFINITY, lrun = 0.f;
  for (int e = 0; e < (int)vis; ++e) {
    int pos, col;
    if (e < P) { pos = e; col = 0; }
    else if (e < P + nb) { pos = e - P; col = m.beacon_off[slot]; }
    else { pos = e - P - nb; col = m.window_off[slot]; }
    col += pos / g.page_size;
    int page = 0;
    if (!m.debug || (unsigned)col < (unsigned)m.max_pages_per_seq) page = m.page_table[(int64_t)slot * m.max_pages_per_seq + col];
    if (m.debug && (unsigned)page >= (unsigned)m.num_pages) page = 0;
    const uint8_t* at = a.pool_layer + ((int64_t)page * g.page_size + pos % g.page_size) * g.entry_bytes;
    const __nv_bfloat16* kp = reinterpret_cast<const __nv_bfloat16*>(at + kvh * g.head_row_bytes);
    const __nv_bfloat16* vp = reinterpret_cast<const __nv_bfloat16*>(at + (g.kv_heads + kvh) * g.head_row_bytes);
    float dot = 0.f, vv[4];
    for (int x = 0; x < per; ++x) {
      const int d = lane * per + x, idx = (((d >> 3) ^ (pos & 7)) << 3) + (d & 7);
      dot += qv[x] * __bfloat162float(kp[idx]);
      vv[x] = __bfloat162float(vp[idx]);
    }
    for (int s = 16; s; s >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, s);
    const float sc = dot * a.sm_scale;
    const float mn = fmaxf(mrun, sc);
    const float al = expf(mrun - mn), pe = expf(sc - mn);
    lrun = lrun * al + pe;
    for (int x = 0; x < per; ++x) acc[x] = acc[x] * al + pe * vv[x];
    mrun = mn;
  }
  for (int x = 0; x < per; ++x) {
    const float val = lrun > 0.f ? acc[x] / lrun : 0.f;
    const int64_t o = ((int64_t)row * g.q_heads + h) * D + lane * per + x;
    if (a.out_f32) reinterpret_cast<float*>(a.out)[o] = val;
    else reinterpret_cast<__nv_bfloat16*>(a.out)[o] = __float2bfloat16_rn(val);
  }
}

// n / d for 0 <= n < 2^31 by a product and a shift: mul = floor(2^32 (2^l - d) / d) + 1 with l = ceil(log2 d) (Granlund and
// Montgomery's round-up method).
struct FastDiv {
  uint32_t mul, shift1, shift2;
  __device__ __forceinline__ int operator()(int n) const {
    const uint32_t t = __umulhi(mul, (uint32_t)n);
    return (int)((t + (((uint32_t)n - t) >> shift1)) >> shift2);
  }
};
FastDiv make_fast_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return {d > 1 ? (uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1) : 1u, l > 0 ? 1u : 0u, l > 0 ? l - 1 : 0u};
}

// ---- the tensor-core form ------------------------------------------------------------------------------------------
struct ChunkParams {
  BcMeta m;
  const int32_t *slots, *first, *cu_q;
  int32_t n, total_q;
  void* out;
  int32_t out_f32, layer, entry_bytes;
  const uint8_t* pool_layer;
  float* part_o;      // [2 grid][2 groups][D / 4][128] float4: a block's partial results, slot 0 continues a unit, slot 1 begins one
  float* part_ml;     // [2 grid][2 groups][2][128]
  // [3][BC_MAX_CHUNK_CTAS][2 groups], zero between launches.  Sixteen pieces count themselves at the block of their first one, in row
  // 0 where that one begins the unit and in row 1 where it continues it (a block has one of either kind at most); row 2: the
  // sixteens of a unit.
  int32_t* tickets;
  int32_t Hq, Hkv, G, page_size;
  FastDiv by_page;
  int32_t half;       // tokens of a group: 128 / G
  int32_t tokens;     // of a unit: two groups
  int32_t R;          // entries per copy: 4, 8, 16 or 32, or 1 (row by row)
  int32_t align;      // segment starts in the virtual row space: max(8, R)
  int32_t min_shift;  // log2 of the key tiles of a piece, at least
  uint32_t wait_limit;
  float scale_log2;
};

// Lengths of the items, in shared memory (structure of arrays).
struct Items {
  int m[kMaxItems], first[kMaxItems], P[kMaxItems], nb[kMaxItems], w[kMaxItems];
  long long before[kMaxItems + 1];   // key tiles of one KV head in the items before
  int large[64], n_large;            // items whose tiles all threads count together
  long long total, units, span;      // weight of the line, number of units, weight per block
  int item0, head0, tile0, n0, tiles;   // where this block's span begins, and its tiles
  int b0, pieces;                    // where units are cut into pieces: first block and number of pieces of this block's unit
};

// One unit: the query tile `t` (two groups) of item `i` for KV head `h`, and the key tiles [n0, n1) of its N that this block does.
struct Unit {
  int i, h, t;
  int count, vis_last;     // tokens in the tile; entries its last token sees
  int P, nb, w, base;      // lengths of the sequence; base: entries the tile's first token sees, minus 1
  int n0, n1, N;
  int solo;                // -1: rows for both groups; else the group that has the rows
};
// Entries `vis` of a sequence as intervals of the virtual row space: [0, p), [b0, b0 + b), [w0, w0 + w).
struct Seen {
  int p, b0, b, w0, w;
};
__device__ __forceinline__ Seen seen_of(int vis, int P, int nb, int w, int align) {
  Seen s;
  s.b0 = (P + align - 1) & -align;
  s.w0 = s.b0 + ((nb + align - 1) & -align);
  s.p = min(vis, P);
  s.b = min(max(vis - P, 0), nb);
  s.w = min(max(vis - P - nb, 0), w);
  return s;
}
__device__ __forceinline__ int virtual_end(const Seen& s) { return s.w > 0 ? s.w0 + s.w : (s.b > 0 ? s.b0 + s.b : s.p); }
__device__ __forceinline__ int clamp_vis(int first, int r, int live) {   // entries that row r of an item sees
  return (int)min((long long)live, max(0ll, (long long)first + r + 1));
}
__device__ __forceinline__ int key_tiles(const Items& it, int i, int t, int tokens, int align) {
  const int last = min((t + 1) * tokens, it.m[i]) - 1;
  const int vis = clamp_vis(it.first[i], last, it.P[i] + it.nb[i] + it.w[i]);
  return max(1, (virtual_end(seen_of(vis, it.P[i], it.nb[i], it.w[i], align)) + kKeys - 1) / kKeys);
}
__device__ __forceinline__ Unit make_unit(const Items& it, int i, int h, int t, int n0, long long left, int tokens, int align, int solo) {
  Unit u;
  u.i = i; u.h = h; u.t = t; u.n0 = n0;
  u.P = it.P[i]; u.nb = it.nb[i]; u.w = it.w[i];
  u.count = min(tokens, it.m[i] - t * tokens);
  const int live = u.P + u.nb + u.w;
  u.vis_last = clamp_vis(it.first[i], t * tokens + u.count - 1, live);
  u.base = it.first[i] + t * tokens;
  u.N = key_tiles(it, i, t, tokens, align);
  u.n1 = (int)min((long long)u.N, n0 + left);
  u.solo = 2 * u.count > tokens ? -1 : solo;
  return u;
}
// The unit behind u on the line (there is one: the caller knows how many key tiles are left).
__device__ __forceinline__ Unit next_unit(const Items& it, const Unit& u, long long left, int Hkv, int tokens, int align) {
  int i = u.i, h = u.h, t = u.t + 1;
  if (t * tokens >= it.m[i]) {
    t = 0;
    if (++h == Hkv) {
      h = 0;
      do ++i; while (it.m[i] == 0);
    }
  }
  return make_unit(it, i, h, t, 0, left, tokens, align, u.solo < 0 ? 0 : u.solo ^ 1);
}

// the tile at k0 lies in one interval entirely
__device__ __forceinline__ bool inside(const Seen& s, int k0) {
  return k0 + kKeys <= s.p || (k0 >= s.b0 && k0 + kKeys <= s.b0 + s.b) || (k0 >= s.w0 && k0 + kKeys <= s.w0 + s.w);
}
// 64-bit mask (bit j of word j / 32: column j of the tile) of the tile's columns inside [lo, hi) of the virtual space
__device__ __forceinline__ void add_range(uint32_t (&mask)[2], int lo, int hi) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int l = min(max(lo - 32 * q, 0), 32), e = min(max(hi - 32 * q, 0), 32);
    if (e > l) mask[q] |= (e - l == 32 ? 0xffffffffu : ((1u << (e - l)) - 1u)) << l;
  }
}
__device__ __forceinline__ void tile_mask(uint32_t (&mask)[2], const Seen& s, int k0) {
  mask[0] = mask[1] = 0;
  add_range(mask, -k0, s.p - k0);
  add_range(mask, s.b0 - k0, s.b0 + s.b - k0);
  add_range(mask, s.w0 - k0, s.w0 + s.w - k0);
}

// What a copy warp needs to issue a tile's copies.  Lane l holds the copies l, l + 32, ... of the tile's 64 / R.
template <int KP>
struct TileIssue {
  int page[KP], rem[KP];     // page id and first entry inside the page
  uint32_t valid[KP];        // ballots: which copies there are
  int h, qrow, solo;         // KV head; packed row of the unit's first token; the unit's group
  bool fresh;                // the unit's first tile here
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <int N>
struct Width { static constexpr int value = N; };

__device__ __forceinline__ void tma_pool(uint32_t dst, const CUtensorMap* map, int head_half, int row, int layer, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(0), "r"(head_half), "r"(row), "r"(layer), "r"(bar)
      : "memory");
}

// Shared memory of a block: the groups' Q, the rings of K and V, the items.
template <int D>
struct Smem {
  static constexpr int kStages = D == 64 ? 8 : 4;
  static constexpr int kHalves = D / 64;
  static constexpr int kQHalf = kTile * 128;                // 128 rows of 64 coordinates
  static constexpr int kHalf = kKeys * 128;                 // 64 rows of 64 coordinates
  static constexpr int kQ = kHalves * kQHalf;
  static constexpr int kOperand = kHalves * kHalf;
  static constexpr int kBytes = 2 * kQ + 2 * kStages * kOperand + 1024 + (int)sizeof(Items);
};

// D: head_dim.  ROWS: the page size is no multiple of 4: a tensor copy would hold one entry or two, and a warp issues one in some
// 70 cycles, so the copy warp's lanes copy the rows 16 bytes each.  2048 rows over 8192 entries, 32 / 8 heads, by rows and by tensor
// copies: pages of 2 0.40 and 0.52 ms, of 4 0.40 and 0.33, of 8 0.40 and 0.25.
//
// Roles: warps 0 .. 3 are group 0's row threads, warps 4 .. 7 group 1's, warps 8 and 9 issue the products of the two groups,
// warp 10 the copies of Q and K, warp 11 those of V.
// S of a group's tile t + 2 is issued right behind the product with P of its tile t, whose place it takes: one thread issues
// both, and they run in that order.
// Barriers (single-phase mbarriers, parity = completions & 1), [g] per group, t counting the group's own tiles:
//   bar_kin[s], bar_vin[s]: K, V of ring buffer s have landed     bar_ke[s], bar_ve[s]: both groups are done with them
//     Both product warps wait for every K and V, also for what only the other group multiplies with, and then say so: a parity
//     tells two completions apart and no more, so no waiter may fall behind or skip one.
//   bar_q[g]: Q of the group's unit has landed                    bar_qe[g]: it has been read
//   bar_s[g][t & 1]: S of tile t is ready                         bar_p[g][t & 1]: the 128 row threads have stored its P
//   bar_o[g][t & 1]: the product with P of tile t is done         bar_f[g]: O of the unit is final
//   bar_e[g]: the rows have read O                                bar_r[g]: the row threads among themselves (bounded, unlike
//                                                                 a block barrier)
template <int D, bool ROWS, bool SHORTW>
__global__ void __launch_bounds__(kThreads, 1) k_chunk_attn(const ChunkParams a, const __grid_constant__ CUtensorMap q_map,
                                                           const __grid_constant__ CUtensorMap pool_map) {
  constexpr int KP = ROWS ? 2 : 1;                          // copies per lane, tensor and tile
  constexpr int kHalves = Smem<D>::kHalves, kHalf = Smem<D>::kHalf, kQ = Smem<D>::kQ, kQHalf = Smem<D>::kQHalf, kOperand = Smem<D>::kOperand, kStages = Smem<D>::kStages;
  constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kKeys >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
  constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sQ = smem_addr(smem), sK = sQ + 2 * kQ, sV = sK + kStages * kOperand;
  Items& it = *reinterpret_cast<Items*>(smem + 2 * kQ + 2 * kStages * kOperand);
  __shared__ __align__(8) uint64_t s_bars[4 * kStages + 24];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail_word, s_ticket[2];
  volatile int* s_fail = &s_fail_word;
  const uint32_t bars = smem_addr(s_bars);
  const uint32_t bar_kin = bars, bar_vin = bars + 8 * kStages, bar_ke = bars + 16 * kStages, bar_ve = bars + 24 * kStages, bar_q = bars + 32 * kStages,
                 bar_qe = bar_q + 16, bar_s = bar_q + 32, bar_o = bar_q + 64, bar_f = bar_q + 96, bar_d = bar_q + 112, bar_p = bar_q + 128,
                 bar_e = bar_q + 160, bar_r = bar_q + 176;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.G, Hq = a.Hq, Hkv = a.Hkv, half = a.half, tokens = a.tokens, align = a.align;

  if (tid == 0) {
    auto init = [&](uint32_t bar, int count, uint32_t arrivals) {
      for (int i = 0; i < count; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar + i * 8), "r"(arrivals) : "memory");
    };
    init(bar_kin, 2 * kStages, 1); init(bar_ke, 2 * kStages, 2);
    init(bar_q, 16, 1);                                     // q, qe (two each), s, o (four each), f, d (two each)
    init(bar_p, 8, kGroup);                                 // p (four), e, r (two each)
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    *s_fail = 0;
  }

  // ---- the line: every item's lengths, its key tiles per KV head, and where this block's span begins ------------------
  for (int i = tid; i < a.n; i += kThreads) {
    const int slot = a.slots[i], c0 = a.cu_q[i], c1 = a.cu_q[i + 1];
    int P = 0, nb = 0, w = 0;
    if (slot >= 0 && slot < a.m.max_seqs && a.m.open[slot]) { P = a.m.prompt_len[slot]; nb = a.m.n_beacons[slot]; w = a.m.window_len[slot]; }
    const int m = c0 < 0 || c0 > a.total_q ? 0 : max(0, min(c1, a.total_q) - c0);
    const int first = a.first != nullptr ? a.first[i] : P + nb + w - m;
    it.m[i] = m; it.first[i] = min(max(first, -(1 << 30)), 1 << 30); it.P[i] = P; it.nb[i] = nb; it.w[i] = w;
  }
  // Pieces of a unit of N tiles, where units are fewer than blocks; share: blocks left over per key tile.  (Together at most as many as
  // blocks: a piece each, or the unit's share of the blocks left over, rounded down, where that is more.)
  auto pieces_of = [&](int N, float share) { return max(1, min(N >> a.min_shift, (int)((float)N * share))); };
  // First before[i + 1] = the key tiles of one KV head in the items up to i; then, where there are fewer units than blocks, the
  // same in pieces (one loop for both: its instructions come from memory in most calls).
  bool by_unit = false;                                      // every block has (at most) one piece of one unit
  float share = 0.f;
#pragma unroll 1
  for (;;) {
    auto weight = [&](int i, int t) {
      const int N = key_tiles(it, i, t, tokens, align);
      return by_unit ? pieces_of(N, share) : N;
    };
    if (tid == 0) it.n_large = 0;
    __syncthreads();
    for (int i = tid; i < a.n; i += kThreads) {
      const int tiles = (it.m[i] + tokens - 1) / tokens;
      long long cost = 0;
      bool mine = true;
      if (tiles > 8) {                                      // a long chunk: counted by all threads below
        const int at = atomicAdd(&it.n_large, 1);
        if (at < 64) { it.large[at] = i; mine = false; }
      }
      if (mine)
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) cost += weight(i, t);
      it.before[i + 1] = cost;
    }
    __syncthreads();
    const int n_large = min(it.n_large, 64);
#pragma unroll 1
    for (int x = 0; x < n_large; ++x) {
      const int i = it.large[x], tiles = (it.m[i] + tokens - 1) / tokens;
      long long cost = 0;
#pragma unroll 1
      for (int t = tid; t < tiles; t += kThreads) cost += weight(i, t);
      atomicAdd(reinterpret_cast<unsigned long long*>(&it.before[i + 1]), (unsigned long long)cost);
    }
    if (n_large) __syncthreads();
    if (warp == 0) {
      long long carry = 0, tiles = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < a.n; i0 += 32) {
        const int i = i0 + lane;
        long long x = i < a.n ? it.before[i + 1] : 0;
        if (i < a.n) tiles += (it.m[i] + tokens - 1) / tokens;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long y = __shfl_up_sync(0xffffffffu, x, d);
          if (lane >= d) x += y;
        }
        if (i < a.n) it.before[i + 1] = carry + x;
        carry += __shfl_sync(0xffffffffu, x, 31);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
      if (lane == 0) { it.before[0] = 0; it.total = carry * Hkv; it.units = tiles * Hkv; }
    }
    __syncthreads();
    if (by_unit || it.units >= (long long)gridDim.x || it.total == 0) break;
    by_unit = true;
    // blocks left over per key tile, a little less so that the rounding cannot hand out one block too many
    share = (float)((long long)gridDim.x - it.units) / (float)it.total * 0.9999f;
    __syncthreads();                                        // it.total has been read
  }
  if (warp == 0) {
    const long long total = it.total;
    long long span = 1;
    if (!by_unit) {
      span = (total + gridDim.x - 1) / gridDim.x;
      if (span < (1 << a.min_shift)) span = 1 << a.min_shift;
    }
    const long long x0 = (long long)blockIdx.x * span;
    if (x0 < total) {
      int lo = 0, hi = a.n;                                 // the item: largest i with before[i] * Hkv <= x0 (a non-empty one)
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (it.before[mid] * Hkv <= x0) lo = mid; else hi = mid; }
      const long long cost = it.before[lo + 1] - it.before[lo], rest = x0 - it.before[lo] * Hkv;
      const int head = (int)(rest / cost);
      long long in_head = rest - head * cost;
      int t = 0;                                            // the query tile: 32 at a time
      for (;; t += 32) {
        const int tt = t + lane;
        int x = 0;
        if (tt * tokens < it.m[lo]) {
          x = key_tiles(it, lo, tt, tokens, align);
          if (by_unit) x = pieces_of(x, share);
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, d);
          if (lane >= d) x += y;
        }
        const uint32_t over = __ballot_sync(0xffffffffu, x > in_head);
        if (over) {
          const int l = __ffs(over) - 1;
          const int before = __shfl_sync(0xffffffffu, x, l > 0 ? l - 1 : 0);
          t += l;
          if (l > 0) in_head -= before;
          break;
        }
        in_head -= __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) {
        it.item0 = lo; it.head0 = head; it.tile0 = t; it.n0 = (int)in_head;
        it.tiles = (int)min(span, total - x0);
        if (by_unit) {                                      // piece number in_head of the unit's `pieces`
          const int N = key_tiles(it, lo, t, tokens, align), c = pieces_of(N, share);
          it.n0 = (int)(in_head * N / c);
          it.tiles = (int)((in_head + 1) * N / c) - it.n0;
          it.pieces = c;
          it.b0 = (int)(blockIdx.x - in_head);
        }
      }
    } else if (lane == 0) {
      it.tiles = 0;
    }
    if (lane == 0) it.span = span;
  }
  __syncthreads();
  const long long x_begin = (long long)blockIdx.x * it.span;  // by_unit: a number without a meaning on the line
  const long long x_end = x_begin + it.tiles;
  if (it.tiles == 0) return;                                // nothing to do: no tensor memory has been taken yet

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(kTmemColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // Rows of the Q buffers that no tensor copy writes (only when G does not divide 128) stay zero.
  const int box_rows = half * G;
  for (int idx = tid; idx < 2 * (kTile - box_rows) * (D / 8); idx += kThreads) {
    const int r = idx / (D / 8), g = r >= kTile - box_rows ? 1 : 0;
    st_zero16(sQ + g * kQ + swz(box_rows + r - g * (kTile - box_rows), idx % (D / 8)));
  }
  proxy_fence();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  // columns: S (then P, in its first 32) of the groups at 0 and 64, 128 and 192, O at 256 and 256 + D
  const Unit u0 = make_unit(it, it.item0, it.head0, it.tile0, it.n0, x_end - x_begin, tokens, align, 0);

  auto wait_all = [&](uint32_t bar, uint32_t parity) {       // every lane polls, a vote joins the answers
    if (!SHORTW && __all_sync(0xffffffffu, mbar_try(bar, parity))) return true;   // mostly so: without the loop's counts and exits
    const bool ok1 = mbar_wait_or_fail<SHORTW>(bar, parity, s_fail, a.wait_limit);
    return (bool)__all_sync(0xffffffffu, ok1);
  };
  if (warp > 2 * kGroup / 32 + 1) {
    // ======================================== copy warps ============================================
    // The first one copies Q and the K tiles, the second one the V tiles.
    const int which = warp - 2 * kGroup / 32 - 2;
    const int R = a.R, copies = kKeys / R;
    // cursor of the look-ahead: the tile whose copies are worked out next
    Unit lu = u0;
    int ln = u0.n0;
    long long lx = x_begin;                                 // position of (lu, ln) on the line
    bool fresh = true;                                      // lu has changed
    const int32_t* table = nullptr;
    int boff = 0, woff = 0;
    Seen lseen = {};
    auto look = [&]() {                                     // the tile at the cursor; the page ids' loads are left in flight
      TileIssue<KP> ti;
      ti.fresh = fresh;
      if (fresh) {
        // of a slot that is not open no entry is seen: no copy is valid and nothing below is read
        if (lu.vis_last > 0) {
          const int seq = a.slots[lu.i];
          table = a.m.page_table + (int64_t)seq * a.m.max_pages_per_seq;
          if (lu.vis_last > lu.P) { boff = a.m.beacon_off[seq]; woff = a.m.window_off[seq]; }
        }
        lseen = seen_of(lu.vis_last, lu.P, lu.nb, lu.w, align);
        ti.qrow = a.cu_q[lu.i] + lu.t * tokens;
        ti.solo = lu.solo;
        fresh = false;
      }
      ti.h = lu.h;
#pragma unroll
      for (int c = 0; c < KP; ++c) {
        const int p = lane + 32 * c, v = ln * kKeys + p * R;   // first virtual row of the copy
        int pos = -1, col = 0;
        if (p < copies) {
          if (v < lseen.p) pos = v;
          else if (v >= lseen.b0 && v < lseen.b0 + lseen.b) { pos = v - lseen.b0; col = boff; }
          else if (v >= lseen.w0 && v < lseen.w0 + lseen.w) { pos = v - lseen.w0; col = woff; }
        }
        ti.valid[c] = __ballot_sync(0xffffffffu, pos >= 0);
        ti.page[c] = 0; ti.rem[c] = 0;
        if (pos >= 0) {
          const int pg = a.by_page(pos);
          col += pg;
          ti.rem[c] = pos - pg * a.page_size;
          if (a.m.debug && (unsigned)col >= (unsigned)a.m.max_pages_per_seq) { debug_note(a.m, col); col = 0; }
          ti.page[c] = table[col];
        }
      }
      ++lx;
      if (++ln == lu.n1 && lx < x_end) {
        lu = next_unit(it, lu, x_end - lx, Hkv, tokens, align);
        ln = lu.n0;
        fresh = true;
      }
      return ti;
    };
    const uint32_t ring = which ? sV : sK, bar_in = which ? bar_vin : bar_kin, bar_read = which ? bar_ve : bar_ke;
    auto issue = [&](const TileIssue<KP>& ti, int slot) {       // a tile into ring buffer `slot`
      const uint32_t dst = ring + slot * kOperand, bar = bar_in + slot * 8;
      if constexpr (ROWS) {
        constexpr int kPieces = D / 8, kRows = 32 / kPieces;     // 16-byte pieces of a row, rows per instruction
        const int piece = lane % kPieces;
        const uint8_t* src = a.pool_layer + (int64_t)(which * Hkv + ti.h) * (D * 2) + piece * 16;
        const uint32_t at = dst + (piece >> 3) * kHalf + (piece & 7) * 16;
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          int page = ti.page[k];
          if (a.m.debug && (ti.valid[k] >> lane & 1) && (unsigned)page >= (unsigned)a.m.num_pages) { debug_note(a.m, page); page = 0; }
          const int own = page * a.page_size + ti.rem[k];        // pool row of the tile's row 32 k + lane
#pragma unroll 4
          for (int i = 0; i < 32 / kRows; ++i) {
            const int r = i * kRows + lane / kPieces, from = __shfl_sync(0xffffffffu, own, r);
            if (ti.valid[k] >> r & 1) cp_async16(at + (32 * k + r) * 128, src + (int64_t)from * a.entry_bytes);
          }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        proxy_fence();   // the product reads shared memory through the asynchronous proxy
        __syncwarp();
        if (elect_one()) mbar_arrive_cta(bar);
      } else {
        if (elect_one()) mbar_expect_tx(bar, (uint32_t)(__popc(ti.valid[0]) * R * D * 2));
        __syncwarp();
        if (ti.valid[0] >> lane & 1) {
          int page = ti.page[0];
          if (a.m.debug && (unsigned)page >= (unsigned)a.m.num_pages) { debug_note(a.m, page); page = 0; }
#pragma unroll
          for (int s = 0; s < kHalves; ++s)
            tma_pool(dst + s * kHalf + lane * R * 128, &pool_map, (which * Hkv + ti.h) * kHalves + s, page * a.page_size + ti.rem[0], a.layer, bar);
        }
      }
      __syncwarp();
    };
    const uint32_t T = (uint32_t)(x_end - x_begin);          // tiles of the span (far below 2^31)
    uint32_t issued = 0, nq[2] = {0, 0};                      // copies of tiles and of the groups' Q issued so far
    bool ok = true;
    TileIssue<KP> ti = look();
    for (uint32_t j = 0; j < T; ++j) {
      const int slot = (int)(j % kStages);
      if (which == 0 && ti.fresh) {                            // the unit's Q, once the groups' last ones have been read
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (!ok || (ti.solo >= 0 && ti.solo != g)) continue;
          if (nq[g] > 0) ok = wait_all(bar_qe + g * 8, (nq[g] - 1) & 1u);
          if (ok && elect_one()) {
            mbar_expect_tx(bar_q + g * 8, (uint32_t)(box_rows * D * 2));
#pragma unroll
            for (int s = 0; s < kHalves; ++s)
              tma_3d(sQ + g * kQ + s * kQHalf, &q_map, s * 64, ti.h * G, ti.qrow + (ti.solo < 0 ? g * half : 0), bar_q + g * 8);
          }
          __syncwarp();
          if (ok) ++nq[g];
        }
        if (!ok) break;
      }
      if (j >= (uint32_t)kStages) ok = wait_all(bar_read + slot * 8, (j / kStages - 1) & 1u);   // the buffer's last tile has been read
      if (!ok) break;
      issue(ti, slot); ++issued;
      if (j + 1 < T) ti = look();                              // its page ids arrive while the warp waits for the next buffer
    }
    // No copy may still be on its way into this block's shared memory when the block leaves, whichever warp gives up and when.
    // Wait, with the full limit, for the last copy into every buffer (tile s + kStages * j is copy j of buffer s).
    if (!ok) *s_fail = 1;
    __syncwarp();
    if (elect_one()) {
      int never = 0;
#pragma unroll
      for (int g = 0; g < 2; ++g)
        if (nq[g] > 0) mbar_wait_or_fail<false>(bar_q + g * 8, (nq[g] - 1) & 1u, &never, kWaitLimit);
#pragma unroll 1
      for (uint32_t s = 0; s < (uint32_t)kStages; ++s)
        if (issued > s) mbar_wait_or_fail<false>(bar_in + s * 8, ((issued - 1 - s) / kStages) & 1u, &never, kWaitLimit);
    }
    __syncwarp();
  } else if (warp >= 2 * kGroup / 32) {
    // ======================================== product warps =========================================
    // All 32 lanes walk the loop and the waits together; one elected lane issues the products.
    const int g = warp - 2 * kGroup / 32;
    const uint64_t dQ = umma_desc(sQ + g * kQ), dK = umma_desc(sK), dV = umma_desc_nmajor(sV, kHalf);
    const uint32_t tS = tmem + g * 2 * kKeys, tO = tmem + 4 * kKeys + g * D;
    const uint32_t T = (uint32_t)(x_end - x_begin);
    Unit u = u0;
    uint32_t j0 = 0, t = 0, units = 0;                          // the unit's first tile in the block's stream; tiles and units of this group so far
    bool ok = true, products = false;
    while (ok) {
      const int tiles = u.n1 - u.n0;
      if (u.solo < 0 || u.solo == g) {
        const Seen seen = seen_of(u.vis_last, u.P, u.nb, u.w, align);
        auto k_in = [&](int d) { const uint32_t j = j0 + (uint32_t)d; return wait_all(bar_kin + (j % kStages) * 8, (j / kStages) & 1u); };
        auto qk = [&](int d) {                                  // one lane: S of the unit's tile d, the group's tile t + d
          const uint32_t place = (t + (uint32_t)d) & 1u, slot = (j0 + (uint32_t)d) % kStages;
          const uint64_t k = dK + (uint64_t)(slot * kOperand >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)                   // descriptor start addresses advance in 16-byte units
            umma<kIdescQK>(tS + place * kKeys, dQ + (uint64_t)(((kk >> 2) * kQHalf + (kk & 3) * 32) >> 4),
                           k + (uint64_t)(((kk >> 2) * kHalf + (kk & 3) * 32) >> 4), kk > 0);
          umma_commit(bar_s + g * 16 + place * 8);
          umma_commit(bar_ke + slot * 8);
          if (d + 1 == tiles) umma_commit(bar_qe + g * 8);
        };
        ok = wait_all(bar_q + g * 8, units & 1u);
#pragma unroll 1
        for (int d = 0; ok && d < min(tiles, 2); ++d) {
          ok = k_in(d);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) qk(d);
          __syncwarp();
          products = true;
        }
        for (int d = 0; ok && d < tiles; ++d) {
          const uint32_t j = j0 + (uint32_t)d, at = t + (uint32_t)d, place = at & 1u;
          const int slot = (int)(j % kStages);
          // all that the two products need but P, so that they follow P without another wait
          ok = wait_all(bar_vin + slot * 8, (j / kStages) & 1u);
          if (d + 2 < tiles) ok = ok && k_in(d + 2);
          if (!ok) break;
          // V rows of the tile that hold no entry the unit can see (unwritten entries of the last page, gaps between
          // segments, rows that no copy wrote) are cleared, since a weight of 0 does not cancel a NaN.  In a unit with two groups
          // both clear them: neither may begin before they are clear, and zeros over zeros change nothing.
          const int k0 = (u.n0 + d) * kKeys;
          if (!inside(seen, k0)) {
            const uint32_t dst = sV + slot * kOperand;
            auto clear = [&](int from, int to) {                // rows of the virtual space
              from = max(from - k0, 0); to = min(to - k0, kKeys);
#pragma unroll
              for (int s = 0; s < kHalves; ++s)
#pragma unroll 4
                for (int b = from * 128 + lane * 16; b < to * 128; b += 512) st_zero16(dst + s * kHalf + b);
            };
            clear(seen.p, seen.b > 0 ? seen.b0 : (seen.w > 0 ? seen.w0 : k0 + kKeys));
            if (seen.b > 0) clear(seen.b0 + seen.b, seen.w > 0 ? seen.w0 : k0 + kKeys);
            if (seen.w > 0) clear(seen.w0 + seen.w, k0 + kKeys);
            proxy_fence();   // the product reads shared memory through the asynchronous proxy
            __syncwarp();
          }
          if (d == 0 && units > 0) ok = wait_all(bar_e + g * 8, (units - 1) & 1u);   // the rows have read the last unit's O
          ok = ok && wait_all(bar_p + g * 16 + place * 8, (at >> 1) & 1u);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t v = dV + (uint64_t)(slot * kOperand >> 4);
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk)             // 16 keys at a time
              umma_ts<kIdescPV>(tO, tS + place * kKeys + (uint32_t)(kk * 8), v + (uint64_t)((kk * 16 * 128) >> 4), (d > 0 || kk > 0) ? 1u : 0u);
            umma_commit(bar_o + g * 16 + place * 8);
            umma_commit(bar_ve + slot * 8);
            if (d + 1 == tiles) umma_commit(bar_f + g * 8);     // the last one: the block leaves behind it
            if (d + 2 < tiles) qk(d + 2);
          }
          __syncwarp();
        }
        t += (uint32_t)tiles;
        ++units;
      } else {                                                  // the other group's unit
        for (int d = 0; ok && d < tiles; ++d) {
          const uint32_t j = j0 + (uint32_t)d, slot = j % kStages, parity = (j / kStages) & 1u;
          ok = wait_all(bar_kin + slot * 8, parity);
          if (ok && elect_one()) mbar_arrive_cta(bar_ke + slot * 8);
          __syncwarp();
          ok = ok && wait_all(bar_vin + slot * 8, parity);
          if (ok && elect_one()) mbar_arrive_cta(bar_ve + slot * 8);
          __syncwarp();
        }
      }
      j0 += (uint32_t)tiles;
      if (!ok || j0 >= T) break;
      u = next_unit(it, u, x_end - (x_begin + j0), Hkv, tokens, align);
    }
    // every product issued ends before the block leaves, also where the rows give up (one more commit arrives when all have)
    if (!ok) *s_fail = 1;
    __syncwarp();
    if (products && elect_one()) {
      int never = 0;
      umma_commit(bar_d + g * 8);
      mbar_wait_or_fail<false>(bar_d + g * 8, 0, &never, kWaitLimit);
    }
    __syncwarp();
  } else {
    // ========================================= row threads ==========================================
    const int grp = warp >> 2, row = tid & (kGroup - 1);      // group, row inside it
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + grp * 2 * kKeys + lane_base, tO = tmem + 4 * kKeys + grp * D + lane_base;
    const uint32_t my_s = bar_s + grp * 16, my_p = bar_p + grp * 16, my_o = bar_o + grp * 16, my_f = bar_f + grp * 8, my_e = bar_e + grp * 8,
                   my_r = bar_r + grp * 8;
    const int my_local = row / G, my_head = row % G;
    constexpr float kMaxSlack = 8.f;                          // as in bc_mask_attn.cu
    bool failed = false;
    uint32_t t = 0, e = 0, ph_r = 0;
    auto rows_sync = [&]() {
      mbar_arrive_cta(my_r);
      const bool ok = mbar_wait_or_fail<SHORTW>(my_r, ph_r, s_fail, a.wait_limit);
      ph_r ^= 1;
      return (bool)__all_sync(0xffffffffu, ok);
    };
    auto store8 = [&](int64_t at, const float* v, float f) {    // eight results, times f, at element `at` of the output
      if (a.out_f32) {
        float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at);
        dst[0] = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
        dst[1] = make_float4(v[4] * f, v[5] * f, v[6] * f, v[7] * f);
      } else {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i] * f, v[2 * i + 1] * f);
          b[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
        *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at) = make_uint4(b[0], b[1], b[2], b[3]);
      }
    };
    long long x = x_begin;
    Unit u = u0;
    for (;;) {
      // this group's rows of the unit (none of the other group's solo units)
      const int mine = u.solo < 0 ? min(u.count - grp * half, half) : (u.solo == grp ? u.count : 0);
      const int token0 = u.solo < 0 ? grp * half : 0;
      if (mine > 0) {
      const int rows = mine * G;
      const bool row_valid = row < rows;
      const bool warp_live = (warp & 3) * 32 < rows;          // a warp without a row only keeps the barriers' count
      const int vis = row_valid ? clamp_vis(u.base, token0 + my_local, u.P + u.nb + u.w) : 0;
      const Seen seen = seen_of(vis, u.P, u.nb, u.w, align);
      const int row0 = a.cu_q[u.i] + u.t * tokens + token0;   // packed row of the group's first token
      float m_ref = -INFINITY, l_run = 0.f;
      for (int n = u.n0; n < u.n1; ++n, ++t) {
        const bool ok = mbar_wait_or_fail<SHORTW>(my_s + (t & 1u) * 8, (t >> 1) & 1u, s_fail, a.wait_limit);
        if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
        if (warp_live) {
          tc_fence_after();
          const int k0 = n * kKeys;
          const uint32_t tMine = tS + (t & 1u) * kKeys;
          const bool all_visible = __all_sync(0xffffffffu, !row_valid || inside(seen, k0));
          float s[kKeys];
          tmem_ld32_async(tMine, s);
          tmem_ld32_async(tMine + 32, s + 32);
          tmem_wait_ld();
          if (!all_visible) {
            uint32_t mask[2];
            tile_mask(mask, seen, k0);
#pragma unroll
            for (int j = 0; j < kKeys; ++j)
              if (!(mask[j >> 5] >> (j & 31) & 1)) s[j] = -INFINITY;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < kKeys; j += 8) {
            mx[0] = max3(mx[0], s[j], s[j + 1]); mx[1] = max3(mx[1], s[j + 2], s[j + 3]);
            mx[2] = max3(mx[2], s[j + 4], s[j + 5]); mx[3] = max3(mx[3], s[j + 6], s[j + 7]);
          }
          const float tile_max = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;   // the scale is positive
          float alpha = 1.f;
          const bool raise = tile_max > m_ref + kMaxSlack || (m_ref == -INFINITY && tile_max > -INFINITY);
          if (raise) {
            alpha = fast_exp2(m_ref - tile_max);
            m_ref = tile_max;
            l_run *= alpha;
          }
          const float m_safe = m_ref == -INFINITY ? 0.f : m_ref;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            uint32_t pk[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float p0 = fast_exp2(fmaf(s[cb * 32 + j], a.scale_log2, -m_safe));
              const float p1 = fast_exp2(fmaf(s[cb * 32 + j + 1], a.scale_log2, -m_safe));
              sum[(j >> 1) & 3] += p0 + p1;
              const __nv_bfloat162 pb = __floats2bfloat162_rn(p0, p1);   // the second product's operand type: off by 2^-8 of the weight at most
              pk[j >> 1] = *reinterpret_cast<const uint32_t*>(&pb);
            }
            tmem_st16(tMine + cb * 16, pk);
          }
          l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          // The rows whose reference has moved are rescaled, once the product of the tile before is done.  (Its barrier's completion
          // before that one, of tile t - 3, lies a tile back: S of tile t - 1 was issued behind that product.  So the parity tells.)
          if (n > u.n0 && __any_sync(0xffffffffu, raise)) {
            const bool done = mbar_wait_or_fail<SHORTW>(my_o + ((t - 1) & 1u) * 8, ((t - 1) >> 1) & 1u, s_fail, a.wait_limit);
            if (!__all_sync(0xffffffffu, done)) { failed = true; break; }
            tc_fence_after();
#pragma unroll 1
            for (int cb = 0; cb < D / 32; ++cb) {
              float v[32];
              tmem_ld32_async(tO + cb * 32, v);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] *= alpha;
              tmem_st32(tO + cb * 32, v);
            }
          }
          tmem_wait_st();
          tc_fence_before();
        }
        mbar_arrive_cta(my_p + (t & 1u) * 8);
      }
      if (failed) break;

      // ---- the piece's result -----------------------------------------------------------------------------------------
      const bool complete = u.n0 == 0 && u.n1 == u.N;
      const int my_half = u.solo < 0 ? grp : 0;               // of the block's partial results
      auto po_of = [&](int64_t slot) { return reinterpret_cast<float4*>(a.part_o) + (slot * 2 + my_half) * (D / 4) * kTile; };
      auto ml_of = [&](int64_t slot) { return a.part_ml + (slot * 2 + my_half) * 2 * kTile; };
      if (warp_live) {
        const bool ok = mbar_wait_or_fail<SHORTW>(my_f, e & 1u, s_fail, a.wait_limit);
        if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
        tc_fence_after();
        const float inv = l_run > 0.f ? 1.f / l_run : (l_run == 0.f ? 0.f : l_run);   // NaN stays NaN
        const int64_t at = ((int64_t)(row0 + my_local) * Hq + u.h * G + my_head) * D;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (u.n0 == 0 ? 1 : 0);
        float4* po = po_of(slot) + row;
        // 32 columns at a time, not unrolled: this runs once per unit, and its instructions come from memory the first time
#pragma unroll 1
        for (int cb = 0; cb < D / 32; ++cb) {
          float o[32];
          tmem_ld32_async(tO + cb * 32, o);
          tmem_wait_ld();
          if (row_valid && complete) {
#pragma unroll
            for (int d = 0; d < 32; d += 8) store8(at + cb * 32 + d, o + d, inv);
          }
          if (row_valid && !complete) {
#pragma unroll
            for (int d = 0; d < 8; ++d) po[(cb * 8 + d) * kTile] = make_float4(o[4 * d], o[4 * d + 1], o[4 * d + 2], o[4 * d + 3]);
          }
        }
        tc_fence_before();
        mbar_arrive_cta(my_e);
        if (!complete) {
          if (row_valid) {
            ml_of(slot)[row] = m_ref;
            ml_of(slot)[kTile + row] = l_run;
          }
          __threadfence();
        }
      } else {
        // the barrier's every completion is waited for (a parity tells two of them apart, no more)
        const bool ok = mbar_wait_or_fail<SHORTW>(my_f, e & 1u, s_fail, a.wait_limit);
        if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
        mbar_arrive_cta(my_e);
      }
      if (!complete) {
        if (!rows_sync()) { failed = true; break; }
        // the unit's first block and number of pieces: from its place on the line, where units are not cut one by one
        const long long x0 = x - u.n0;
        const int b0 = by_unit ? it.b0 : (int)(x0 / it.span);
        const int pieces = by_unit ? it.pieces : (int)((x0 + u.N - 1) / it.span) - b0 + 1;
        auto slot_of = [&](int j) { return 2 * (int64_t)(b0 + j) + (j == 0 ? 1 : 0); };
        // true for the last of `count` callers
        auto last_of = [&](int32_t* ticket, int count, bool* is_last) {
          if (row == 0) {
            const int got = atomicAdd(ticket, 1);
            if (got == count - 1) *ticket = 0;                  // all have come: zero again for the next launch
            s_ticket[grp] = got;
          }
          if (!rows_sync()) return false;
          *is_last = s_ticket[grp] == count - 1;
          if (*is_last) __threadfence();
          return true;
        };
        // Joins pieces j0, j0 + step, ... (`count`, at most 32) in this order, into the output or into the first one's place.
        // Threads are spread over the rows there are and, where these are few, over the head's coordinates.
        int rows2 = 8;
        while (rows2 < rows) rows2 <<= 1;                      // 8 .. 128
        const int r = row & (rows2 - 1), part = row / rows2, parts = kGroup / rows2;
        auto join = [&](int j0, int step, int count, bool final) {
          float m_all = -INFINITY, l_all = 0.f;
          if (r < rows) {
#pragma unroll 4
            for (int j = 0; j < count; ++j) {
              const float* ml = ml_of(slot_of(j0 + j * step));
              const float m = __ldcg(ml + r), l = __ldcg(ml + kTile + r), to = fmaxf(m_all, m), safe = to == -INFINITY ? 0.f : to;
              l_all = l_all * fast_exp2(m_all - safe) + l * fast_exp2(m - safe);
              m_all = to;
            }
          }
          const float m_safe = m_all == -INFINITY ? 0.f : m_all;
          const float inv = final ? (l_all > 0.f ? 1.f / l_all : (l_all == 0.f ? 0.f : l_all)) : 1.f;
          const int64_t at = ((int64_t)(row0 + r / G) * Hq + u.h * G + r % G) * D;
          const int each = max(1, D / 8 / parts);              // groups of eight coordinates per thread
          auto some = [&](int d8, auto width) {                // `width` of them at a time
            constexpr int kWidth = decltype(width)::value;
            float v[8 * kWidth];
#pragma unroll
            for (int i = 0; i < 8 * kWidth; ++i) v[i] = 0.f;
#pragma unroll (kWidth == 1 ? 4 : 2)
            for (int j = 0; j < count; ++j) {
              const int64_t slot = slot_of(j0 + j * step);
              const float f = fast_exp2(__ldcg(ml_of(slot) + r) - m_safe);
              const float4* po = po_of(slot) + 2 * d8 * kTile + r;
#pragma unroll
              for (int i = 0; i < 2 * kWidth; ++i) {
                const float4 p = __ldcg(po + i * kTile);
                v[4 * i] = fmaf(p.x, f, v[4 * i]); v[4 * i + 1] = fmaf(p.y, f, v[4 * i + 1]);
                v[4 * i + 2] = fmaf(p.z, f, v[4 * i + 2]); v[4 * i + 3] = fmaf(p.w, f, v[4 * i + 3]);
              }
            }
            if (final) {
#pragma unroll
              for (int i = 0; i < kWidth; ++i) store8(at + (d8 + i) * 8, v + 8 * i, inv);
            } else {
              float4* po = po_of(slot_of(j0)) + 2 * d8 * kTile + r;
#pragma unroll
              for (int i = 0; i < 2 * kWidth; ++i) po[i * kTile] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
          };
          if (r < rows) {
            const int d0 = part * each, d1 = min(D / 8, d0 + each);
            if (each >= 4) for (int d8 = d0; d8 < d1; d8 += 4) some(d8, Width<4>());
            else for (int d8 = d0; d8 < d1; ++d8) some(d8, Width<1>());
          }
          if (final) return true;
          if (!rows_sync()) return false;                      // everybody has read the first one's (m, l)
          if (r < rows && part == 0) { ml_of(slot_of(j0))[r] = m_all; ml_of(slot_of(j0))[kTile + r] = l_all; }
          __threadfence();
          return rows_sync();
        };
        constexpr int kFan = 16;
        const int mine = by_unit ? (int)blockIdx.x - b0 : (int)(x / it.span) - b0;   // number of this piece
        const int group = mine / kFan, groups = (pieces + kFan - 1) / kFan, in_group = min(kFan, pieces - group * kFan);
        int32_t* ticket = a.tickets + 2 * ((group > 0 ? BC_MAX_CHUNK_CTAS : 0) + b0 + group * kFan) + my_half;
        int j0 = group * kFan, step = 1, count = in_group;
        bool last = false;
#pragma unroll 1
        for (bool final = groups == 1;; final = true) {         // first these sixteen, then the sixteens
          failed = !last_of(ticket, count, &last);
          if (failed || !last) break;
          failed = !join(j0, step, count, final);
          if (failed || final) break;
          ticket = a.tickets + 2 * (2 * BC_MAX_CHUNK_CTAS + b0) + my_half;
          j0 = 0; step = kFan; count = groups;
        }
        if (failed) break;
      }
      ++e;
      }
      x += u.n1 - u.n0;
      if (x >= x_end) break;
      u = next_unit(it, u, x_end - x, Hkv, tokens, align);
    }
    if (failed) *s_fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (*s_fail && tid == 0) atomicCAS(a.m.status, 0, BC_ERR_TIMEOUT);
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
  }
}

template <int D, bool ROWS, bool SHORTW>
cudaError_t launch(const ChunkParams& p, const CUtensorMap& q_map, const CUtensorMap& pool_map, int grid, cudaStream_t s) {
  const int smem = Smem<D>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(k_chunk_attn<D, ROWS, SHORTW>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  k_chunk_attn<D, ROWS, SHORTW><<<grid, kThreads, smem, s>>>(p, q_map, pool_map);
  return cudaGetLastError();
}

// Entries per copy: the largest power of two up to 32 that divides the page size.
int copy_height(int page_size) {
  int r = 1;
  while (r < 32 && page_size % (2 * r) == 0) r *= 2;
  return r;
}

}  // namespace

// two pieces per block, two groups of rows each
size_t bc_chunk_part_o_bytes(int head_dim) { return (size_t)4 * BC_MAX_CHUNK_CTAS * head_dim * kTile * 4; }
size_t bc_chunk_part_ml_bytes() { return (size_t)4 * BC_MAX_CHUNK_CTAS * 2 * kTile * 4; }

// Tensor map of the whole pool: (64 coordinates, K|V x head x half, row, layer), unswizzled: the store's own chunk
// permutation is the swizzle.
bool bc_chunk_pool_map(const BcGeom& g, int layers, int64_t rows, void* pool, CUtensorMap* map) {
  if (!encode_tiled()) return false;
  const cuuint64_t dims[4] = {64, (cuuint64_t)(g.entry_bytes / 128), (cuuint64_t)rows, (cuuint64_t)layers};
  const cuuint64_t strides[3] = {128, (cuuint64_t)g.entry_bytes, (cuuint64_t)g.layer_bytes};
  const cuuint32_t box[4] = {64, 1, (cuuint32_t)copy_height(g.page_size), 1}, es[4] = {1, 1, 1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, pool, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t bc_launch_chunk_reference(const BcMeta& m, const BcGeom& g, const BcChunkArgs& a, cudaStream_t s) {
  k_chunk_reference<<<dim3(a.total_q, g.q_heads), 32, 0, s>>>(m, g, a);
  return cudaGetLastError();
}

cudaError_t bc_launch_chunk(const BcMeta& m, const BcGeom& g, const BcChunkArgs& a, const CUtensorMap& pool_map, int sms, cudaStream_t s) {
  ChunkParams p;
  p.m = m;
  p.slots = a.slots; p.first = a.first; p.cu_q = a.cu_q; p.n = a.n; p.total_q = a.total_q;
  p.out = a.out; p.out_f32 = a.out_f32; p.layer = a.layer; p.entry_bytes = g.entry_bytes; p.pool_layer = a.pool_layer;
  p.part_o = a.part_o; p.part_ml = a.part_ml; p.tickets = a.tickets;
  p.Hq = g.q_heads; p.Hkv = g.kv_heads; p.G = g.q_heads / g.kv_heads; p.page_size = g.page_size;
  p.by_page = make_fast_div((uint32_t)g.page_size);
  p.half = kTile / p.G;
  p.tokens = 2 * p.half;
  const int height = copy_height(g.page_size);
  const bool rows = height < 4;
  p.R = rows ? 1 : height;
  p.align = p.R > 8 ? p.R : 8;
  // Pieces of 8 tiles at least.  4, 8, 16: 512 rows over 1024 entries, 12 / 2 heads, 31.5, 29.0, 30.5 us; 13 rows over 512 18.2, 16.0,
  // 15.9; 64 x 5 rows over 585, 32 / 8 heads, 49.2, 47.8, 48.1.  (12, 2 and 512 units: none of them between 50 and 147.)
  p.min_shift = 3;
  p.wait_limit = a.wait_limit ? a.wait_limit : kWaitLimit;
  p.scale_log2 = a.sm_scale * 1.4426950408889634f;
  if (!encode_tiled()) return cudaErrorNotSupported;
  CUtensorMap q_map;
  const cuuint64_t dims[3] = {(cuuint64_t)g.head_dim, (cuuint64_t)g.q_heads, (cuuint64_t)a.total_q};
  const cuuint64_t strides[2] = {(cuuint64_t)g.head_dim * 2, (cuuint64_t)g.q_heads * g.head_dim * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.half}, es[3] = {1, 1, 1};
  if (encode_tiled()(&q_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  const int want = a.ctas > 0 ? a.ctas : sms, grid = want < BC_MAX_CHUNK_CTAS ? want : BC_MAX_CHUNK_CTAS;   // one resident block per SM
  if (a.ctas > 0) p.min_shift = 0;   // a given number of blocks is for the cuts it makes
  if (a.wait_limit) {   // bc_set_wait_limit: head_dim 128 only
    if (g.head_dim != 128) return cudaErrorNotSupported;
    return rows ? launch<128, true, true>(p, q_map, pool_map, grid, s) : launch<128, false, true>(p, q_map, pool_map, grid, s);
  }
  if (g.head_dim == 128) return rows ? launch<128, true, false>(p, q_map, pool_map, grid, s) : launch<128, false, false>(p, q_map, pool_map, grid, s);
  return rows ? launch<64, true, false>(p, q_map, pool_map, grid, s) : launch<64, false, false>(p, q_map, pool_map, grid, s);
}
