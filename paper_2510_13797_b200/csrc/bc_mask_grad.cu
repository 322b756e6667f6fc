// Gradient of the mask form (bc_mask_attn_forward): dense attention of the token and beacon rows over prompt, beacons and
// their own window, backwards, on the tcgen05 tensor cores.
//
// With the forward call's outputs O, the logarithm L of every row's sum of exp(scale S), S = Q K^T, and dO:
//     P = exp(scale S - L),   D = sum_d dO O,   dV = P^T dO,   dS = P (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q.
// Nothing of size rows x keys is stored: S and dP = dO V^T are computed again from tiles.  Two kernels share that work, so
// that every gradient is added up by one block in a fixed order and no atomic operation is needed (seven products instead
// of five; the results are reproducible):
//   k_dkv  one item per tile of 128 keys and KV head; walks the query tiles (64 rows = 64 / G tokens or beacons times the G
//          query heads of the KV head) that see any of its keys.  Transposed: S^T = K Q^T and dP^T = V dO^T (keys are the
//          rows of tensor memory), then P^T and dS^T, bf16, go back to tensor memory as the first operands of
//          dV += P^T dO and dK += dS^T Q, so the heads of a group are added up in the accumulator.
//   k_dq   one item per 256 query rows in two groups of 128, which share tiles of 64 keys: S = Q K^T, dP = dO V^T,
//          dS in tensor memory as the first operand of dQ += dS K.
// Both: one block per SM; a copy warp (tensor copies into a ring), a product warp, and two groups of four warps that turn S
// and dP into P and dS, one tile each in turn, so that the tensor pipe has the other tile's products to run meanwhile.
// The operands that are read along their rows (dO, Q, K in the second products) are the tiles as they are stored, N-major.
// Long items of k_dkv (the prompt's keys are seen by every row of a trajectory) are cut into pieces whose fp32 sums
// k_join adds up in order.  k_delta computes D and lays D and L out by KV head beforehand.
//
// Rows that a copy brings in past a sequence's end belong to its neighbour: their weights are set to zero by selection, and
// where such a row is itself a factor (K in dS K; Q and dO in dS^T Q and P^T dO) it is cleared in shared memory first.
#include <cuda.h>

#include <algorithm>
#include <vector>

#include "bc_common.cuh"

namespace {

#include "bc_tc.cuh"

constexpr int kD = 128;                            // head_dim
constexpr int kHalf = 64;                          // query rows of a k_dkv tile, keys of a k_dq tile
constexpr int kWide = kTile * kD * 2;              // bytes of a 128-row operand
constexpr int kSlim = kHalf * kD * 2;              // bytes of a 64-row operand
constexpr int kGroups = 2;
constexpr int kThreads = 64 + kGroups * 128;       // warp 0: copies, warp 1: products, then the groups
constexpr int kKvRing = 4, kQRing = 3;
constexpr float kLog2e = 1.4426950408889634f;

constexpr uint32_t kIdescN64 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kHalf >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);

struct SeqDesc {
  int32_t P, T, nb;                                // lengths
  int32_t prompt_row, tok_row, bea_row;            // first rows in the packed arrays
};
// A tile of keys and the query tiles that see any of them (tiles of 64 / G tokens or beacons)
struct KvItem {
  SeqDesc s;
  int32_t seg, k0, kvh;                            // 0 prompt, 1 beacons, 2 tokens; first key
  int32_t ta, nt, ba, nb_tiles;                    // first token tile, how many, first beacon tile, how many
  int32_t slot;                                    // place of the partial sums, -1: the whole item in one piece
  int32_t pad[2];
};
// Up to 256 / G tokens or beacons
struct QItem {
  SeqDesc s;
  int32_t kind, first, count, kvh;                 // 0 tokens, 1 beacons
  int32_t nt0, nt1, nt2, lo2;                      // tiles of 64 keys: prompt, beacons, tokens from lo2 on
  int32_t pad[2];
};
// A split item: its pieces are the slots first .. first + count - 1
struct JoinItem {
  SeqDesc s;
  int32_t seg, k0, kvh, first, count;
  int32_t pad[5];
};
static_assert(sizeof(KvItem) == 64 && sizeof(QItem) == 64 && sizeof(JoinItem) == 64, "descriptors are 64 bytes");

struct KvMaps { CUtensorMap q[2], o[2], k[3], v[3]; };   // q, dO by kind; k, v by segment
struct GradArgs {
  const void* items;
  int32_t n_items;
  const float *lse2, *delta;                       // [kv_heads][rows][G]: log2(e) L and D; rows: tokens, then beacons
  int64_t rows, tok_rows;
  __nv_bfloat16 *dk[3], *dv[3], *dq[2];
  float* partial;                                  // [slots][2][128][128]
  int32_t* status;
  int32_t Hq, Hkv, G, c, per;                      // per: tokens or beacons per query tile
  float scale, scale_log2;
  uint32_t wait_limit;
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ uint32_t swz64(int r, int ch16) {   // as swz, for operands of 64 rows
  return (uint32_t)((ch16 >> 3) * (kHalf * 128) + r * 128 + (((ch16 & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ int64_t stat_at(const GradArgs& a, const SeqDesc& s, int kvh, int kind, int first) {
  return ((int64_t)kvh * a.rows + (kind == 0 ? s.tok_row : a.tok_rows + s.bea_row) + first) * a.G;
}
// One row of an accumulator: 128 columns, times f, as bf16
__device__ __forceinline__ void store_row(__nv_bfloat16* dst, const float* o, float f) {
#pragma unroll
  for (int d = 0; d < kD; d += 16)
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + d), "r"(pack2(o[d] * f, o[d + 1] * f)),
                 "r"(pack2(o[d + 2] * f, o[d + 3] * f)), "r"(pack2(o[d + 4] * f, o[d + 5] * f)), "r"(pack2(o[d + 6] * f, o[d + 7] * f)),
                 "r"(pack2(o[d + 8] * f, o[d + 9] * f)), "r"(pack2(o[d + 10] * f, o[d + 11] * f)), "r"(pack2(o[d + 12] * f, o[d + 13] * f)),
                 "r"(pack2(o[d + 14] * f, o[d + 15] * f))
                 : "memory");
}
// Items of this block: round r hands out items [r * grid, (r + 1) * grid), forwards in even rounds, backwards in odd ones.
__device__ __forceinline__ int item_of(int r, int n) {
  const int grid = (int)gridDim.x, it = r * grid + ((r & 1) ? grid - 1 - (int)blockIdx.x : (int)blockIdx.x);
  return it < n ? it : -1;
}

// ---- dK and dV ---------------------------------------------------------------------------------------------------------------
// Tensor memory: stage b (tile t & 1): columns [128 b, 128 b + 64) S^T, then P^T in its first 32; [128 b + 64, 128 b + 128) dP^T, then
// dS^T in its first 32; [256, 384) dV, [384, 512) dK.  The tensor pipe runs a block's products in the order they were issued, so the
// products of tile t + 2 overwrite P and dS of tile t only after the products that read them.
//
// Barriers (t counts query tiles, e items; parity = uses so far & 1):
//   full[r] / empty[r]: Q and dO of ring place r have landed / been read      kv / kvfree: K and V of item e have landed / been read
//   s[b]: S^T and dP^T of the stage are there      p[b]: the group has stored P^T and dS^T
//   f: dK and dV of item e are final               x: both groups have read them          d: drain on the give-up path
template <bool SHORTW>
__global__ void __launch_bounds__(kThreads, 1) k_dkv(const GradArgs a, const __grid_constant__ KvMaps maps) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sK = smem_addr(smem), sV = sK + kWide, sRing = sV + kWide;   // ring place r: Q at sRing + r * 2 kSlim, dO behind it
  __shared__ __align__(8) uint64_t s_bars[2 * kKvRing + 9];
  __shared__ __align__(16) float s_stat[kGroups * 4][2][kHalf];   // a warp's copy of the tile's L and D
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail_word;
  volatile int* s_fail = &s_fail_word;
  const uint32_t bar_full = smem_addr(s_bars), bar_empty = bar_full + 8 * kKvRing, bar_kv = bar_empty + 8 * kKvRing, bar_kvfree = bar_kv + 8,
                 bar_s = bar_kv + 16, bar_p = bar_kv + 32, bar_f = bar_kv + 48, bar_x = bar_kv + 56, bar_d = bar_kv + 64;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const KvItem* items = static_cast<const KvItem*>(a.items);

  if (tid == 0) {
    for (int i = 0; i < 2 * kKvRing + 9; ++i) {
      const uint32_t bar = bar_full + 8 * i;
      const uint32_t count = bar == bar_p || bar == bar_p + 8 ? 128u : (bar == bar_x ? 256u : 1u);
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    *s_fail = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int box_rows = a.per * a.G;      // rows that a copy writes; the others (G does not divide 64) stay zero
  for (int idx = tid; idx < (kHalf - box_rows) * 16 * 2 * kKvRing; idx += kThreads) {
    const int op = idx / ((kHalf - box_rows) * 16), rest = idx % ((kHalf - box_rows) * 16);
    st_zero16(sRing + op * kSlim + swz64(box_rows + (rest >> 4), rest & 15));
  }
  proxy_fence();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem, tV = tmem + 256, tK = tmem + 384;

  if (warp == 0) {
    // ---- copies ----------------------------------------------------------------------------------------------------------
    bool ok = true;
    uint32_t t = 0, e = 0;
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_or_fail<SHORTW>(bar, parity, s_fail, a.wait_limit)) != 0;
    };
    const uint32_t bytes = (uint32_t)(2 * box_rows * kD * 2);
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const KvItem im = items[it];
      const int N = im.nt + im.nb_tiles;
      if (N == 0) continue;
      if (e > 0) ok = wait_all(bar_kvfree, (e - 1) & 1u);
      if (!ok) break;
      if (elect_one()) {
        const int row = (im.seg == 0 ? im.s.prompt_row : (im.seg == 1 ? im.s.bea_row : im.s.tok_row)) + im.k0;
        mbar_expect_tx(bar_kv, 2 * kWide);
        tma_3d(sK, &maps.k[im.seg], 0, im.kvh, row, bar_kv);
        tma_3d(sK + kTile * 128, &maps.k[im.seg], 64, im.kvh, row, bar_kv);
        tma_3d(sV, &maps.v[im.seg], 0, im.kvh, row, bar_kv);
        tma_3d(sV + kTile * 128, &maps.v[im.seg], 64, im.kvh, row, bar_kv);
      }
      __syncwarp();
      ++e;
      for (int n = 0; n < N; ++n, ++t) {
        const uint32_t place = t % kKvRing;
        if (t >= kKvRing) ok = wait_all(bar_empty + 8 * place, (t / kKvRing - 1) & 1u);
        if (!ok) break;
        if (elect_one()) {
          const int kind = n < im.nt ? 0 : 1, tile = kind == 0 ? im.ta + n : im.ba + n - im.nt;
          const int row = (kind == 0 ? im.s.tok_row : im.s.bea_row) + tile * a.per;
          const uint32_t dst = sRing + place * 2 * kSlim, bar = bar_full + 8 * place;
          mbar_expect_tx(bar, bytes);
          tma_3d(dst, &maps.q[kind], 0, im.kvh * a.G, row, bar);
          tma_3d(dst + kHalf * 128, &maps.q[kind], 64, im.kvh * a.G, row, bar);
          tma_3d(dst + kSlim, &maps.o[kind], 0, im.kvh * a.G, row, bar);
          tma_3d(dst + kSlim + kHalf * 128, &maps.o[kind], 64, im.kvh * a.G, row, bar);
        }
        __syncwarp();
      }
    }
    // no copy may be on its way when the block leaves: every one that was begun is waited for (at the end of ordinary work all have landed)
    if (!ok) *s_fail = 1;
    __syncwarp();
    int never = 0;
    if (e > 0) mbar_wait_or_fail<false>(bar_kv, (e - 1) & 1u, &never, kWaitLimit);
    for (uint32_t b = t > kKvRing ? t - kKvRing : 0; b < t; ++b)
      mbar_wait_or_fail<false>(bar_full + 8 * (b % kKvRing), (b / kKvRing) & 1u, &never, kWaitLimit);
    __syncwarp();
  } else if (warp == 1) {
    // ---- products --------------------------------------------------------------------------------------------------------
    bool ok = true, issued = false;
    uint32_t t0 = 0, e = 0;
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_or_fail<SHORTW>(bar, parity, s_fail, a.wait_limit)) != 0;
    };
    const uint64_t dK = umma_desc(sK), dV = umma_desc(sV), dQ = umma_desc(sRing), dQn = umma_desc_nmajor(sRing, kHalf * 128);
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const KvItem im = items[it];
      const int N = im.nt + im.nb_tiles;
      if (N == 0) continue;
      auto first_products = [&](int n) {           // S^T and dP^T of tile n
        const uint32_t t = t0 + n, place = t % kKvRing, stage = t & 1u;
        if (!wait_all(bar_full + 8 * place, (t / kKvRing) & 1u)) return false;
        const int kind = n < im.nt ? 0 : 1, tile = kind == 0 ? im.ta + n : im.ba + n - im.nt;
        const int valid = min((kind == 0 ? im.s.T : im.s.nb) - tile * a.per, a.per) * a.G;
        if (valid < box_rows) {                    // rows of the next sequence: cleared, they are factors of the second products
          for (int idx = valid * 16 + lane; idx < box_rows * 16; idx += 32) {
            st_zero16(sRing + place * 2 * kSlim + swz64(idx >> 4, idx & 15));
            st_zero16(sRing + place * 2 * kSlim + kSlim + swz64(idx >> 4, idx & 15));
          }
          proxy_fence();
          __syncwarp();
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t q = dQ + (uint64_t)((place * 2 * kSlim) >> 4), o = q + (uint64_t)(kSlim >> 4);
          const uint32_t tS = tmem + stage * 128;
#pragma unroll
          for (int kk = 0; kk < kD / 16; ++kk) {
            const uint64_t off_a = (uint64_t)(((kk >> 2) * (kTile * 128) + (kk & 3) * 32) >> 4), off_b = (uint64_t)(((kk >> 2) * (kHalf * 128) + (kk & 3) * 32) >> 4);
            umma<kIdescN64>(tS, dK + off_a, q + off_b, kk > 0);
          }
#pragma unroll
          for (int kk = 0; kk < kD / 16; ++kk) {
            const uint64_t off_a = (uint64_t)(((kk >> 2) * (kTile * 128) + (kk & 3) * 32) >> 4), off_b = (uint64_t)(((kk >> 2) * (kHalf * 128) + (kk & 3) * 32) >> 4);
            umma<kIdescN64>(tS + 64, dV + off_a, o + off_b, kk > 0);
          }
          umma_commit(bar_s + 8 * stage);
          if (n == N - 1) umma_commit(bar_kvfree);
        }
        __syncwarp();
        issued = true;
        return true;
      };
      ok = wait_all(bar_kv, e & 1u) && first_products(0) && (N < 2 || first_products(1));
      for (int n = 0; n < N && ok; ++n) {
        const uint32_t t = t0 + n, place = t % kKvRing, stage = t & 1u;
        ok = wait_all(bar_p + 8 * stage, (t >> 1) & 1u);
        if (ok && n == 0 && e > 0) ok = wait_all(bar_x, (e - 1) & 1u);     // the groups have read the last item's sums
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t q = dQn + (uint64_t)((place * 2 * kSlim) >> 4), o = q + (uint64_t)(kSlim >> 4);
          const uint32_t tP = tmem + stage * 128, tdS = tP + 64;
#pragma unroll
          for (int kk = 0; kk < kHalf / 16; ++kk) umma_ts(tV, tP + kk * 8, o + (uint64_t)((kk * 16 * 128) >> 4), (n > 0 || kk > 0) ? 1u : 0u);
#pragma unroll
          for (int kk = 0; kk < kHalf / 16; ++kk) umma_ts(tK, tdS + kk * 8, q + (uint64_t)((kk * 16 * 128) >> 4), (n > 0 || kk > 0) ? 1u : 0u);
          umma_commit(bar_empty + 8 * place);
          if (n == N - 1) umma_commit(bar_f);
        }
        __syncwarp();
        if (n + 2 < N) ok = first_products(n + 2);
      }
      t0 += N;
      ++e;
    }
    if (!ok) {
      *s_fail = 1;
      __syncwarp();
      if (issued && elect_one()) {                 // no product may be running when the block leaves
        int never = 0;
        umma_commit(bar_d);
        mbar_wait_or_fail<false>(bar_d, 0, &never, kWaitLimit);
      }
    }
    __syncwarp();
  } else {
    // ---- weights: one key per thread -----------------------------------------------------------------------------------------
    const int grp = (warp - 2) >> 2;
    float (*stats)[kHalf] = s_stat[warp - 2];
    // a warp reaches the 32 lanes of tensor memory that belong to its number modulo 4; its keys are those lanes
    const int key = (warp & 3) * 32 + lane;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + grp * 128 + lane_base, tP = tS, tD = tS + 64;
    bool ok = true;
    uint32_t t0 = 0, e = 0;
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const KvItem im = items[it];
      const int N = im.nt + im.nb_tiles, G = a.G, c = a.c;
      const int k = im.k0 + key, seg_len = im.seg == 0 ? im.s.P : (im.seg == 1 ? im.s.nb : im.s.T);
      const bool live = k < seg_len;
      // the token and beacon rows that see this key: [tok_lo, tok_hi) and [bea_lo, bea_hi)
      int tok_lo = 0, tok_hi = im.s.T, bea_lo = 0, bea_hi = im.s.nb;
      if (im.seg == 1) { tok_lo = (k + 1) * c; bea_lo = k; }
      if (im.seg == 2) {
        tok_lo = k;
        if (c > 1) { tok_hi = min(im.s.T, (k / c + 1) * c); bea_lo = k / c; bea_hi = min(im.s.nb, k / c + 1); }
      }
      if (!live) tok_hi = bea_hi = 0;
      float4 stat;                                 // this lane's share of the next tile's numbers: L and D of rows lane and lane + 32
      auto fetch = [&](int n) {
        const int kind = n < im.nt ? 0 : 1, first = (kind == 0 ? im.ta + n : im.ba + n - im.nt) * a.per;
        const int valid = min((kind == 0 ? im.s.T : im.s.nb) - first, a.per) * G;
        const int64_t at = stat_at(a, im.s, im.kvh, kind, first) + lane;
        stat = make_float4(0.f, 0.f, 0.f, 0.f);
        if (lane < valid) { stat.x = a.lse2[at]; stat.z = a.delta[at]; }
        if (lane + 32 < valid) { stat.y = a.lse2[at + 32]; stat.w = a.delta[at + 32]; }
      };
      const int n_first = (int)((t0 & 1u) ^ (uint32_t)grp);
      if (n_first < N) fetch(n_first);
      for (int n = n_first; n < N; n += 2) {
        const uint32_t t = t0 + n;
        __syncwarp();                              // the last tile's numbers have been read
        stats[0][lane] = stat.x; stats[0][lane + 32] = stat.y; stats[1][lane] = stat.z; stats[1][lane + 32] = stat.w;
        __syncwarp();
        if (n + 2 < N) fetch(n + 2);
        const int kind = n < im.nt ? 0 : 1, first = (kind == 0 ? im.ta + n : im.ba + n - im.nt) * a.per;
        const int all = min((kind == 0 ? im.s.T : im.s.nb) - first, a.per) * G;
        const int lo = kind == 0 ? tok_lo : bea_lo, hi = kind == 0 ? tok_hi : bea_hi;
        const int jlo = min(max(lo - first, 0), a.per) * G, jhi = min(min(hi - first, a.per) * G, all);
        const bool ok1 = mbar_wait_or_fail<SHORTW>(bar_s + 8 * grp, (t >> 1) & 1u, s_fail, a.wait_limit);
        ok = __all_sync(0xffffffffu, ok1);
        if (!ok) break;
        tc_fence_after();
        const bool whole = __all_sync(0xffffffffu, jlo == 0 && jhi == kHalf);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float s[32], dp[32];
          tmem_ld32_async(tS + h * 32, s);
          tmem_ld32_async(tD + h * 32, dp);
          tmem_wait_ld();
          uint32_t pp[16], ds[16];
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 l4 = *reinterpret_cast<const float4*>(&stats[0][h * 32 + j]);
            const float4 d4 = *reinterpret_cast<const float4*>(&stats[1][h * 32 + j]);
            const float ll[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
            float p[4], q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[i] = fast_exp2(fmaf(s[j + i], a.scale_log2, -ll[i]));
              q[i] = p[i] * (dp[j + i] - dd[i]);
              if (!whole) {
                const bool sees = h * 32 + j + i >= jlo && h * 32 + j + i < jhi;
                p[i] = sees ? p[i] : 0.f;
                q[i] = sees ? q[i] : 0.f;
              }
            }
            pp[j / 2] = pack2(p[0], p[1]); pp[j / 2 + 1] = pack2(p[2], p[3]);
            ds[j / 2] = pack2(q[0], q[1]); ds[j / 2 + 1] = pack2(q[2], q[3]);
          }
          tmem_st16(tP + h * 16, pp);
          tmem_st16(tD + h * 16, ds);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_cta(bar_p + 8 * grp);
      }
      if (!ok) break;
      // ---- the item's sums: the first group has dV, the second dK
      float o[kD];
      if (N > 0) {
        const bool ok1 = mbar_wait_or_fail<SHORTW>(bar_f, e & 1u, s_fail, a.wait_limit);
        ok = __all_sync(0xffffffffu, ok1);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) tmem_ld32_async((grp == 0 ? tV : tK) + lane_base + cb * 32, o + cb * 32);
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive_cta(bar_x);
        t0 += N;
        ++e;
      } else {
#pragma unroll
        for (int d = 0; d < kD; ++d) o[d] = 0.f;
      }
      if (im.slot >= 0) {
        float4* dst = reinterpret_cast<float4*>(a.partial + (((int64_t)im.slot * 2 + grp) * kTile + key) * kD);
#pragma unroll
        for (int d = 0; d < kD; d += 4) dst[d / 4] = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
      } else if (live) {
        const int row = (im.seg == 0 ? im.s.prompt_row : (im.seg == 1 ? im.s.bea_row : im.s.tok_row)) + k;
        store_row((grp == 0 ? a.dv : a.dk)[im.seg] + ((int64_t)row * a.Hkv + im.kvh) * kD, o, grp == 0 ? 1.f : a.scale);
      }
    }
    if (!ok) *s_fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (*s_fail && tid == 0) atomicCAS(a.status, 0, BC_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ---- dQ ------------------------------------------------------------------------------------------------------------------------
// Tensor memory, group g: columns [256 g, + 64) S, then dS in its first 32; [256 g + 64, + 64) dP; [256 g + 128, + 128) dQ.
// Barriers as above, with q / qfree for the item's Q and dO, and f, x per group.
template <bool SHORTW>
__global__ void __launch_bounds__(kThreads, 1) k_dq(const GradArgs a, const __grid_constant__ KvMaps maps) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sQ = smem_addr(smem), sRing = sQ + 4 * kWide;   // group g: Q at sQ + g * 2 kWide, dO behind it; ring place r: K, V
  __shared__ __align__(8) uint64_t s_bars[2 * kQRing + 11];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail_word;
  volatile int* s_fail = &s_fail_word;
  const uint32_t bar_full = smem_addr(s_bars), bar_empty = bar_full + 8 * kQRing, bar_q = bar_empty + 8 * kQRing, bar_qfree = bar_q + 8,
                 bar_s = bar_q + 16, bar_p = bar_q + 32, bar_f = bar_q + 48, bar_x = bar_q + 64, bar_d = bar_q + 80;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const QItem* items = static_cast<const QItem*>(a.items);

  if (tid == 0) {
    for (int i = 0; i < 2 * kQRing + 11; ++i) {
      const uint32_t bar = bar_full + 8 * i;
      const uint32_t count = bar == bar_p || bar == bar_p + 8 || bar == bar_x || bar == bar_x + 8 ? 128u : 1u;
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    *s_fail = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const int box_rows = a.per * a.G;
  for (int idx = tid; idx < (kTile - box_rows) * 16 * 4; idx += kThreads) {
    const int op = idx / ((kTile - box_rows) * 16), rest = idx % ((kTile - box_rows) * 16);
    st_zero16(sQ + op * kWide + swz(box_rows + (rest >> 4), rest & 15));
  }
  proxy_fence();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  auto key_tile = [](const QItem& im, int n, int* k0) {          // segment and first key of tile n
    const int seg = n < im.nt0 ? 0 : (n < im.nt0 + im.nt1 ? 1 : 2);
    *k0 = seg == 0 ? n * kHalf : (seg == 1 ? (n - im.nt0) * kHalf : im.lo2 + (n - im.nt0 - im.nt1) * kHalf);
    return seg;
  };

  if (warp == 0) {
    bool ok = true;
    uint32_t t = 0, e = 0;
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_or_fail<SHORTW>(bar, parity, s_fail, a.wait_limit)) != 0;
    };
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const QItem im = items[it];
      const int N = im.nt0 + im.nt1 + im.nt2, groups = im.count > a.per ? 2 : 1;
      if (e > 0) ok = wait_all(bar_qfree, (e - 1) & 1u);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(bar_q, (uint32_t)(groups * 2 * box_rows * kD * 2));
        for (int g = 0; g < groups; ++g) {
          const int row = (im.kind == 0 ? im.s.tok_row : im.s.bea_row) + im.first + g * a.per;
          const uint32_t dst = sQ + g * 2 * kWide;
          tma_3d(dst, &maps.q[im.kind], 0, im.kvh * a.G, row, bar_q);
          tma_3d(dst + kTile * 128, &maps.q[im.kind], 64, im.kvh * a.G, row, bar_q);
          tma_3d(dst + kWide, &maps.o[im.kind], 0, im.kvh * a.G, row, bar_q);
          tma_3d(dst + kWide + kTile * 128, &maps.o[im.kind], 64, im.kvh * a.G, row, bar_q);
        }
      }
      __syncwarp();
      ++e;
      for (int n = 0; n < N; ++n, ++t) {
        const uint32_t place = t % kQRing;
        if (t >= kQRing) ok = wait_all(bar_empty + 8 * place, (t / kQRing - 1) & 1u);
        if (!ok) break;
        if (elect_one()) {
          int k0;
          const int seg = key_tile(im, n, &k0);
          const int row = (seg == 0 ? im.s.prompt_row : (seg == 1 ? im.s.bea_row : im.s.tok_row)) + k0;
          const uint32_t dst = sRing + place * 2 * kSlim, bar = bar_full + 8 * place;
          mbar_expect_tx(bar, 2 * kSlim);
          tma_3d(dst, &maps.k[seg], 0, im.kvh, row, bar);
          tma_3d(dst + kHalf * 128, &maps.k[seg], 64, im.kvh, row, bar);
          tma_3d(dst + kSlim, &maps.v[seg], 0, im.kvh, row, bar);
          tma_3d(dst + kSlim + kHalf * 128, &maps.v[seg], 64, im.kvh, row, bar);
        }
        __syncwarp();
      }
    }
    if (!ok) *s_fail = 1;
    __syncwarp();
    int never = 0;
    if (e > 0) mbar_wait_or_fail<false>(bar_q, (e - 1) & 1u, &never, kWaitLimit);
    for (uint32_t b = t > kQRing ? t - kQRing : 0; b < t; ++b)
      mbar_wait_or_fail<false>(bar_full + 8 * (b % kQRing), (b / kQRing) & 1u, &never, kWaitLimit);
    __syncwarp();
  } else if (warp == 1) {
    bool ok = true, issued = false;
    uint32_t t0 = 0, e = 0, used[2] = {0, 0}, begun[2] = {0, 0};   // per group: tiles and items so far
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait_or_fail<SHORTW>(bar, parity, s_fail, a.wait_limit)) != 0;
    };
    const uint64_t dQ = umma_desc(sQ), dK = umma_desc(sRing), dKn = umma_desc_nmajor(sRing, kHalf * 128);
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const QItem im = items[it];
      const int N = im.nt0 + im.nt1 + im.nt2, groups = im.count > a.per ? 2 : 1;
      auto landed = [&](int n) {                   // K and V of tile n; keys past the segment are cleared: K is a factor of dS K
        const uint32_t t = t0 + n, place = t % kQRing;
        if (!wait_all(bar_full + 8 * place, (t / kQRing) & 1u)) return false;
        int k0;
        const int seg = key_tile(im, n, &k0), valid = min((seg == 0 ? im.s.P : (seg == 1 ? im.s.nb : im.s.T)) - k0, kHalf);
        if (valid < kHalf) {
          for (int idx = valid * 16 + lane; idx < kHalf * 16; idx += 32) st_zero16(sRing + place * 2 * kSlim + swz64(idx >> 4, idx & 15));
          proxy_fence();
          __syncwarp();
        }
        return true;
      };
      auto first_products = [&](int g, int n) {
        const uint32_t place = (t0 + n) % kQRing;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t q = dQ + (uint64_t)((g * 2 * kWide) >> 4), o = q + (uint64_t)(kWide >> 4);
          const uint64_t k = dK + (uint64_t)((place * 2 * kSlim) >> 4), v = k + (uint64_t)(kSlim >> 4);
          const uint32_t tS = tmem + g * 256;
#pragma unroll
          for (int kk = 0; kk < kD / 16; ++kk) {
            const uint64_t off_a = (uint64_t)(((kk >> 2) * (kTile * 128) + (kk & 3) * 32) >> 4), off_b = (uint64_t)(((kk >> 2) * (kHalf * 128) + (kk & 3) * 32) >> 4);
            umma<kIdescN64>(tS, q + off_a, k + off_b, kk > 0);
          }
#pragma unroll
          for (int kk = 0; kk < kD / 16; ++kk) {
            const uint64_t off_a = (uint64_t)(((kk >> 2) * (kTile * 128) + (kk & 3) * 32) >> 4), off_b = (uint64_t)(((kk >> 2) * (kHalf * 128) + (kk & 3) * 32) >> 4);
            umma<kIdescN64>(tS + 64, o + off_a, v + off_b, kk > 0);
          }
          umma_commit(bar_s + 8 * g);
          if (n == N - 1 && g == groups - 1) umma_commit(bar_qfree);
        }
        __syncwarp();
        issued = true;
      };
      ok = wait_all(bar_q, e & 1u) && landed(0);
      if (!ok) break;
      for (int g = 0; g < groups; ++g) first_products(g, 0);
      for (int n = 0; n < N && ok; ++n) {
        const uint32_t place = (t0 + n) % kQRing;
        for (int g = 0; g < groups && ok; ++g) {
          ok = wait_all(bar_p + 8 * g, used[g] & 1u);
          ++used[g];
          if (ok && n == 0 && begun[g] > 0) ok = wait_all(bar_x + 8 * g, (begun[g] - 1) & 1u);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t k = dKn + (uint64_t)((place * 2 * kSlim) >> 4);
            const uint32_t tdS = tmem + g * 256, tO = tdS + 128;
#pragma unroll
            for (int kk = 0; kk < kHalf / 16; ++kk) umma_ts(tO, tdS + kk * 8, k + (uint64_t)((kk * 16 * 128) >> 4), (n > 0 || kk > 0) ? 1u : 0u);
            if (g == groups - 1) umma_commit(bar_empty + 8 * place);
            if (n == N - 1) umma_commit(bar_f + 8 * g);
          }
          __syncwarp();
          if (n + 1 < N) {
            if (g == 0) ok = landed(n + 1);
            if (ok) first_products(g, n + 1);
          }
        }
      }
      for (int g = 0; g < groups; ++g) ++begun[g];
      t0 += N;
      ++e;
    }
    if (!ok) {
      *s_fail = 1;
      __syncwarp();
      if (issued && elect_one()) {
        int never = 0;
        umma_commit(bar_d);
        mbar_wait_or_fail<false>(bar_d, 0, &never, kWaitLimit);
      }
    }
    __syncwarp();
  } else {
    // ---- weights: one query row per thread
    const int grp = (warp - 2) >> 2, row = (warp & 3) * 32 + lane, G = a.G, c = a.c;
    const uint32_t tS = tmem + grp * 256 + ((uint32_t)((warp & 3) * 32) << 16), tD = tS + 64, tO = tS + 128;
    const int my_local = row / G, my_head = row % G;
    bool ok = true;
    uint32_t t = 0, e = 0;
    for (int r = 0; ok; ++r) {
      const int it = item_of(r, a.n_items);
      if (it < 0) break;
      const QItem im = items[it];
      const int N = im.nt0 + im.nt1 + im.nt2, first = im.first + grp * a.per, count = min(im.count - grp * a.per, a.per);
      if (count <= 0) continue;
      const bool live = row < count * G;
      const int64_t at = stat_at(a, im.s, im.kvh, im.kind, first) + row;
      const float l2 = live ? a.lse2[at] : 0.f, dl = live ? a.delta[at] : 0.f;
      const int idx = first + my_local;
      int bea_hi, tok_lo, tok_hi;                  // visible: the prompt, beacons [0, bea_hi), tokens [tok_lo, tok_hi)
      if (im.kind == 0) { bea_hi = c > 1 ? idx / c : 0; tok_lo = c > 1 ? idx / c * c : 0; tok_hi = idx + 1; }
      else { bea_hi = idx + 1; tok_lo = idx * c; tok_hi = (idx + 1) * c; }
      for (int n = 0; n < N; ++n, ++t) {
        int k0;
        const int seg = key_tile(im, n, &k0);
        int lo = 0, hi = im.s.P;
        if (seg == 1) hi = min(bea_hi, im.s.nb);
        if (seg == 2) { lo = tok_lo; hi = min(tok_hi, im.s.T); }
        if (!live) hi = lo;
        const int jlo = max(lo - k0, 0), jhi = min(hi - k0, kHalf);
        const bool ok1 = mbar_wait_or_fail<SHORTW>(bar_s + 8 * grp, t & 1u, s_fail, a.wait_limit);
        ok = __all_sync(0xffffffffu, ok1);
        if (!ok) break;
        tc_fence_after();
        const bool whole = __all_sync(0xffffffffu, jlo == 0 && jhi == kHalf);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float s[32], dp[32];
          tmem_ld32_async(tS + h * 32, s);
          tmem_ld32_async(tD + h * 32, dp);
          tmem_wait_ld();
          uint32_t ds[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float q[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              q[i] = fast_exp2(fmaf(s[j + i], a.scale_log2, -l2)) * (dp[j + i] - dl);
              if (!whole) q[i] = h * 32 + j + i >= jlo && h * 32 + j + i < jhi ? q[i] : 0.f;
            }
            ds[j / 2] = pack2(q[0], q[1]);
          }
          tmem_st16(tS + h * 16, ds);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_cta(bar_p + 8 * grp);
      }
      if (!ok) break;
      const bool ok1 = mbar_wait_or_fail<SHORTW>(bar_f + 8 * grp, e & 1u, s_fail, a.wait_limit);
      ok = __all_sync(0xffffffffu, ok1);
      if (!ok) break;
      tc_fence_after();
      float o[kD];
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) tmem_ld32_async(tO + cb * 32, o + cb * 32);
      tmem_wait_ld();
      tc_fence_before();
      mbar_arrive_cta(bar_x + 8 * grp);
      ++e;
      if (live)
        store_row(a.dq[im.kind] + ((int64_t)((im.kind == 0 ? im.s.tok_row : im.s.bea_row) + idx) * a.Hq + im.kvh * G + my_head) * kD, o, a.scale);
    }
    if (!ok) *s_fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (*s_fail && tid == 0) atomicCAS(a.status, 0, BC_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// D = sum_d dO O of every row and head, and L, laid out by KV head: 16 lanes per head row, both 16-byte loads.
__global__ void __launch_bounds__(256) k_delta(const uint4* __restrict__ out_tok, const uint4* __restrict__ d_tok, const float* __restrict__ lse_tok,
                                               const uint4* __restrict__ out_bea, const uint4* __restrict__ d_bea, const float* __restrict__ lse_bea,
                                               int64_t tok_rows, int64_t rows, int Hq, int G, float* __restrict__ lse2, float* __restrict__ delta) {
  const int64_t units = rows * Hq;
  const int lane = threadIdx.x & 15;
  // the 16 lanes of a row are in one warp, and the warp's two rows run the loop equally often (an odd last row is computed twice)
  for (int64_t u0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4; u0 < units + (units & 1); u0 += (int64_t)gridDim.x * 16) {
    const int64_t u = u0 < units ? u0 : units - 1;
    const int64_t row = u / Hq;
    const int head = (int)(u - row * Hq);
    const bool tok = row < tok_rows;
    const int64_t in = tok ? u : u - tok_rows * Hq;
    const uint4 x = __ldcs((tok ? out_tok : out_bea) + in * 16 + lane), y = __ldcs((tok ? d_tok : d_bea) + in * 16 + lane);
    const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s = fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), s);
      s = fmaf(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), s);
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0) {
      const int64_t to = ((int64_t)(head / G) * rows + row) * G + head % G;
      delta[to] = s;
      lse2[to] = (tok ? lse_tok : lse_bea)[in] * kLog2e;
    }
  }
}

// Adds the pieces of the split items in order: one block per item, of dK or dV, and eight keys.
__global__ void __launch_bounds__(256) k_join(const JoinItem* __restrict__ items, const GradArgs a) {
  const JoinItem im = items[blockIdx.x];
  const int which = blockIdx.y & 1, key = (int)(blockIdx.y >> 1) * 8 + (int)(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int seg_len = im.seg == 0 ? im.s.P : (im.seg == 1 ? im.s.nb : im.s.T);
  if (im.k0 + key >= seg_len) return;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < im.count; ++p) {
    const float4 v = *reinterpret_cast<const float4*>(a.partial + ((((int64_t)im.first + p) * 2 + which) * kTile + key) * kD + lane * 4);
    t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
  }
  const float f = which == 0 ? 1.f : a.scale;
  const int row = (im.seg == 0 ? im.s.prompt_row : (im.seg == 1 ? im.s.bea_row : im.s.tok_row)) + im.k0 + key;
  uint2 o;
  o.x = pack2(t.x * f, t.y * f); o.y = pack2(t.z * f, t.w * f);
  *reinterpret_cast<uint2*>((which == 0 ? a.dv : a.dk)[im.seg] + ((int64_t)row * a.Hkv + im.kvh) * kD + lane * 4) = o;
}

bool map_3d(CUtensorMap* m, const void* base, int heads, int64_t rows, int box_heads, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)kD, (cuuint64_t)heads, (cuuint64_t)(rows > 0 ? rows : 1)};
  const cuuint64_t strides[2] = {(cuuint64_t)kD * 2, (cuuint64_t)heads * kD * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, es[3] = {1, 1, 1};
  return encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The work lists, and where everything is in the workspace.
struct Plan {
  std::vector<KvItem> kv;
  std::vector<QItem> q;
  std::vector<JoinItem> join;
  int64_t prompts = 0, tokens = 0, beacons = 0;
  int32_t slots = 0;
  size_t at_kv = 0, at_q = 0, at_join = 0, at_lse = 0, at_delta = 0, at_partial = 0, total = 0;   // the status word is at 0
};
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
constexpr int kSms = 148;
constexpr int kMinPiece = 24;   // query tiles: a piece's partial sums cost about five tiles' time

bc_status make_plan(int n_seqs, int q_heads, int kv_heads, int head_dim, int c, const int32_t* cu_prompt, const int32_t* cu_tokens, Plan* p) {
  if (n_seqs < 1 || !cu_prompt || !cu_tokens || c < 1 || kv_heads < 1 || q_heads < 1 || q_heads % kv_heads) return BC_ERR_INVALID_ARG;
  if (head_dim != kD || q_heads / kv_heads > 16) return BC_ERR_UNSUPPORTED;
  const int G = q_heads / kv_heads, per = kHalf / G, wide = 2 * (kTile / G);
  int64_t beacons = 0, work = 0, n_kv = 0, n_q = 0;
  for (int i = 0; i < n_seqs; ++i) {
    const int64_t P = (int64_t)cu_prompt[i + 1] - cu_prompt[i], T = (int64_t)cu_tokens[i + 1] - cu_tokens[i];
    if (P < 0 || T < 0) return BC_ERR_INVALID_ARG;
    const int64_t nb = c > 1 ? T / c : 0;
    beacons += nb;
    n_kv += (P + kTile - 1) / kTile + (nb + kTile - 1) / kTile + (T + kTile - 1) / kTile;
    n_q += (T + wide - 1) / wide + (nb + wide - 1) / wide;
  }
  if (cu_prompt[0] != 0 || cu_tokens[0] != 0) return BC_ERR_INVALID_ARG;
  if ((n_kv + n_q) * kv_heads > (1 << 24)) return BC_ERR_UNSUPPORTED;
  p->prompts = cu_prompt[n_seqs]; p->tokens = cu_tokens[n_seqs]; p->beacons = beacons;

  auto tiles = [&](int rows) { return (rows + per - 1) / per; };
  std::vector<KvItem> whole;
  int64_t bea_row = 0;
  for (int i = 0; i < n_seqs; ++i) {
    SeqDesc s;
    s.P = cu_prompt[i + 1] - cu_prompt[i]; s.T = cu_tokens[i + 1] - cu_tokens[i]; s.nb = c > 1 ? s.T / c : 0;
    s.prompt_row = cu_prompt[i]; s.tok_row = cu_tokens[i]; s.bea_row = (int32_t)bea_row;
    bea_row += s.nb;
    for (int seg = 0; seg < 3; ++seg) {
      const int len = seg == 0 ? s.P : (seg == 1 ? s.nb : s.T);
      for (int k0 = 0; k0 < len; k0 += kTile) {
        const int k1 = std::min(len, k0 + kTile) - 1;          // the last key
        int64_t t_lo = 0, t_hi = s.T, b_lo = 0, b_hi = s.nb;   // the rows that see any of the keys
        if (seg == 1) { t_lo = std::min<int64_t>((int64_t)(k0 + 1) * c, s.T); b_lo = k0; }
        if (seg == 2) {
          t_lo = k0;
          if (c > 1) { t_hi = std::min<int64_t>((int64_t)(k1 / c + 1) * c, s.T); b_lo = std::min(k0 / c, s.nb); b_hi = std::min(k1 / c + 1, s.nb); }
        }
        KvItem im = {};
        im.s = s; im.seg = seg; im.k0 = k0; im.slot = -1;
        im.ta = (int)t_lo / per; im.nt = t_hi > t_lo ? tiles((int)t_hi) - im.ta : 0;
        im.ba = (int)b_lo / per; im.nb_tiles = b_hi > b_lo ? tiles((int)b_hi) - im.ba : 0;
        work += im.nt + im.nb_tiles;
        whole.push_back(im);
      }
    }
    for (int kind = 0; kind < 2; ++kind) {
      const int len = kind == 0 ? s.T : s.nb;
      for (int f = 0; f < len; f += wide) {
        QItem im = {};
        im.s = s; im.kind = kind; im.first = f; im.count = std::min(wide, len - f);
        const int last = f + im.count - 1;
        const int b_hi = kind == 0 ? (c > 1 ? last / c : 0) : last + 1;
        const int t_lo = kind == 0 ? (c > 1 ? f / c * c : 0) : f * c, t_hi = kind == 0 ? last + 1 : (last + 1) * c;
        im.lo2 = t_lo / kHalf * kHalf;
        im.nt0 = (s.P + kHalf - 1) / kHalf; im.nt1 = (b_hi + kHalf - 1) / kHalf; im.nt2 = (t_hi - im.lo2 + kHalf - 1) / kHalf;
        for (int h = 0; h < kv_heads; ++h) { im.kvh = h; p->q.push_back(im); }
      }
    }
  }
  // An item is cut where it is longer than a third of an SM's share of all the work, so that the last items to end are short
  const int64_t piece = std::max<int64_t>(kMinPiece, work * kv_heads / (kSms * 3));
  for (const KvItem& w : whole) {
    const int N = w.nt + w.nb_tiles;
    const int pieces = N > piece + piece / 2 ? (int)((N + piece - 1) / piece) : 1;
    for (int h = 0; h < kv_heads; ++h) {
      KvItem im = w;
      im.kvh = h;
      if (pieces > 1) {
        JoinItem j = {};
        j.s = w.s; j.seg = w.seg; j.k0 = w.k0; j.kvh = h; j.first = p->slots; j.count = pieces;
        p->join.push_back(j);
      }
      for (int q = 0; q < pieces; ++q) {
        const int a = (int)((int64_t)N * q / pieces), b = (int)((int64_t)N * (q + 1) / pieces);   // tiles [a, b) of the item
        im.ta = w.ta + std::min(a, w.nt); im.nt = std::min(b, w.nt) - std::min(a, w.nt);
        im.ba = w.ba + std::max(a - w.nt, 0); im.nb_tiles = std::max(b - w.nt, 0) - std::max(a - w.nt, 0);
        im.slot = pieces > 1 ? p->slots++ : -1;
        p->kv.push_back(im);
      }
    }
  }
  std::stable_sort(p->kv.begin(), p->kv.end(), [](const KvItem& x, const KvItem& y) { return x.nt + x.nb_tiles > y.nt + y.nb_tiles; });
  std::stable_sort(p->q.begin(), p->q.end(), [](const QItem& x, const QItem& y) { return x.nt0 + x.nt1 + x.nt2 > y.nt0 + y.nt1 + y.nt2; });
  size_t o = 256;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes); return at; };
  p->at_kv = take(p->kv.size() * sizeof(KvItem));
  p->at_q = take(p->q.size() * sizeof(QItem));
  p->at_join = take(p->join.size() * sizeof(JoinItem));
  const size_t stats = (size_t)(p->tokens + p->beacons) * q_heads * sizeof(float);
  p->at_lse = take(stats);
  p->at_delta = take(stats);
  p->at_partial = take((size_t)p->slots * 2 * kTile * kD * sizeof(float));
  p->total = o;
  return BC_OK;
}

int sm_count() {
  static int n = 0;
  if (!n) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = kSms;
  }
  return n;
}

uint32_t g_wait_limit = 0;   // bc_mask_attn_backward_set_wait_limit (0: kWaitLimit)

}  // namespace

extern "C" {

bc_status bc_mask_attn_backward_query_bytes(int32_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t c,
                                            const int32_t* cu_prompt, const int32_t* cu_tokens, size_t* workspace_bytes) {
  if (!workspace_bytes) return BC_ERR_INVALID_ARG;
  try {
    Plan p;
    const bc_status st = make_plan(n_seqs, q_heads, kv_heads, head_dim, c, cu_prompt, cu_tokens, &p);
    if (st == BC_OK) *workspace_bytes = p.total;
    return st;
  } catch (...) {   // no host memory for the lists
    return BC_ERR_UNSUPPORTED;
  }
}

bc_status bc_mask_attn_backward(int32_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t c,
                                const int32_t* cu_prompt, const int32_t* cu_tokens, const void* prompt_k, const void* prompt_v,
                                const void* tok_q, const void* tok_k, const void* tok_v, const void* beacon_q, const void* beacon_k,
                                const void* beacon_v, const void* out_tok, const void* out_beacon, const float* lse_tok,
                                const float* lse_beacon, const void* d_out_tok, const void* d_out_beacon, void* d_prompt_k,
                                void* d_prompt_v, void* d_tok_q, void* d_tok_k, void* d_tok_v, void* d_beacon_q, void* d_beacon_k,
                                void* d_beacon_v, float sm_scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || !(sm_scale > 0.f)) return BC_ERR_INVALID_ARG;
  try {
    Plan p;
    const bc_status st = make_plan(n_seqs, q_heads, kv_heads, head_dim, c, cu_prompt, cu_tokens, &p);
    if (st != BC_OK) return st;
    if (workspace_bytes < p.total) return BC_ERR_INVALID_ARG;
    auto bad = [](std::initializer_list<const void*> v, int mask) {
      for (const void* x : v) if (!x || (reinterpret_cast<uintptr_t>(x) & mask)) return true;
      return false;
    };
    if ((p.prompts && (bad({prompt_k, prompt_v}, 15) || bad({d_prompt_k, d_prompt_v}, 31))) ||
        (p.tokens && (bad({tok_q, tok_k, tok_v, out_tok, d_out_tok}, 15) || bad({lse_tok}, 3) || bad({d_tok_q, d_tok_k, d_tok_v}, 31))) ||
        (p.beacons && (bad({beacon_q, beacon_k, beacon_v, out_beacon, d_out_beacon}, 15) || bad({lse_beacon}, 3) ||
                       bad({d_beacon_q, d_beacon_k, d_beacon_v}, 31))))
      return BC_ERR_INVALID_ARG;
    const int G = q_heads / kv_heads;
    cudaStream_t s = (cudaStream_t)stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (!encode_tiled()) return BC_ERR_CUDA;
    // the lists are pageable host memory: they have been staged when the calls return
    if (cudaMemsetAsync(ws, 0, 4, s) != cudaSuccess) return BC_ERR_CUDA;
    if (p.kv.empty()) return BC_OK;
    if (cudaMemcpyAsync(ws + p.at_kv, p.kv.data(), p.kv.size() * sizeof(KvItem), cudaMemcpyHostToDevice, s) != cudaSuccess ||
        (!p.q.empty() && cudaMemcpyAsync(ws + p.at_q, p.q.data(), p.q.size() * sizeof(QItem), cudaMemcpyHostToDevice, s) != cudaSuccess) ||
        (!p.join.empty() && cudaMemcpyAsync(ws + p.at_join, p.join.data(), p.join.size() * sizeof(JoinItem), cudaMemcpyHostToDevice, s) != cudaSuccess))
      return BC_ERR_CUDA;

    GradArgs a = {};
    a.lse2 = reinterpret_cast<float*>(ws + p.at_lse); a.delta = reinterpret_cast<float*>(ws + p.at_delta);
    a.rows = p.tokens + p.beacons; a.tok_rows = p.tokens;
    a.dk[0] = (__nv_bfloat16*)d_prompt_k; a.dk[1] = (__nv_bfloat16*)d_beacon_k; a.dk[2] = (__nv_bfloat16*)d_tok_k;
    a.dv[0] = (__nv_bfloat16*)d_prompt_v; a.dv[1] = (__nv_bfloat16*)d_beacon_v; a.dv[2] = (__nv_bfloat16*)d_tok_v;
    a.dq[0] = (__nv_bfloat16*)d_tok_q; a.dq[1] = (__nv_bfloat16*)d_beacon_q;
    a.partial = reinterpret_cast<float*>(ws + p.at_partial);
    a.status = reinterpret_cast<int32_t*>(ws);
    a.Hq = q_heads; a.Hkv = kv_heads; a.G = G; a.c = c;
    a.scale = sm_scale; a.scale_log2 = sm_scale * kLog2e;
    a.wait_limit = g_wait_limit ? g_wait_limit : kWaitLimit;
    const void* dummy = ws;   // arrays that do not exist get a map that is never used
    auto maps_for = [&](KvMaps* m, int q_box, int k_box) {
      const void* q[2] = {tok_q, beacon_q};
      const void* o[2] = {d_out_tok, d_out_beacon};
      const void* k[3] = {prompt_k, beacon_k, tok_k};
      const void* v[3] = {prompt_v, beacon_v, tok_v};
      const int64_t q_rows[2] = {p.tokens, p.beacons}, k_rows[3] = {p.prompts, p.beacons, p.tokens};
      bool ok = true;
      for (int i = 0; i < 2; ++i)
        ok = ok && map_3d(&m->q[i], q_rows[i] ? q[i] : dummy, q_heads, q_rows[i], G, q_box) &&
             map_3d(&m->o[i], q_rows[i] ? o[i] : dummy, q_heads, q_rows[i], G, q_box);
      for (int i = 0; i < 3; ++i)
        ok = ok && map_3d(&m->k[i], k_rows[i] ? k[i] : dummy, kv_heads, k_rows[i], 1, k_box) &&
             map_3d(&m->v[i], k_rows[i] ? v[i] : dummy, kv_heads, k_rows[i], 1, k_box);
      return ok;
    };
    KvMaps kv_maps, q_maps;
    if (!maps_for(&kv_maps, kHalf / G, kTile) || !maps_for(&q_maps, kTile / G, kHalf)) return BC_ERR_CUDA;
    const bool shortw = g_wait_limit != 0;
    const int kv_smem = 2 * kWide + kKvRing * 2 * kSlim + 1024, q_smem = 4 * kWide + kQRing * 2 * kSlim + 1024;
    auto* dkv = shortw ? k_dkv<true> : k_dkv<false>;
    auto* dq = shortw ? k_dq<true> : k_dq<false>;
    if (cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, kv_smem) != cudaSuccess ||
        cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, q_smem) != cudaSuccess)
      return BC_ERR_CUDA;
    const int sms = sm_count();
    if (a.rows > 0) {
      const int64_t blocks = (a.rows * q_heads + 15) / 16;
      k_delta<<<(unsigned)std::min<int64_t>(blocks, sms * 8), 256, 0, s>>>(
          (const uint4*)out_tok, (const uint4*)d_out_tok, lse_tok, (const uint4*)out_beacon, (const uint4*)d_out_beacon, lse_beacon, p.tokens,
          a.rows, q_heads, G, const_cast<float*>(a.lse2), const_cast<float*>(a.delta));
      GradArgs b = a;
      b.items = ws + p.at_q; b.n_items = (int32_t)p.q.size(); b.per = kTile / G;
      dq<<<std::min(b.n_items, sms), kThreads, q_smem, s>>>(b, q_maps);
    }
    a.items = ws + p.at_kv; a.n_items = (int32_t)p.kv.size(); a.per = kHalf / G;
    dkv<<<std::min(a.n_items, sms), kThreads, kv_smem, s>>>(a, kv_maps);
    if (!p.join.empty()) k_join<<<dim3((unsigned)p.join.size(), 2 * kTile / 8), 256, 0, s>>>(reinterpret_cast<const JoinItem*>(ws + p.at_join), a);
    return cudaGetLastError() == cudaSuccess ? BC_OK : BC_ERR_CUDA;
  } catch (...) {
    return BC_ERR_UNSUPPORTED;
  }
}

bc_status bc_mask_attn_backward_set_wait_limit(uint32_t polls) {
  g_wait_limit = polls;
  return BC_OK;
}

bc_status bc_mask_attn_backward_status(const void* workspace, void* stream, int32_t* code) {
  if (!workspace || !code) return BC_ERR_INVALID_ARG;
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return BC_ERR_CUDA;
  return cudaMemcpy(code, workspace, 4, cudaMemcpyDeviceToHost) == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}

}  // extern "C"
