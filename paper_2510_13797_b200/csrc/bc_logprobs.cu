// Log-probabilities of given tokens, with the entropy of every row and its most likely alternatives, and their gradient.
//
// A row x of logits with maximum m:   s = sum_j exp(x_j - m),  t = sum_j exp(x_j - m) (x_j - m)
//     log p_j = (x_j - m) - ln s,     H = - sum_j p_j log p_j = ln s - t / s
// and for g = d loss / d log p_target, h = d loss / d H:
//     d loss / d x_j = g [j = target] - p_j (g + h (log p_j + H)).
// The difference to the maximum is taken first and exactly, so large logits lose nothing; the maximum and ln s are kept
// apart for the gradient for the same reason.
//
// Forward: one pass over the row in memory.  A cluster of up to eight blocks has a row (304 KB for a vocabulary of 151,936 in
// bf16); every thread copies its 16-byte pieces to shared memory, all of them in flight at once, and folds each into a
// running (reference, s, t) as it lands.  What a thread copied only that thread reads, so the pieces need no barrier.
// The alternatives come from the copy in shared memory: the K / blocks-th largest of a block's threads' maxima is a value
// that at least K / blocks elements of the block reach, and the smallest of these over the blocks one that K elements of the
// row reach; the few elements that reach it (a hundred and some for K = 100) are gathered in the first block and ranked by
// counting.  Where more reach it than the buffer holds (many equal logits, or the large ones all with one thread), the
// cluster finds the K-th largest (value, index) pair bit by bit, counting in shared memory.
#include <cooperative_groups.h>

#include "bc_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxParts = 8;          // blocks per row
constexpr int kPartBytes = 4096;      // a block is given at least this much of a row
constexpr int kMaxTop = kThreads;     // alternatives per row
constexpr int kCands = 1024;          // elements that are ranked at most
constexpr int kMaxVocab = 262144;
constexpr int kIndexBits = 18;        // of a vocabulary index
constexpr float kFar = 0x1p126f;      // logits count as no further from 0 than this, so that differences stay finite
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 6.f;         // the reference follows the maximum when it is this far behind (exp(6) does not lose bits)

typedef unsigned long long F2;        // two fp32 numbers
__device__ __forceinline__ F2 pair(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(F2 v, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t max_bf2(uint32_t a, uint32_t b) {   // the number where one is a NaN
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t min_bf2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ float near(float x) { return fminf(fmaxf(x, -kFar), kFar); }   // NaN: -kFar

// The logits' type: elements per 16-byte piece, a piece as numbers, its largest element, keys that order as the numbers do.
template <bool F32>
struct Logits;
template <>
struct Logits<false> {
  static constexpr int kPer = 8, kBytes = 2, kKeyBits = 16;
  static constexpr uint32_t kFar2 = 0x7e807e80u;                         // kFar, twice
  __device__ static float load(const void* p, int64_t i) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); }
  __device__ static float top(const uint4& v) {
    const uint32_t m = max_bf2(max_bf2(v.x, v.y), max_bf2(v.z, v.w));
    return fmaxf(bf_lo(m), bf_hi(m));
  }
  __device__ static uint32_t clamp(uint32_t v) { return min_bf2(max_bf2(v, kFar2 | 0x80008000u), kFar2); }
  __device__ static void near_pairs(const uint4& v, F2* x) {
    const uint32_t w[4] = {clamp(v.x), clamp(v.y), clamp(v.z), clamp(v.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair(bf_lo(w[i]), bf_hi(w[i]));
  }
  __device__ static float element(const uint4& v, int i) {
    const uint32_t w = i < 4 ? (i < 2 ? v.x : v.y) : (i < 6 ? v.z : v.w);
    return (i & 1) ? bf_hi(w) : bf_lo(w);
  }
};
template <>
struct Logits<true> {
  static constexpr int kPer = 4, kBytes = 4, kKeyBits = 32;
  __device__ static float load(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
  __device__ static float top(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  __device__ static void near_pairs(const uint4& v, F2* x) {
    x[0] = pair(near(__uint_as_float(v.x)), near(__uint_as_float(v.y)));
    x[1] = pair(near(__uint_as_float(v.z)), near(__uint_as_float(v.w)));
  }
  __device__ static float element(const uint4& v, int i) { return __uint_as_float(i < 2 ? (i == 0 ? v.x : v.y) : (i == 2 ? v.z : v.w)); }
};

// Keys of kKeyBits bits; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key32(float x) {
  const uint32_t b = __float_as_uint(x != x ? -INFINITY : x + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key32_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k); }
template <bool F32>
__device__ __forceinline__ uint32_t key_of(float x) { return key32(x) >> (32 - Logits<F32>::kKeyBits); }
template <bool F32>
__device__ __forceinline__ float key_value(uint32_t k) {                 // a negative number's key ends in ones
  return F32 ? key32_value(k) : key32_value((k << 16) | ((k & 0x8000u) ? 0u : 0xffffu));
}
template <bool F32>
__device__ __forceinline__ unsigned long long place_of(float x, int i) {  // orders by value, then lowest index first
  return ((unsigned long long)key_of<F32>(x) << kIndexBits) | (unsigned)(kMaxVocab - 1 - i);
}

// Running sums relative to a reference.
struct Sums {
  float m, s, t;
  __device__ __forceinline__ void move(float to) {
    const float d = m - to, f = ex2(d * kLog2e);
    t = f * t + (f * d) * s;
    s *= f;
    m = to;
  }
  __device__ __forceinline__ void join(Sums o) {
    const float to = fmaxf(m, o.m);
    move(to);
    o.move(to);
    s += o.s;
    t += o.t;
  }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

struct LogprobArgs {
  const uint8_t* logits;
  int64_t row_bytes;
  int vocab, top_k;
  const int64_t* targets;
  float *logprob, *entropy, *stats, *top_logprob;
  int32_t* top_idx;
};

template <bool F32>
__global__ void __launch_bounds__(kThreads, 4) k_logprobs(const LogprobArgs a) {
  using L = Logits<F32>;
  extern __shared__ __align__(16) uint4 piece[];           // this block's share of the row
  __shared__ unsigned long long cand[kCands];              // the first block's: the elements to be ranked
  __shared__ Sums warp_sums[kWarps];
  __shared__ Sums block_sums;
  __shared__ uint32_t block_key;
  __shared__ int n_cand, counts[2];
  cg::cluster_group cluster = cg::this_cluster();
  const int part = (int)cluster.block_rank(), parts = (int)cluster.num_blocks();
  const int64_t r = blockIdx.x / parts;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, vocab = a.vocab;
  const uint8_t* row = a.logits + r * a.row_bytes;
  // elements ahead of the first 16-byte boundary and behind the last are taken one by one, by threads of the first and last block
  const int head = min(vocab, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / L::kBytes);
  const int pieces = (vocab - head) / L::kPer, tail0 = head + pieces * L::kPer;
  const int per = (pieces + parts - 1) / parts, p0 = min(pieces, part * per), mine = min(pieces, p0 + per) - p0;
  const uint4* src = reinterpret_cast<const uint4*>(row + head * L::kBytes) + p0;

  if (tid == 0) n_cand = 0;
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(piece);
  const int quarter = (mine + 4 * kThreads - 1) / (4 * kThreads) * kThreads;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    for (int i = g * quarter + tid; i < min(mine, (g + 1) * quarter); i += kThreads) copy16(dst + i * 16, src + i);
    copies_begun();
  }
  int extra_at = -1;
  if (part == 0 && tid < head) extra_at = tid;
  if (part == parts - 1 && tid >= 32 && tail0 + tid - 32 < vocab) extra_at = tail0 + tid - 32;
  const float extra = extra_at >= 0 ? L::load(row, extra_at) : -INFINITY;

  Sums st = {-kFar, 0.f, 0.f};
  float best = -INFINITY;                                  // of this thread's elements
  F2 s2 = pair(0.f, 0.f), t2 = s2;
  const F2 log2e2 = pair(kLog2e, kLog2e);
  auto fold = [&](int g) {
    for (int i = g * quarter + tid; i < min(mine, (g + 1) * quarter); i += kThreads) {
      const uint4 v = piece[i];
      const float top = L::top(v);
      best = fmaxf(best, top);
      if (near(top) > st.m + kSlack) {
        float s0, s1, t0, t1;
        split(s2, &s0, &s1); split(t2, &t0, &t1);
        st.s = s0 + s1; st.t = t0 + t1;
        st.move(near(top));
        s2 = pair(st.s, 0.f); t2 = pair(st.t, 0.f);
      }
      const F2 minus = pair(-st.m, -st.m);
      F2 x[L::kPer / 2];
      L::near_pairs(v, x);
#pragma unroll
      for (int k = 0; k < L::kPer / 2; ++k) {
        const F2 d = add2(x[k], minus);
        float y0, y1;
        split(mul2(d, log2e2), &y0, &y1);
        const F2 e = pair(ex2(y0), ex2(y1));
        s2 = add2(s2, e);
        t2 = fma2(e, d, t2);
      }
    }
  };
  copies_landed<3>(); fold(0);
  copies_landed<2>(); fold(1);
  copies_landed<1>(); fold(2);
  copies_landed<0>(); fold(3);
  {
    float s0, s1, t0, t1;
    split(s2, &s0, &s1); split(t2, &t0, &t1);
    st.s = s0 + s1; st.t = t0 + t1;
  }
  if (extra_at >= 0) {
    best = fmaxf(best, extra);
    st.join({near(extra), 1.f, 0.f});
  }
  if (best > -kFar) st.move(near(best));                   // from the reference, which may lie behind, to the maximum itself
  else st = {-kFar, 0.f, 0.f};                             // nothing but -inf and NaN: no mass

#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const Sums o = {__shfl_xor_sync(0xffffffffu, st.m, d), __shfl_xor_sync(0xffffffffu, st.s, d), __shfl_xor_sync(0xffffffffu, st.t, d)};
    st.join(o);
  }
  if (lane == 0) warp_sums[warp] = st;
  uint32_t bound = 0;                                      // key that enough threads' maxima reach
  if (a.top_k > 0) {
    const int need = (a.top_k + parts - 1) / parts;
    const uint32_t k = key_of<F32>(best);
#pragma unroll 1
    for (int b = L::kKeyBits - 1; b >= 0; --b) {
      const uint32_t trial = bound | (1u << b);
      if (__syncthreads_count(k >= trial) >= need) bound = trial;
    }
  }
  __syncthreads();
  if (tid == 0) {
    Sums all = warp_sums[0];
    for (int w = 1; w < kWarps; ++w) all.join(warp_sums[w]);
    block_sums = all;
    block_key = bound;
  }
  cluster.sync();
  if (part == 0 && tid == 0) {
    Sums all = block_sums;
    for (int p = 1; p < parts; ++p) all.join(*cluster.map_shared_rank(&block_sums, p));
    const bool some = all.m > -kFar;
    const float ls = some ? logf(all.s) : 0.f, m = some ? all.m : -INFINITY;
    warp_sums[0] = {m, ls, 0.f};                           // for the alternatives
    if (a.stats) { a.stats[2 * r] = m; a.stats[2 * r + 1] = ls; }
    if (a.entropy) a.entropy[r] = some ? fmaxf(ls - all.t / all.s, 0.f) : 0.f;
    if (a.logprob) {
      const int64_t t = a.targets[r];
      float lp = 0.f;                                      // no token is given for this row
      if (t >= 0 && t < vocab) {
        const float x = L::load(row, t);
        lp = x > -kFar ? (near(x) - m) - ls : -INFINITY;
      }
      a.logprob[r] = lp;
    }
  }
  if (a.top_k == 0) {
    cluster.sync();                                        // no block leaves while its sums may still be read
    return;
  }

  // ---- the elements that reach the bound, to the first block ---------------------------------------------------------------
  bound = block_key;
  for (int p = 0; p < parts; ++p) bound = min(bound, *cluster.map_shared_rank(&block_key, p));
  int* total = cluster.map_shared_rank(&n_cand, 0);
  unsigned long long* to = cluster.map_shared_rank(cand, 0);
  // calls f(value, index) for every element of this thread that may reach `least` (a NaN does so where nothing else counts)
  auto each = [&](float least, auto f) {
    for (int i = tid; i < mine; i += kThreads) {
      const uint4 v = piece[i];
      if (!(L::top(v) < least)) {
        const int at = head + (p0 + i) * L::kPer;
#pragma unroll
        for (int k = 0; k < L::kPer; ++k) {
          const float x = L::element(v, k);
          if (!(x < least)) f(x, at + k);
        }
      }
    }
    if (extra_at >= 0 && !(extra < least)) f(extra, extra_at);
  };
  const uint32_t lowest = key_of<F32>(-INFINITY);
  auto push = [&](unsigned long long least) {              // two steps: the place of every element, then its store
    const uint32_t key = (uint32_t)(least >> kIndexBits);
    each(key <= lowest ? -INFINITY : key_value<F32>(key), [&](float x, int i) {
      const unsigned long long c = place_of<F32>(x, i);
      if (c >= least) {
        const int at = atomicAdd(total, 1);
        if (at < kCands) to[at] = c;
      }
    });
  };
  push((unsigned long long)bound << kIndexBits);
  cluster.sync();
  int found = *total;
  cluster.sync();                                          // everyone has read it
  if (found > kCands) {
    // the K-th largest (value, index) pair, bit by bit; any pair that K to kCands elements reach will do
    unsigned long long least = 0;
    int turn = 0;
    for (int b = L::kKeyBits + kIndexBits - 1; b >= 0; --b) {
      const unsigned long long trial = least | (1ull << b);
      const uint32_t key = (uint32_t)(trial >> kIndexBits);
      int mine_n = 0;
      each(key <= lowest ? -INFINITY : key_value<F32>(key), [&](float x, int i) { mine_n += place_of<F32>(x, i) >= trial; });
      mine_n = __reduce_add_sync(0xffffffffu, mine_n);
      if (tid == 0) counts[turn] = 0;
      __syncthreads();
      if (lane == 0) atomicAdd(&counts[turn], mine_n);
      cluster.sync();
      found = 0;
      for (int p = 0; p < parts; ++p) found += *cluster.map_shared_rank(&counts[turn], p);
      turn ^= 1;                                           // a block may begin the next count while another reads this one
      if (found >= a.top_k) least = trial;
      if (found >= a.top_k && found <= kCands) break;
    }
    if (part == 0 && tid == 0) n_cand = 0;
    cluster.sync();
    push(least);
    cluster.sync();
    found = *total;
    cluster.sync();
  }
  if (part != 0) return;
  // ---- rank them: a place is larger than exactly those behind it -----------------------------------------------------------
  const float m = warp_sums[0].m, ls = warp_sums[0].s;
  for (int i = tid; i < found; i += kThreads) {
    const unsigned long long c = cand[i];
    int rank = 0;
    for (int j = 0; j < found; ++j) rank += cand[j] > c;
    if (rank < a.top_k) {
      const float x = key_value<F32>((uint32_t)(c >> kIndexBits));
      a.top_idx[r * a.top_k + rank] = kMaxVocab - 1 - (int)(c & (kMaxVocab - 1));
      a.top_logprob[r * a.top_k + rank] = x > -kFar ? (near(x) - m) - ls : -INFINITY;
    }
  }
}

struct LogprobGradArgs {
  const uint8_t* logits;
  uint8_t* grad;
  int64_t row_bytes, grad_row_bytes;
  int vocab, spans;                     // blocks per row
  const int64_t* targets;
  const float *stats, *entropy, *d_logprob, *d_entropy;
};

// The gradient: every element read and written once.  A block has kSpan pieces of a row, four per thread, all loads in flight
// before the row's numbers are needed.  Where logits and gradient do not lie alike to 16 bytes, the loads are element by
// element (whole lines, from the first-level cache) and the stores still 16 bytes.
constexpr int kSpan = 4 * kThreads;
template <bool F32>
__global__ void __launch_bounds__(kThreads) k_logprobs_grad(const LogprobGradArgs a) {
  using L = Logits<F32>;
  const int64_t r = blockIdx.x / a.spans;
  const int span = (int)(blockIdx.x - r * a.spans), tid = threadIdx.x, vocab = a.vocab;
  const uint8_t* row = a.logits + r * a.row_bytes;
  uint8_t* out = a.grad + r * a.grad_row_bytes;
  const int head = min(vocab, (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / L::kBytes);
  const int pieces = (vocab - head) / L::kPer, tail0 = head + pieces * L::kPer;
  const bool alike = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
  const int64_t given = a.targets ? a.targets[r] : -1;
  const int target = given >= 0 && given < vocab ? (int)given : -1;
  const float g = a.d_logprob && target >= 0 ? a.d_logprob[r] : 0.f;
  const float h = a.d_entropy ? a.d_entropy[r] : 0.f;
  const float m = a.stats[2 * r], ls = a.stats[2 * r + 1];
  const bool none = (g == 0.f && h == 0.f) || !(m > -INFINITY);      // the row's gradient is zero: its logits are not read
  const float c0 = a.d_entropy ? fmaf(h, a.entropy[r], g) : g;
  auto of = [&](float x, int j) {
    // between the maximum (+inf counts as kFar) and a distance at which the weight is 0 (-inf and NaN)
    const float lp = fminf(fmaxf(x - m, -1e5f), 0.f) - ls;
    const float p = ex2(lp * kLog2e);
    return (j == target ? g : 0.f) - p * fmaf(h, lp, c0);
  };
  auto store1 = [&](int j) {
    const float v = none ? 0.f : of(L::load(row, j), j);
    if (F32) reinterpret_cast<float*>(out)[j] = v;
    else reinterpret_cast<__nv_bfloat16*>(out)[j] = __float2bfloat16_rn(v);
  };
  if (span == 0 && tid < head) store1(tid);
  if (span == a.spans - 1 && tid >= 32 && tail0 + tid - 32 < vocab) store1(tail0 + tid - 32);
  uint4 v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = span * kSpan + k * kThreads + tid;
    v[k] = make_uint4(0, 0, 0, 0);
    if (i < pieces && !none) {
      const int j = head + i * L::kPer;
      if (alike) {
        v[k] = __ldcs(reinterpret_cast<const uint4*>(row + (int64_t)j * L::kBytes));
      } else if (F32) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(row) + j;
        v[k] = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        const uint16_t* w = reinterpret_cast<const uint16_t*>(row) + j;
        v[k] = make_uint4(w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16, w[4] | (uint32_t)w[5] << 16, w[6] | (uint32_t)w[7] << 16);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = span * kSpan + k * kThreads + tid;
    if (i >= pieces) break;
    const int j = head + i * L::kPer;
    uint4 o = make_uint4(0, 0, 0, 0);
    if (!none) {
      float y[L::kPer];
#pragma unroll
      for (int e = 0; e < L::kPer; ++e) y[e] = of(L::element(v[k], e), j + e);
      if (F32) {
        o = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
      } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(y[(2 * e) % L::kPer], y[(2 * e + 1) % L::kPer]);
          w[e] = *reinterpret_cast<const uint32_t*>(&t);
        }
        o = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    __stcs(reinterpret_cast<uint4*>(out + (int64_t)j * L::kBytes), o);
  }
}

bc_status check(const void* logits, int32_t f32, int64_t row_stride, int32_t n, int32_t vocab) {
  if (!logits || n <= 0 || vocab <= 0 || row_stride < vocab || (f32 != 0 && f32 != 1)) return BC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) & (f32 ? 3 : 1)) return BC_ERR_INVALID_ARG;
  if (vocab > kMaxVocab) return BC_ERR_UNSUPPORTED;
  return BC_OK;
}

template <bool F32>
bc_status launch_logprobs(const LogprobArgs& a, int n, cudaStream_t s) {
  using L = Logits<F32>;
  // as many blocks per row as have kPartBytes each
  int parts = 1;
  while (parts < kMaxParts && (int64_t)a.vocab * L::kBytes >= 2 * parts * kPartBytes) parts *= 2;
  if ((int64_t)n * parts > 0x7fffffff) return BC_ERR_UNSUPPORTED;
  const int pieces = a.vocab / L::kPer, per = (pieces + parts - 1) / parts;
  const int most = (kMaxVocab / L::kPer + kMaxParts - 1) / kMaxParts * 16;
  // the opt-in is always that of the largest vocabulary: a setting that followed the call could be lowered under another thread's
  if (cudaFuncSetAttribute(k_logprobs<F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) return BC_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n * parts)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = (size_t)per * 16; cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_logprobs<F32>, a) == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}

}  // namespace

extern "C" {

bc_status bc_token_logprobs(const void* logits, int32_t logits_f32, int64_t row_stride, int32_t n, int32_t vocab, const int64_t* targets,
                            int32_t top_k, float* logprob, float* entropy, float* stats, int32_t* top_idx, float* top_logprob,
                            void* stream) {
  const bc_status st = check(logits, logits_f32, row_stride, n, vocab);
  if (st) return st;
  if (top_k < 0 || top_k > vocab || (top_k > 0 && (!top_idx || !top_logprob)) || (logprob && !targets)) return BC_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(logprob) | reinterpret_cast<uintptr_t>(entropy) | reinterpret_cast<uintptr_t>(stats) |
        reinterpret_cast<uintptr_t>(top_idx) | reinterpret_cast<uintptr_t>(top_logprob)) & 3) || (reinterpret_cast<uintptr_t>(targets) & 7))
    return BC_ERR_INVALID_ARG;
  if (top_k > kMaxTop) return BC_ERR_UNSUPPORTED;
  if (!logprob && !entropy && !stats && top_k == 0) return BC_OK;
  LogprobArgs a;
  a.logits = (const uint8_t*)logits; a.row_bytes = row_stride * (logits_f32 ? 4 : 2);
  a.vocab = vocab; a.top_k = top_k; a.targets = targets;
  a.logprob = logprob; a.entropy = entropy; a.stats = stats; a.top_logprob = top_logprob; a.top_idx = top_idx;
  return logits_f32 ? launch_logprobs<true>(a, n, (cudaStream_t)stream) : launch_logprobs<false>(a, n, (cudaStream_t)stream);
}

bc_status bc_token_logprobs_backward(const void* logits, int32_t logits_f32, int64_t row_stride, int32_t n, int32_t vocab,
                                     const int64_t* targets, const float* stats, const float* entropy, const float* d_logprob,
                                     const float* d_entropy, void* grad, int64_t grad_row_stride, void* stream) {
  const bc_status st = check(logits, logits_f32, row_stride, n, vocab);
  if (st) return st;
  if (!stats || !grad || grad_row_stride < vocab || (d_logprob && !targets) || (d_entropy && !entropy) || (!d_logprob && !d_entropy))
    return BC_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(grad) & (logits_f32 ? 3 : 1)) || (reinterpret_cast<uintptr_t>(targets) & 7) ||
      ((reinterpret_cast<uintptr_t>(stats) | reinterpret_cast<uintptr_t>(entropy) | reinterpret_cast<uintptr_t>(d_logprob) |
        reinterpret_cast<uintptr_t>(d_entropy)) & 3))
    return BC_ERR_INVALID_ARG;
  const int bytes = logits_f32 ? 4 : 2, pieces = vocab / (16 / bytes);
  LogprobGradArgs a;
  a.logits = (const uint8_t*)logits; a.grad = (uint8_t*)grad;
  a.row_bytes = row_stride * bytes; a.grad_row_bytes = grad_row_stride * bytes;
  a.vocab = vocab; a.spans = pieces > 0 ? (pieces + kSpan - 1) / kSpan : 1;
  a.targets = targets; a.stats = stats; a.entropy = entropy; a.d_logprob = d_logprob; a.d_entropy = d_entropy;
  if ((int64_t)n * a.spans > 0x7fffffff) return BC_ERR_UNSUPPORTED;
  if (logits_f32) k_logprobs_grad<true><<<(unsigned)(n * a.spans), kThreads, 0, (cudaStream_t)stream>>>(a);
  else k_logprobs_grad<false><<<(unsigned)(n * a.spans), kThreads, 0, (cudaStream_t)stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}

}  // extern "C"
