// Sampling of the next token from a row of logits, with temperature, top-k, top-p and min-p, from a given uniform
// random number per row (Algorithm 1 samples the next token from the model's distribution; bc_argmax is the greedy
// choice).  For a row x with maximum m and temperature T > 0:
//     e_j = exp((x_j - m) / T)
//     K   = the top_k largest x_j (of equal ones the lowest indices)                          [top_k on]
//     N   = the shortest prefix of K, largest first, whose mass reaches top_p * mass(K)       [top_p on]
//     S   = the elements of N with e_j >= min_p                                               [min_p on]
//     token = the first j of S in index order with sum_{i in S, i <= j} e_i > u * mass(S).
//
// Masses are sums of INTEGERS: e_j, evaluated in double precision, is rounded to a multiple of 2^-45, so a row of up
// to 2^18 elements adds up exactly in 64 bits, in any order -- the split over threads and blocks and the order of
// the shared-memory atomics cannot change a result.  What the rounding drops is at most 2^-46 of the largest weight per
// element; an element that rounds to zero is never chosen.
//
// One cluster of eight thread blocks per row (a batch of 64 rows is too few blocks otherwise, and a single row still
// gets eight SMs).  Each block copies its slice of the row into shared memory, the only time the row is read from
// memory, and everything after works on the slices, joined through distributed shared memory:
//   1. maximum of the row (and its lowest index: the greedy answer);
//   2. with top-k or top-p: the threshold key, by a histogram of counts and masses over 512 bins of (m - x) / T, 1/11
//      octave wide (logits spread over many of them, so the atomics rarely collide), then, inside the bin in which
//      the limit is crossed, by histograms over the keys' own bits until the bin holds one key; elements that equal
//      the threshold are kept lowest index first, as many as the limit needs;
//   3. the kept mass of every thread's run of elements, a prefix sum over threads and blocks, and the element in
//      which u * mass falls.
// Bound by the latency of these steps (two cluster barriers without top-k and top-p, about four more with one of them),
// not by the 300 KB a row has.
#include <cooperative_groups.h>

#include "bc_common.cuh"

namespace cg = cooperative_groups;

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int kBins = 512;
constexpr int kMaxVocab = 1 << 18;     // 2^18 weights of at most 2^45 add up in 63 bits
constexpr int kWeightBits = 45;
static_assert(kBins == 2 * kThreads, "a thread scans two bins");

struct Sum2 {   // a mass and a count, added up together
  u64 mass;
  uint32_t count;
};
__device__ __forceinline__ Sum2 operator+(const Sum2& a, const Sum2& b) { return {a.mass + b.mass, a.count + b.count}; }

// Exclusive prefix over the block's threads; *total gets the block's sum.  All threads call.
__device__ __forceinline__ Sum2 block_scan(Sum2 x, Sum2* total) {
  __shared__ u64 sh_mass[kWarps];
  __shared__ uint32_t sh_count[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sum2 incl = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 m = __shfl_up_sync(0xffffffffu, incl.mass, d);
    const uint32_t c = __shfl_up_sync(0xffffffffu, incl.count, d);
    if (lane >= d) { incl.mass += m; incl.count += c; }
  }
  __syncthreads();   // the last call's readers are done
  if (lane == 31) { sh_mass[warp] = incl.mass; sh_count[warp] = incl.count; }
  __syncthreads();
  Sum2 before = {0, 0}, all = {0, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const Sum2 v = {sh_mass[w], sh_count[w]};
    if (w < warp) before = before + v;
    all = all + v;
  }
  *total = all;
  return {before.mass + incl.mass - x.mass, before.count + incl.count - x.count};
}

template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
  static constexpr int kVec = 8;
  // element i of a 16-byte piece, NaN read as -inf
  __device__ static __forceinline__ float get(const uint4& v, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&v)[i >> 1];
    const float f = __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
    return f == f ? f + 0.f : -INFINITY;   // + 0: the two zeros are one value
  }
  __device__ static __forceinline__ __nv_bfloat16 none() { return __ushort_as_bfloat16(0xff80); }
};
template <> struct Raw<float> {
  static constexpr int kVec = 4;
  __device__ static __forceinline__ float get(const uint4& v, int i) {
    const float f = __uint_as_float(reinterpret_cast<const uint32_t*>(&v)[i]);
    return f == f ? f + 0.f : -INFINITY;
  }
  __device__ static __forceinline__ float none() { return -INFINITY; }
};

// order-preserving key of a float (no NaN, one zero), and back
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

struct Scale {
  float top;      // the row's maximum
  double c;       // log2(e) / T
  float bins;     // 11 bins per octave
  double min_p;
  // e(x) in double precision; 0 where it is far below the weights' resolution
  __device__ __forceinline__ double e(float x) const {
    if (x == top) return 1.0;
    const double t = ((double)top - (double)x) * c;
    return t < (double)(kWeightBits + 2) ? exp2(-t) : 0.0;    // also 0 for inf * 0
  }
  __device__ __forceinline__ u64 fixed(double e) const { return __double2ull_rn(e * (double)(1ull << kWeightBits)); }
  __device__ __forceinline__ u64 weight(float x) const { return fixed(e(x)); }
  __device__ __forceinline__ u64 kept_weight(float x) const {   // 0 below min_p
    const double v = e(x);
    return v >= min_p ? fixed(v) : 0;
  }
  __device__ __forceinline__ int bin(float x) const { return min(kBins - 1, (int)((top - x) * bins)); }
};

struct Shared {
  u64 mass[2][kBins];            // histograms: two, used in turn (one may still be read by other blocks)
  uint32_t count[2][kBins];
  uint32_t key_lo[2], key_hi[2];
  float best;                    // this block's maximum and its lowest index
  int at;
  Sum2 part;                     // this block's mass above the threshold and number of elements at it
  // results of a search, for the whole block
  int cross_bin;
  Sum2 cross_before, cross_in;
  int owner;
  u64 owner_skip;
  uint32_t owner_ties;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(const T* __restrict__ logits, int64_t row_stride, int vocab,
                                                     const float* __restrict__ temperature, const int32_t* __restrict__ top_k,
                                                     const float* __restrict__ top_p, const float* __restrict__ min_p,
                                                     const float* __restrict__ uniform, long long* __restrict__ out) {
  constexpr int kVec = Raw<T>::kVec;
  extern __shared__ uint4 slice[];
  __shared__ Shared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int part = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = blockIdx.x / kCluster;
  const T* row = logits + r * row_stride;

  // ---- the slice: elements [first, first + cnt) of the row, kept at their 16-byte phase ---------------------------
  const int per = (vocab + kCluster * kVec - 1) / (kCluster * kVec) * kVec;
  const int first = min(part * per, vocab), cnt = min(vocab - first, per);
  const int phase = (int)((reinterpret_cast<uintptr_t>(row + first) & 15) / sizeof(T));
  const int pieces = cnt > 0 ? (phase + cnt + kVec - 1) / kVec : 0;
  T* flat = reinterpret_cast<T*>(slice);
  float best = -INFINITY;
  int at = 0x7fffffff;
  auto take = [&](float v, int i) { if (v > best || (v == best && i < at)) { best = v; at = i; } };
  for (int p = tid; p < pieces; p += kThreads) {
    const int e0 = p * kVec - phase;               // element of the slice in which the piece begins
    uint4 v;
    if (e0 >= 0 && e0 + kVec <= cnt) {
      v = __ldcs(reinterpret_cast<const uint4*>(row + first + e0));
      slice[p] = v;
    } else {                                       // the row's ends: only what belongs to it is read
      for (int i = 0; i < kVec; ++i) flat[p * kVec + i] = e0 + i >= 0 && e0 + i < cnt ? row[first + e0 + i] : Raw<T>::none();
      v = slice[p];
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (e0 + i >= 0 && e0 + i < cnt) take(Raw<T>::get(v, i), first + e0 + i);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const float v = __shfl_xor_sync(0xffffffffu, best, d);
    const int i = __shfl_xor_sync(0xffffffffu, at, d);
    take(v, i);
  }
  __shared__ float warp_best[kWarps];
  __shared__ int warp_at[kWarps];
  if (lane == 0) { warp_best[warp] = best; warp_at[warp] = at; }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) take(warp_best[w], warp_at[w]);
    sh.best = best; sh.at = at;
  }
  for (int b = tid; b < kBins; b += kThreads) { sh.mass[0][b] = 0; sh.count[0][b] = 0; }
  cluster.sync();
  best = -INFINITY; at = 0x7fffffff;
  for (int b = 0; b < kCluster; ++b) take(*cluster.map_shared_rank(&sh.best, b), *cluster.map_shared_rank(&sh.at, b));

  const float temp = temperature != nullptr ? temperature[r] : 1.f;
  if (!(temp > 0.f) || best == -INFINITY) {        // greedy; a row without a finite element: its first index, as bc_argmax
    if (part == 0 && tid == 0) out[r] = at == 0x7fffffff ? 0 : at;
    cluster.sync();                                // no block leaves while its shared memory may still be read
    return;
  }
  Scale sc;
  sc.top = best;
  sc.c = 1.4426950408889634 / (double)temp;
  sc.bins = (float)(11.0 * sc.c);
  const float mp = min_p != nullptr ? min_p[r] : 0.f;
  sc.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;   // at most 1: the largest element is always kept
  const int k = top_k != nullptr ? top_k[r] : 0;
  const float p = top_p != nullptr ? top_p[r] : 1.f;
  const bool by_count = k > 0 && k < vocab, by_mass = p < 1.f;

  // ---- threshold: keep every key above thr and the first `ties` elements (in index order) that equal it ------------
  uint32_t thr = 0;
  u64 ties = 0;                                     // with no limit: every key is above 0, the key no float has
  int round = 0;                                    // histograms filled so far, which of the two is next
  // Adds the cluster's histograms up (this thread: bins 2 tid, 2 tid + 1).
  auto totals = [&](int which, Sum2* b0, Sum2* b1) {
    *b0 = {0, 0}; *b1 = {0, 0};
#pragma unroll
    for (int b = 0; b < kCluster; ++b) {
      const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(cluster.map_shared_rank(&sh.mass[which][2 * tid], b));
      const uint2 c = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sh.count[which][2 * tid], b));
      b0->mass += m.x; b1->mass += m.y; b0->count += c.x; b1->count += c.y;
    }
  };
  // The bin in which the running count (or mass), largest keys first, reaches `limit`: false if it never does.
  auto cross = [&](const Sum2& b0, const Sum2& b1, const Sum2& before0, bool count, u64 limit, Sum2* all) {
    if (tid == 0) sh.cross_bin = -1;
    Sum2 e0 = block_scan(b0 + b1, all);             // its barriers order the store above
    e0 = e0 + before0;
    const Sum2 e1 = e0 + b0, e2 = e1 + b1;
    auto val = [&](const Sum2& s) { return count ? (u64)s.count : s.mass; };
    if (val(e0) < limit && limit <= val(e1)) { sh.cross_bin = 2 * tid; sh.cross_before = e0; sh.cross_in = b0; }
    if (val(e1) < limit && limit <= val(e2)) { sh.cross_bin = 2 * tid + 1; sh.cross_before = e1; sh.cross_in = b1; }
    __syncthreads();
    return sh.cross_bin >= 0;
  };
  if (by_count || by_mass) {
    for (int q = tid; q < pieces; q += kThreads) {
      const uint4 v = slice[q];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float x = Raw<T>::get(v, i);
        const u64 w = sc.weight(x);
        if (w) {
          const int b = sc.bin(x);
          atomicAdd(&sh.mass[0][b], w);
          atomicAdd(&sh.count[0][b], 1u);
        }
      }
    }
    cluster.sync();
    Sum2 l0, l1, all;
    totals(0, &l0, &l1);
    round = 1;
    // From the bin that cross() found to the key: histograms over the bits in which the bin's keys differ.
    auto refine = [&](bool count, u64 limit, Sum2* before, Sum2* in) {
      const int bin = sh.cross_bin;
      *before = sh.cross_before;
      *in = sh.cross_in;
      uint32_t lo = 0, hi = 0xffffffffu;
      for (;;) {
        uint32_t mn = 0xffffffffu, mx = 0;
        for (int q = tid; q < pieces; q += kThreads) {
          const uint4 v = slice[q];
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const float x = Raw<T>::get(v, i);
            const uint32_t key = key_of(x);
            if (key >= lo && key <= hi && sc.bin(x) == bin && sc.weight(x)) { mn = min(mn, key); mx = max(mx, key); }
          }
        }
        const int which = round & 1;
        if (tid == 0) { sh.key_lo[which] = 0xffffffffu; sh.key_hi[which] = 0; }
        for (int b = tid; b < kBins; b += kThreads) { sh.mass[which][b] = 0; sh.count[which][b] = 0; }
        __syncthreads();
        if (mn <= mx) { atomicMin(&sh.key_lo[which], mn); atomicMax(&sh.key_hi[which], mx); }
        cluster.sync();
        mn = 0xffffffffu; mx = 0;
#pragma unroll
        for (int b = 0; b < kCluster; ++b) {
          mn = min(mn, *cluster.map_shared_rank(&sh.key_lo[which], b));
          mx = max(mx, *cluster.map_shared_rank(&sh.key_hi[which], b));
        }
        if (mn >= mx) { ++round; return mx; }        // one key: the threshold
        const int shift = max(0, 32 - __clz(mx - mn) - 9);   // (mx - mn) >> shift is below 512
        for (int q = tid; q < pieces; q += kThreads) {
          const uint4 v = slice[q];
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const float x = Raw<T>::get(v, i);
            const uint32_t key = key_of(x);
            if (key >= mn && key <= mx && sc.bin(x) == bin) {
              const u64 w = sc.weight(x);
              if (w) {
                const int b = (int)((mx - key) >> shift);
                atomicAdd(&sh.mass[which][b], w);
                atomicAdd(&sh.count[which][b], 1u);
              }
            }
          }
        }
        cluster.sync();
        Sum2 b0, b1, sub;
        totals(which, &b0, &b1);
        ++round;
        cross(b0, b1, *before, count, limit, &sub);
        *before = sh.cross_before;
        *in = sh.cross_in;
        const uint32_t b = (uint32_t)sh.cross_bin;
        hi = mx - (b << shift);
        lo = max(mn, hi - ((1u << shift) - 1u));
        __syncthreads();                             // sh.cross_* have been read
      }
    };
    bool cut = false;
    Sum2 before, in;
    u64 mass = 0;
    if (by_count) {
      cut = cross(l0, l1, Sum2{0, 0}, true, (u64)k, &all);
      mass = all.mass;
      if (cut) {
        thr = refine(true, (u64)k, &before, &in);
        ties = (u64)k - before.count;
        mass = before.mass + ties * sc.weight(of_key(thr));
      }
    }
    if (by_mass) {
      __syncthreads();
      if (!cut) { block_scan(l0 + l1, &all); mass = all.mass; }
      const double want = ceil((double)p * (double)mass);
      const u64 limit = want >= 1.0 ? (u64)want : 1;   // the largest element is always kept; NaN never comes here
      if (cross(l0, l1, Sum2{0, 0}, false, limit, &all)) {
        thr = refine(false, limit, &before, &in);
        const u64 w = sc.weight(of_key(thr));
        ties = (limit - before.mass + w - 1) / w;
      }
    }
  }

  // ---- the draw ---------------------------------------------------------------------------------------------------
  // Thread t takes a run of consecutive pieces, so that threads are in index order; an odd run keeps the 16-byte
  // reads of neighbouring threads off one another's banks.
  const int run = ((per / kVec + 1 + kThreads - 1) / kThreads) | 1;
  const u64 tie_weight = thr != 0 ? sc.kept_weight(of_key(thr)) : 0;
  Sum2 mine = {0, 0};                                // mass above the threshold, elements at it
  for (int q = tid * run; q < min(pieces, (tid + 1) * run); ++q) {
    const uint4 v = slice[q];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float x = Raw<T>::get(v, i);
      const uint32_t key = key_of(x);
      if (key > thr) mine.mass += sc.kept_weight(x);
      mine.count += key == thr;
    }
  }
  Sum2 block_all;
  const Sum2 mine_before = block_scan(mine, &block_all);
  if (tid == 0) sh.part = block_all;
  cluster.sync();
  u64 skip = 0, all_mass = 0, my_skip = 0, my_mass = 0, my_tied = 0, tied = 0;
  for (int b = 0; b < kCluster; ++b) {
    const Sum2* o = cluster.map_shared_rank(&sh.part, b);
    const u64 here = o->count, kept = tied >= ties ? 0 : (here < ties - tied ? here : ties - tied);
    const u64 m = o->mass + kept * tie_weight;
    if (b == part) { my_skip = all_mass; my_tied = tied; my_mass = m; }
    all_mass += m;
    tied += here;
  }
  float u = uniform[r];
  u = u > 0.f ? fminf(u, 0.99999994f) : 0.f;         // NaN and negatives count as 0
  const u64 point = (u64)((double)u * (double)all_mass);   // the first running sum ABOVE u * mass is the first above its floor
  if (point >= my_skip && point < my_skip + my_mass) {     // this block holds the element (uniform over the block)
    // mass of the threads before this one in the block, ties kept lowest index first
    auto kept_ties = [&](u64 t0, u64 t1) { return min(t1, ties) - min(t0, ties); };
    const u64 t0 = my_tied + mine_before.count, t1 = t0 + mine.count;
    skip = my_skip + mine_before.mass + kept_ties(my_tied, t0) * tie_weight;
    const u64 own = mine.mass + kept_ties(t0, t1) * tie_weight;
    if (point >= skip && point < skip + own) { sh.owner = tid; sh.owner_skip = skip; sh.cross_before.mass = t0; }
    __syncthreads();
    const int owner = sh.owner;
    skip = sh.owner_skip;
    const u64 tie0 = sh.cross_before.mass;
    // the owner's run, one element per thread (a run has at most 17 pieces of 8 or 33 of 4 elements)
    const int e = owner * run * kVec + tid, end = min(pieces, (owner + 1) * run) * kVec;
    Sum2 one = {0, 0};
    if (e < end) {
      const float x = Raw<T>::get(slice[e / kVec], e % kVec);
      const uint32_t key = key_of(x);
      if (key > thr) one.mass = sc.kept_weight(x);
      one.count = key == thr;
    }
    Sum2 unused;
    const Sum2 b = block_scan(one, &unused);
    const u64 from = skip + b.mass + kept_ties(tie0, tie0 + b.count) * tie_weight;
    const u64 width = one.mass + kept_ties(tie0 + b.count, tie0 + b.count + one.count) * tie_weight;
    if (point >= from && point < from + width) out[r] = first + e - phase;
  }
  cluster.sync();   // no block leaves while its shared memory may still be read
}

template <typename T>
cudaError_t launch(const void* logits, int64_t row_stride, int n, int vocab, const float* temperature, const int32_t* top_k,
                   const float* top_p, const float* min_p, const float* uniform, int64_t* out, cudaStream_t s) {
  constexpr int kVec = Raw<T>::kVec;
  const int per = (vocab + kCluster * kVec - 1) / (kCluster * kVec);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n * kCluster); cfg.blockDim = dim3(kThreads); cfg.stream = s;
  cfg.dynamicSmemBytes = (size_t)(per + 1) * 16;     // one more piece: a slice that does not begin on a 16-byte boundary
  if (cudaError_t e = cudaFuncSetAttribute(k_sample<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes)) return e;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kCluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_sample<T>, (const T*)logits, row_stride, vocab, temperature, top_k, top_p, min_p, uniform,
                            reinterpret_cast<long long*>(out));
}

}  // namespace

extern "C" bc_status bc_sample(const void* logits, int32_t logits_f32, int64_t row_stride, int32_t n, int32_t vocab,
                               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                               const float* uniform, int64_t* out, void* stream) {
  if (!logits || !uniform || !out || n <= 0 || vocab <= 0 || row_stride < vocab) return BC_ERR_INVALID_ARG;
  const uintptr_t words = reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
                          reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(uniform);
  if ((words & 3) || (reinterpret_cast<uintptr_t>(out) & 7) || (reinterpret_cast<uintptr_t>(logits) & (logits_f32 ? 3 : 1)))
    return BC_ERR_INVALID_ARG;
  if (vocab > kMaxVocab || n > 0x7fffffff / kCluster) return BC_ERR_UNSUPPORTED;
  const cudaError_t e = logits_f32 ? launch<float>(logits, row_stride, n, vocab, temperature, top_k, top_p, min_p, uniform, out, (cudaStream_t)stream)
                                   : launch<__nv_bfloat16>(logits, row_stride, n, vocab, temperature, top_k, top_p, min_p, uniform, out,
                                                           (cudaStream_t)stream);
  return e == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}
