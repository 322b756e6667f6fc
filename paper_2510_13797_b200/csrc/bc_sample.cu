// Sampling of the next token from a row of logits, with temperature, top-k, top-p and min-p, from a given uniform
// random number per row (Algorithm 1 samples the next token from the model's distribution; bc_argmax is the greedy
// choice).  For a row x with maximum m and temperature T > 0:
//     e_j = exp((x_j - m) / T)
//     K   = the top_k largest x_j (of equal ones the lowest indices)                          [top_k on]
//     N   = the shortest prefix of K, largest first, whose mass reaches top_p * mass(K)       [top_p on]
//     S   = the elements of N with e_j >= min_p                                               [min_p on]
//     token = the first j of S in index order with sum_{i in S, i <= j} e_i > u * mass(S).
//
// Masses are sums of INTEGERS: e_j, evaluated in double precision (to 2^-48 of its value, see scaled()), is rounded to a
// multiple of 2^-45, so a row of up to 2^18 elements adds up exactly in 64 bits, in any order -- the split over threads and blocks
// and the order of the shared-memory atomics cannot change a result.  What the rounding drops is at most 2^-46 of the largest
// weight per element; an element that rounds to zero is never chosen.
//
// One cluster of eight thread blocks per row (a batch of 64 rows is too few blocks otherwise, and a single row still
// gets eight SMs).  Each block copies its slice of the row into shared memory, the only time the row is read from
// memory, and everything after works on the slices, joined through distributed shared memory:
//   1. maximum of the row (and its lowest index: the greedy answer);
//   2. with top-k or top-p: the threshold key.  For a top-k of up to 256: the k-th largest of the threads' maxima bounds it
//      from below, the elements from there on (a few more than k) are gathered, and each counts what lies above it.
//      Otherwise: a histogram of counts and masses over 512 bins of (m - x) / T, 1/11 octave wide (logits spread over many
//      of them, so the atomics rarely collide), then, inside the bin in which the limit is crossed, histograms over the keys'
//      own bits until the bin holds one key or its elements are few enough for the list.  Elements that equal the
//      threshold are kept lowest index first, as many as the limit needs;
//   3. the kept mass of every thread's run of elements, a prefix sum over threads and blocks, and the element in
//      which u * mass falls.
//
// Measured (T = 0.7; 64 rows of 151,936 bf16 = 19 MB, 3 us at the copy rate): greedy 10 us, temperature alone 24, top-k 50 22,
// top-k 50 and top-p 0.95 24, top-p 0.95 61 to 66 (by the rows); one row: 5, 10, 13, 14, 30 us.  Bounds: for one row the steps' latency
// (cluster barriers, that at the end included: three for temperature alone, seven with a small top-k, eight with top-p besides, nine and
// three per refining histogram with top-p alone; about 1 us each with what is read behind them); for many rows
// the double-precision weights of all elements (13 us of the 24) and, with top-p alone, three shared-memory atomics for
// each element of the first 22 octaves (about 25 us).  Tried for these: weights in single precision from 24
// octaves on (the branch costs more than the arithmetic: 87 us); a histogram of counts alone and masses of the few bins that they leave
// open (96 us, for the same reason).
#include <cooperative_groups.h>

#include "bc_common.cuh"

namespace cg = cooperative_groups;

namespace {

typedef unsigned long long u64;

constexpr int kCluster = 8;
constexpr int kBins = 512;
constexpr int kList = 512;             // elements that are ordered directly, by counting
constexpr int kFew = 256;              // a top-k up to here is looked for among the threads' maxima first
constexpr int kMaxVocab = 1 << 18;     // 2^18 weights of at most 2^45 add up in 63 bits
constexpr int kWeightBits = 45;

struct Sum2 {   // a mass and a count, added up together
  u64 mass;
  uint32_t count;
};
__device__ __forceinline__ Sum2 operator+(const Sum2& a, const Sum2& b) { return {a.mass + b.mass, a.count + b.count}; }

// Exclusive prefix over the block's threads; *total gets the block's sum.  All threads call.
template <int THREADS>
__device__ __forceinline__ Sum2 block_scan(Sum2 x, Sum2* total) {
  constexpr int kWarps = THREADS / 32;
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

// order-preserving key of a float that is not a NaN, and back
__device__ __forceinline__ uint32_t key32(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // the two zeros are one value
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key32(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

template <typename T> struct Raw;   // key, of_key: the same for the type's values, as small numbers (bf16: 16 bits)
template <> struct Raw<__nv_bfloat16> {
  static constexpr int kVec = 8;
  // element i of a 16-byte piece (a NaN compares below everything that is asked for)
  __device__ static __forceinline__ float get(const uint4& v, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&v)[i >> 1];
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  __device__ static __forceinline__ uint32_t key(float x) { return key32(x) >> 16; }   // of any float: rounded down
  __device__ static __forceinline__ float of_key(uint32_t k) { return of_key32(k << 16 | (k < 0x8000u ? 0xffffu : 0u)); }
  __device__ static __forceinline__ __nv_bfloat16 of(float x) { return __float2bfloat16_rn(x); }
  __device__ static __forceinline__ __nv_bfloat16 none() { return __ushort_as_bfloat16(0xff80); }
  typedef __nv_bfloat162 Max;               // running maximum; the maximum of a number and a NaN is the number
  __device__ static __forceinline__ Max start() { return __halves2bfloat162(none(), none()); }
  __device__ static __forceinline__ void fold(Max& m, const uint4& v) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
    m = __hmax2(m, __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
  }
  __device__ static __forceinline__ float value(const Max& m) { return fmaxf(__low2float(m), __high2float(m)) + 0.f; }
};
template <> struct Raw<float> {
  static constexpr int kVec = 4;
  __device__ static __forceinline__ float get(const uint4& v, int i) {
    return __uint_as_float(reinterpret_cast<const uint32_t*>(&v)[i]);
  }
  __device__ static __forceinline__ uint32_t key(float x) { return key32(x); }
  __device__ static __forceinline__ float of_key(uint32_t k) { return of_key32(k); }
  __device__ static __forceinline__ float of(float x) { return x; }
  __device__ static __forceinline__ float none() { return -INFINITY; }
  typedef float Max;
  __device__ static __forceinline__ Max start() { return -INFINITY; }
  __device__ static __forceinline__ void fold(Max& m, const uint4& v) {
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w))));
  }
  __device__ static __forceinline__ float value(Max m) { return m + 0.f; }
};

struct Scale {
  float top;      // the row's maximum, finite
  double dtop;
  double c;       // log2(e) / T
  float bins;     // 11 bins per octave
  float low;      // elements up to here have a weight of 0 (-inf at least)
  double min_w;   // 2^45 min_p
  // 2^45 e(x) for x > low, in double precision: 2^-t for t = (top - x) log2(e) / T octaves, t = n - f with |f| <= 1/2, and
  // 2^f = 1 + f g(f), where g is the polynomial through (2^f - 1) / f at the ten Chebyshev points of [-1/2, 1/2]: off by at most 2^-50 of
  // the value, and exactly 1 at f = 0.  The rounding of c adds up to 2^-53 ln(2) for each octave, 46 of them at most.  (Taylor's series with one
  // term less is off by 2^-37, 256 times the rounding of the largest weights, and a border between two elements moves with it.  The term
  // costs 1 to 3 %: 64 x 200,000 fp32, temperature alone, 58.9 and 59.4 us.)
  __device__ __forceinline__ double scaled(float x) const {
    constexpr double kMagic = 6755399441055744.0;              // 1.5 * 2^52: adding it rounds to an integer
    const double d = dtop - (double)x;
    const double m = fma(d, c, kMagic);
    const int n = __double2loint(m);
    const double f = fma(-d, c, m - kMagic);
    double p = 7.070977866508138e-09;
    p = fma(p, f, 1.0205905413765595e-07);
    p = fma(p, f, 1.3215451633221434e-06);
    p = fma(p, f, 1.5252672924850737e-05);
    p = fma(p, f, 1.5403530424776529e-04);
    p = fma(p, f, 1.3333558200794592e-03);
    p = fma(p, f, 9.618129107618665e-03);
    p = fma(p, f, 5.550410866465167e-02);
    p = fma(p, f, 2.4022650695910075e-01);
    p = fma(p, f, 6.931471805599462e-01);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + ((kWeightBits - n) << 20), __double2loint(p));
  }
  // a double of at most 2^46, rounded to an integer, as the low 52 bits of its sum with 2^52
  static constexpr u64 kBias = 0x4330000000000000ull;
  __device__ __forceinline__ static u64 biased(double v) { return (u64)__double_as_longlong(v + 4503599627370496.0); }
  // without branches, so that the evaluations of several elements overlap
  __device__ __forceinline__ u64 weight(float x) const {
    const u64 w = biased(scaled(x > low ? x : top)) - kBias;
    return x > low ? w : 0;
  }
  __device__ __forceinline__ u64 kept_weight(float x) const {   // 0 below min_p
    const double v = scaled(x > low ? x : top);
    return x > low && v >= min_w ? biased(v) - kBias : 0;
  }
  // in bins, of an element above low.  The difference is taken in halves: that of two finite numbers can be beyond the largest one.
  __device__ __forceinline__ float depth(float x) const { return fmaf(x, -0.5f, 0.5f * top) * (2.f * bins); }
  __device__ __forceinline__ int bin(float x) const { return min(kBins - 1, (int)depth(x)); }
  // of an element above low; the last bin has no lower end
  __device__ __forceinline__ bool in_bin(float x, int b) const {
    const float d = depth(x);
    return d >= (float)b && (d < (float)(b + 1) || b == kBins - 1);
  }
};

struct Cross {                   // where a search ended
  Sum2 before, all;
  int bin;
  uint32_t in;
};

struct Pick {                    // a key that a limit falls on, and what lies above it
  Sum2 above;
  uint32_t key;
  int found;
};

// A histogram, or a list of candidates: one search step has one or the other.  Small, because a slice of 150,000 bf16 logits
// leaves room for four blocks on an SM only while all of this stays below 18 KB.
union Work {
  // A mass is three sums of 32 bits, of the weights' bits 0 .. 15, 16 .. 31 and 32 .. 45 (at most 2^15 elements of a block):
  // shared memory adds 64 bits ten times slower.
  struct { uint32_t mass[3][kBins], count[kBins]; } h;
  struct {
    uint32_t list[kList];        // this block's candidates
    uint32_t keys[kList];        // all blocks' candidates, and their weights
    u64 weights[kList];
  } c;
  Sum2 total[kBins];             // block 0: a histogram of the whole cluster
};

struct Shared {
  Work work[2];                  // used in turn: one may still be read by other blocks
  int n_list[2];
  u64 rest, row_rest;            // mass of the elements that the histogram leaves out: this block's, the row's
  float best, row_best;          // this block's maximum, the row's
  int at;                        // its lowest index (greedy rows)
  Sum2 part;                     // this block's mass above the threshold and number of elements at it
  Sum2 parts[kCluster];          // every block's
  int offset[kCluster + 1];
  Cross cross;
  Pick pick[2];
  int owner;
  u64 owner_skip, owner_ties;
};

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_sample(const T* __restrict__ logits, int64_t row_stride, int vocab,
                                                                   const float* __restrict__ temperature, const int32_t* __restrict__ top_k,
                                                                   const float* __restrict__ top_p, const float* __restrict__ min_p,
                                                                   const float* __restrict__ uniform, long long* __restrict__ out) {
  constexpr int kVec = Raw<T>::kVec, kWarps = THREADS / 32, kPer = kBins / THREADS;   // kPer: bins a thread adds up
  extern __shared__ uint4 slice[];
  __shared__ Shared sh;
  __shared__ float warp_best[kWarps];
  cg::cluster_group cluster = cg::this_cluster();
  const int part = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = blockIdx.x / kCluster;
  const T* row = logits + r * row_stride;

  // ---- the slice: elements [first, first + cnt) of the row, kept at their 16-byte phase; its maximum --------------
  const int per = (vocab + kCluster * kVec - 1) / (kCluster * kVec) * kVec;
  const int first = min(part * per, vocab), cnt = min(vocab - first, per);
  const int phase = (int)((reinterpret_cast<uintptr_t>(row + first) & 15) / sizeof(T));
  const int pieces = cnt > 0 ? (phase + cnt + kVec - 1) / kVec : 0;
  typename Raw<T>::Max run_max = Raw<T>::start();
  const int whole0 = phase > 0 ? 1 : 0, whole1 = (phase + cnt) / kVec;          // pieces that lie in the slice entirely
  const uint4* aligned = reinterpret_cast<const uint4*>(row + first - phase);   // piece p at aligned + p
#pragma unroll 4
  for (int p = whole0 + tid; p < whole1; p += THREADS) {
    const uint4 v = __ldcs(aligned + p);
    slice[p] = v;
    Raw<T>::fold(run_max, v);
  }
  if (tid < 2 && pieces > 0) {                                                    // the ends: only what belongs to the row is read
    const int p = tid == 0 ? 0 : pieces - 1;
    if ((p < whole0 || p >= whole1) && !(tid == 1 && pieces == 1)) {
      T e[kVec];
      for (int i = 0; i < kVec; ++i) {
        const int at = p * kVec - phase + i;
        e[i] = at >= 0 && at < cnt ? row[first + at] : Raw<T>::none();
      }
      uint4 v;
      memcpy(&v, e, 16);
      slice[p] = v;
      Raw<T>::fold(run_max, v);
    }
  }
  float thread_best = Raw<T>::value(run_max);
  if (!(thread_best == thread_best)) thread_best = -INFINITY;
  float best = thread_best;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
  if (lane == 0) warp_best[warp] = best;
  for (int b = tid; b < kBins; b += THREADS) sh.work[0].h.mass[0][b] = sh.work[0].h.mass[1][b] = sh.work[0].h.mass[2][b] = sh.work[0].h.count[b] = sh.work[1].h.count[b] = 0;
  if (tid == 0) { sh.at = 0x7fffffff; sh.n_list[0] = 0; sh.pick[0] = sh.pick[1] = Pick{{0, 0}, 0, 0}; }
  __syncthreads();
  if (warp == 0) {
    best = lane < kWarps ? warp_best[lane] : -INFINITY;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
    if (lane == 0) sh.best = best;
  }
  cluster.sync();
  if (warp == 0) {                                 // one warp asks the other blocks, lane b block b
    best = *cluster.map_shared_rank(&sh.best, lane & (kCluster - 1));
#pragma unroll
    for (int d = kCluster / 2; d > 0; d >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
    if (lane == 0) sh.row_best = best;
  }
  __syncthreads();
  best = sh.row_best;

  const float temp = temperature != nullptr ? temperature[r] : 1.f;
  if (!(temp > 0.f) || best == -INFINITY) {        // greedy; a row of -inf and NaN: its first index
    int at = 0x7fffffff;
    for (int q = tid; q < pieces; q += THREADS) {
      const uint4 v = slice[q];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int e = q * kVec - phase + i;
        if (Raw<T>::get(v, i) == best && e >= 0 && e < cnt) at = min(at, first + e);
      }
    }
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) atomicMin(&sh.at, at);
    cluster.sync();
    if (part == 0 && tid == 0) {
      for (int b = 0; b < kCluster; ++b) at = min(at, *cluster.map_shared_rank(&sh.at, b));
      out[r] = best == -INFINITY ? 0 : at;         // NaN counts as -inf: every element is the maximum
    }
    cluster.sync();                                // no block leaves while its shared memory may still be read
    return;
  }
  if (best == INFINITY) {                          // infinite logits share the mass: 0 in a row of -inf
    for (int q = tid; q < pieces; q += THREADS) {
      T e[kVec];
      for (int i = 0; i < kVec; ++i) e[i] = Raw<T>::get(slice[q], i) == INFINITY ? Raw<T>::of(0.f) : Raw<T>::none();
      memcpy(&slice[q], e, 16);
    }
    best = 0.f;
    thread_best = thread_best == INFINITY ? 0.f : -INFINITY;
    __syncthreads();
  }
  Scale sc;
  sc.top = best;
  sc.dtop = (double)best;
  sc.c = fmax(1.4426950408889634 / (double)temp, 1e-300);   // not 0 for an infinite temperature: 0 * inf
  sc.bins = (float)fmin(11.0 * sc.c, 1e38);                 // finite, and twice as much as well: 0 * inf again
  sc.low = fminf((float)(sc.dtop - (kWeightBits + 1) / sc.c), nextafterf(best, -INFINITY));
  const float mp = min_p != nullptr ? min_p[r] : 0.f;
  sc.min_w = mp > 0.f ? fmin((double)mp, 1.0) * (double)(1ull << kWeightBits) : 0.0;   // at most 1: the largest element is always kept
  const int k = top_k != nullptr ? top_k[r] : 0;
  const float p = top_p != nullptr ? top_p[r] : 1.f;
  const bool by_count = k > 0 && k < vocab, by_mass = p < 1.f;

  // ---- threshold: keep every key above thr and the first `ties` elements (in index order) that equal it ------------
  uint32_t thr = 0;
  u64 ties = 0;                                     // with no limit: every key is above 0, the key no float has
  int round = 1;                                    // which of the two histograms and lists is next
  auto val = [](const Sum2& s, bool count) { return count ? (u64)s.count : s.mass; };
  auto add = [&](int which, int b, u64 w, bool count, bool mass) {
    if (count) atomicAdd(&sh.work[which].h.count[b], 1u);
    if (!mass) return;
    atomicAdd(&sh.work[which].h.mass[0][b], (uint32_t)w & 0xffffu);
    atomicAdd(&sh.work[which].h.mass[1][b], (uint32_t)(w >> 16) & 0xffffu);
    if (w >> 32) atomicAdd(&sh.work[which].h.mass[2][b], (uint32_t)(w >> 32));
  };
  // The cluster's histograms added up, for block 0, which searches them for all (all blocks together would read eight times as much
  // of one another's memory): thread t gets its bins kPer t ...  Counts alone it reads itself.  With masses (`masses`) each
  // block adds up an eighth of the bins, kLanes threads a bin, and hands the sums over: a barrier more, but block 0 alone
  // takes 3 to 6 us for what the others hold.
  auto totals = [&](int which, bool masses, Sum2 (&b)[kPer]) {
    if (!masses) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        b[i] = {0, 0};
        if (part == 0)
#pragma unroll
          for (int o = 0; o < kCluster; ++o) b[i].count += *cluster.map_shared_rank(&sh.work[which].h.count[kPer * tid + i], o);
      }
      return;
    }
    constexpr int kShare = kBins / kCluster, kLanes = THREADS / kShare, kEach = kCluster / kLanes;
    const int bin = part * kShare + tid / kLanes;
    Sum2 sum = {0, 0};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int o = tid % kLanes * kEach + i;
      sum.count += *cluster.map_shared_rank(&sh.work[which].h.count[bin], o);
#pragma unroll
      for (int j = 0; j < 3; ++j) sum.mass += (u64)*cluster.map_shared_rank(&sh.work[which].h.mass[j][bin], o) << (16 * j);
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
      sum.mass += __shfl_xor_sync(0xffffffffu, sum.mass, d);
      sum.count += __shfl_xor_sync(0xffffffffu, sum.count, d);
    }
    // into the other of the two, which nobody reads any more: its readers have passed a cluster barrier since
    if (tid % kLanes == 0) *cluster.map_shared_rank(&sh.work[which ^ 1].total[bin], 0) = sum;
    cluster.sync();
#pragma unroll
    for (int i = 0; i < kPer; ++i) b[i] = part == 0 ? sh.work[which ^ 1].total[kPer * tid + i] : Sum2{0, 0};
  };
  auto mass_limit = [&](u64 mass) {                  // the largest element is always kept; NaN never comes here
    const double want = ceil((double)p * (double)mass);
    return want >= 1.0 ? (u64)want : (u64)1;
  };
  // The bin in which the running count (or mass), largest keys first, reaches `limit`: false if it never does.  *all: the sum of
  // the bins.  Block 0 searches its totals, the others take over what it finds.  limit 0: the top-p limit of
  // the sum.
  auto cross = [&](const Sum2 (&b)[kPer], const Sum2& before0, bool count, u64 limit, Sum2* all) {
    if (part == 0) {
      if (tid == 0) sh.cross.bin = -1;
      Sum2 mine = b[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) mine = mine + b[i];
      Sum2 sum;
      Sum2 e = block_scan<THREADS>(mine, &sum) + before0;   // its barriers order the store above
      if (limit == 0) { sum.mass += sh.row_rest; limit = mass_limit(sum.mass); }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const Sum2 n = e + b[i];
        if (val(e, count) < limit && limit <= val(n, count)) { sh.cross.bin = kPer * tid + i; sh.cross.before = e; sh.cross.in = b[i].count; }
        e = n;
      }
      if (tid == 0) sh.cross.all = sum;
    }
    cluster.sync();
    if (warp == 0 && part != 0) {
      const uint32_t* from = reinterpret_cast<const uint32_t*>(cluster.map_shared_rank(&sh.cross, 0));
      if (lane < (int)(sizeof(Cross) / 4)) reinterpret_cast<uint32_t*>(&sh.cross)[lane] = from[lane];
    }
    __syncthreads();
    *all = sh.cross.all;
    return sh.cross.bin >= 0;
  };
  // The lengths of all blocks' lists, as offsets; their sum.
  auto offsets = [&](int which) {
    if (warp == 0) {
      int x = lane < kCluster ? *cluster.map_shared_rank(&sh.n_list[which], lane) : 0;
#pragma unroll
      for (int d = 1; d < kCluster; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      if (lane < kCluster) sh.offset[lane + 1] = x;
      if (lane == 0) sh.offset[0] = 0;
    }
    __syncthreads();
    return sh.offset[kCluster];
  };
  // All blocks' candidate lists, one behind the other, with their weights, in this block's memory.
  auto gather = [&](int which) {
    for (int at = tid; at < min(kList, sh.offset[kCluster]); at += THREADS) {
      int o = 0;
#pragma unroll
      for (int b = 1; b < kCluster; ++b) o += at >= sh.offset[b];
      const uint32_t key = *cluster.map_shared_rank(&sh.work[which].c.list[at - sh.offset[o]], o);
      sh.work[which].c.keys[at] = key;
      sh.work[which].c.weights[at] = sc.weight(Raw<T>::of_key(key));
    }
    __syncthreads();
  };
  // Among `len` gathered candidates, with `before` above them: the key at which the running count (or mass) reaches `limit`, and
  // what lies above that key (false if the limit is not reached).  Every candidate counts what is above itself; the blocks share
  // the candidates, kLanes threads each, and the one that finds the key tells the others.
  int picks = 0;                                     // two at most: by count, then by mass
  auto select = [&](int which, int len, bool count, u64 limit, Sum2* before, uint32_t* key_out) {
    constexpr int kLanes = THREADS / (kList / kCluster);
    const uint32_t* keys = sh.work[which].c.keys;
    const u64* weights = sh.work[which].c.weights;
    const int at = tid / kLanes * kCluster + part;
    const uint32_t key = at < len ? keys[at] : 0xffffffffu;
    Sum2 above = {0, 0};
    uint32_t same = 0;
    if (at < len) {
#pragma unroll 4
      for (int j = tid % kLanes; j < len; j += kLanes) {
        const uint32_t o = keys[j];
        if (o > key) { above.mass += weights[j]; ++above.count; }
        same += o == key;
      }
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) {
      above.mass += __shfl_xor_sync(0xffffffffu, above.mass, d);
      above.count += __shfl_xor_sync(0xffffffffu, above.count, d);
      same += __shfl_xor_sync(0xffffffffu, same, d);
    }
    above = above + *before;
    if (at < len && tid % kLanes == 0 && val(above, count) < limit && limit <= val(above + Sum2{same * weights[at], same}, count)) {
#pragma unroll
      for (int b = 0; b < kCluster; ++b) {           // equal keys write equal values
        Pick* to = cluster.map_shared_rank(&sh.pick[picks], b);
        to->found = 1; to->key = key; to->above = above;
      }
    }
    cluster.sync();
    const Pick& got = sh.pick[picks++];
    *before = got.above;
    *key_out = got.key;
    return got.found != 0;
  };
  // A small top-k: the elements no deeper than the k-th largest of the threads' maxima are few (unless the large ones are
  // neighbours) and hold the limit.  One atomic per thread instead of several per element, and no weights but theirs.
  bool open = by_count || by_mass;                    // the threshold is still to be found
  if (by_count && k <= kFew) {
    if (thread_best > sc.low) atomicAdd(&sh.work[1].h.count[sc.bin(thread_best)], 1u);
    cluster.sync();
    Sum2 bins[kPer], all;
    totals(1, false, bins);
    const int last = cross(bins, Sum2{0, 0}, true, (u64)k, &all) ? sh.cross.bin : kBins - 1;
    const float reach = last == kBins - 1 ? INFINITY : (float)(last + 1);
    for (int q = tid; q < pieces; q += THREADS) {
      const uint4 v = slice[q];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float x = Raw<T>::get(v, i);
        if (x > sc.low && sc.depth(x) < reach) {
          const int at = atomicAdd(&sh.n_list[0], 1);
          if (at < kList) sh.work[0].c.list[at] = Raw<T>::key(x);
        }
      }
    }
    cluster.sync();
    const int len = offsets(0);
    if (len <= kList) {
      gather(0);
      Sum2 before = {0, 0};
      uint32_t key = 0;
      u64 mass;
      open = false;
      if (select(0, len, true, (u64)k, &before, &key)) {
        thr = key;
        ties = (u64)k - before.count;
        mass = before.mass + ties * sc.weight(Raw<T>::of_key(thr));
      } else {                                        // fewer than k elements have a weight, and all of them are here
        block_scan<THREADS>(Sum2{(tid < len ? sh.work[0].c.weights[tid] : 0) + (THREADS < kList && tid + THREADS < len ? sh.work[0].c.weights[tid + THREADS] : 0), 0}, &all);
        mass = all.mass;
      }
      if (by_mass) {
        const u64 limit = mass_limit(mass);
        before = {0, 0};
        if (select(0, len, false, limit, &before, &key)) {
          thr = key;
          const u64 w = sc.weight(Raw<T>::of_key(thr));
          ties = (limit - before.mass + w - 1) / w;
        }
      }
    }
  }
  if (open) {
    if (by_count && k <= kFew) {                      // the list of the first try lies where the histogram goes
      for (int b = tid; b < kBins; b += THREADS) sh.work[0].h.mass[0][b] = sh.work[0].h.mass[1][b] = sh.work[0].h.mass[2][b] = sh.work[0].h.count[b] = 0;
      __syncthreads();
    }
    // The general search.  Counts and masses of the elements by bins of depth.  Without a top-k the elements of
    // log2(vocab / (1 - top_p)) octaves and more are left out: all of them together are less than (1 - top_p) of the largest
    // weight, so the limit is reached before them; they are most of a row at low temperatures.
    const bool masses = by_mass;
    const float deep = by_count ? INFINITY : 11.f * (log2f((float)vocab / (1.f - fmaxf(p, 0.f))) + 1.f);
    u64 rest = 0;
    for (int q = tid; q < pieces; q += THREADS) {
      const uint4 v = slice[q];
#pragma unroll
      for (int i0 = 0; i0 < kVec; i0 += 4) {            // the weights of four at a time before their branches
        u64 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sc.weight(Raw<T>::get(v, i0 + i));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = Raw<T>::get(v, i0 + i);
          const bool out = sc.depth(x) >= deep;
          rest += out ? w[i] : 0;
          if (w[i] && !out) add(0, sc.bin(x), w[i], by_count, masses);
        }
      }
    }
    Sum2 bins[kPer], all;
    {
      Sum2 sum;
      block_scan<THREADS>(Sum2{rest, 0}, &sum);
      if (tid == 0) sh.rest = sum.mass;
    }
    cluster.sync();
    totals(0, masses, bins);
    if (part == 0 && warp == 0) {
      u64 m = lane < kCluster ? *cluster.map_shared_rank(&sh.rest, lane) : 0;
#pragma unroll
      for (int d = kCluster / 2; d > 0; d >>= 1) m += __shfl_xor_sync(0xffffffffu, m, d);
      if (lane == 0) sh.row_rest = m;
    }
    // From the bin that cross() found to the key: a histogram over the keys of the bin (over their upper bits while they are too
    // many for one: the next step then takes the keys of one of its entries), or, once the elements are few, all of them ordered.
    // Returns the key, *before: what lies above it.
    auto refine = [&](bool count, u64 limit, Sum2* before) {
      const int bin = sh.cross.bin;
      *before = sh.cross.before;
      uint32_t in = count ? sh.cross.in : 0xffffffffu;
      // keys the bin can hold: its ends, rounded outwards
      const float x1 = (float)bin / sc.bins, x0 = (float)(bin + 1) / sc.bins, slack = (fabsf(sc.top) + x0) * 4e-7f;
      const float high = sc.top - x1 + slack, low = bin == kBins - 1 ? sc.low : sc.top - x0 - slack;
      uint32_t lo = 0, hi = Raw<T>::key(sc.top);
      if (high >= low) { lo = Raw<T>::key(fmaxf(low, sc.low)); hi = min(hi, Raw<T>::key(high)); }
      for (int left = 4; in > kList && lo != hi && left > 0; ++round, --left) {   // 9 bits of the keys' 32 at a time
        const int which = round & 1;
        for (int b = tid; b < kBins; b += THREADS) sh.work[which].h.mass[0][b] = sh.work[which].h.mass[1][b] = sh.work[which].h.mass[2][b] = sh.work[which].h.count[b] = 0;
        __syncthreads();
        const int shift = max(0, 32 - __clz(hi - lo) - 9);   // (hi - lo) >> shift is below 512
        for (int q = tid; q < pieces; q += THREADS) {
          const uint4 v = slice[q];
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const float x = Raw<T>::get(v, i);
            if (x > sc.low && sc.in_bin(x, bin)) {
              const uint32_t key = Raw<T>::key(x);
              const u64 w = key >= lo && key <= hi ? sc.weight(x) : 0;
              if (w) add(which, (int)((hi - key) >> shift), w, true, true);
            }
          }
        }
        cluster.sync();
        Sum2 sub[kPer], unused;
        totals(which, true, sub);
        cross(sub, *before, count, limit, &unused);
        *before = sh.cross.before;
        in = sh.cross.in;
        hi -= (uint32_t)sh.cross.bin << shift;
        lo = max(lo, hi - ((1u << shift) - 1u));
        __syncthreads();                             // sh.cross has been read
      }
      if (lo == hi) return lo;
      const int which = round & 1;
      ++round;
      if (tid == 0) sh.n_list[which] = 0;
      __syncthreads();
      for (int q = tid; q < pieces; q += THREADS) {
        const uint4 v = slice[q];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float x = Raw<T>::get(v, i);
          if (x > sc.low && sc.in_bin(x, bin)) {
            const uint32_t key = Raw<T>::key(x);
            if (key >= lo && key <= hi && sc.weight(x)) {
              const int at = atomicAdd(&sh.n_list[which], 1);
              if (at < kList) sh.work[which].c.list[at] = key;   // always so: they are `in`
            }
          }
        }
      }
      cluster.sync();
      offsets(which);
      gather(which);
      uint32_t key = 0;
      select(which, min(kList, sh.offset[kCluster]), count, limit, before, &key);
      return key;
    };
    bool cut = false;
    Sum2 before;
    u64 mass = 0;
    if (by_count) {
      cut = cross(bins, Sum2{0, 0}, true, (u64)k, &all);
      if (cut) {
        thr = refine(true, (u64)k, &before);
        ties = (u64)k - before.count;
        mass = before.mass + ties * sc.weight(Raw<T>::of_key(thr));
      }
    }
    if (by_mass) {
      cluster.sync();                                // the other blocks have taken over what the search before found
      const bool found = cross(bins, Sum2{0, 0}, false, cut ? mass_limit(mass) : 0, &all);
      const u64 limit = mass_limit(cut ? mass : all.mass);
      if (found) {
        thr = refine(false, limit, &before);
        const u64 w = sc.weight(Raw<T>::of_key(thr));
        ties = (limit - before.mass + w - 1) / w;
      }
    }
  }

  // ---- the draw ---------------------------------------------------------------------------------------------------
  // Thread t takes a run of consecutive pieces, so that threads are in index order; an odd run keeps the 16-byte
  // reads of neighbouring threads off one another's banks.
  const int run = ((per / kVec + 1 + THREADS - 1) / THREADS) | 1;
  const u64 tie_weight = thr != 0 ? sc.kept_weight(Raw<T>::of_key(thr)) : 0;
  const float floor_x = thr != 0 ? Raw<T>::of_key(thr) : sc.low;         // nothing below it is kept
  Sum2 mine = {0, 0};                                // mass above the threshold, elements at it
  const T* flat = reinterpret_cast<const T*>(slice);
  const int run_end = min(pieces, (tid + 1) * run);
  if (thr == 0) {                                    // nearly all are kept
#pragma unroll 1
    for (int q = tid * run; q < run_end; ++q) {
      const uint4 v = slice[q];
#pragma unroll
      for (int i = 0; i < kVec; ++i) mine.mass += sc.kept_weight(Raw<T>::get(v, i));
    }
  }
  for (int q = tid * run; thr != 0 && q < run_end; q += 32 / kVec) {
    // 32 elements at a time: first which of them are kept, then their weights, so that a warp whose lanes keep few
    // elements evaluates few
    uint32_t above = 0;
#pragma unroll
    for (int o = 0; o < 32 / kVec; ++o) {
      if (q + o < run_end) {
        const uint4 v = slice[q + o];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float x = Raw<T>::get(v, i);
          above |= (x > floor_x ? 1u : 0u) << (o * kVec + i);
          mine.count += x == floor_x;
        }
      }
    }
    for (; above; above &= above - 1) mine.mass += sc.kept_weight((float)flat[q * kVec + __ffs(above) - 1]);
  }
  Sum2 block_all;
  const Sum2 mine_before = block_scan<THREADS>(mine, &block_all);
  if (tid == 0) sh.part = block_all;
  cluster.sync();
  if (tid < kCluster) {
    const Sum2* o = cluster.map_shared_rank(&sh.part, tid);
    sh.parts[tid] = *o;
  }
  __syncthreads();
  u64 all_mass = 0, my_skip = 0, my_mass = 0, my_tied = 0, tied = 0;
#pragma unroll
  for (int b = 0; b < kCluster; ++b) {
    const u64 here = sh.parts[b].count, kept = tied >= ties ? 0 : (here < ties - tied ? here : ties - tied);
    const u64 m = sh.parts[b].mass + kept * tie_weight;
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
    const u64 skip = my_skip + mine_before.mass + kept_ties(my_tied, t0) * tie_weight;
    const u64 own = mine.mass + kept_ties(t0, t1) * tie_weight;
    if (point >= skip && point < skip + own) { sh.owner = tid; sh.owner_skip = skip; sh.owner_ties = t0; }
    __syncthreads();
    const int owner = sh.owner;
    // the owner's run, one element per thread (with 256 threads a run has at most 17 pieces of 8 or 33 of 4 elements)
    const int e = owner * run * kVec + tid, end = min(pieces, (owner + 1) * run) * kVec;
    Sum2 one = {0, 0};
    if (e < end) {
      const float x = Raw<T>::get(slice[e / kVec], e % kVec);
      if (x > floor_x) one.mass = sc.kept_weight(x);
      one.count = thr != 0 && x == floor_x;
    }
    Sum2 unused;
    const Sum2 b = block_scan<THREADS>(one, &unused);
    const u64 tie0 = sh.owner_ties;
    const u64 from = sh.owner_skip + b.mass + kept_ties(tie0, tie0 + b.count) * tie_weight;
    const u64 width = one.mass + kept_ties(tie0 + b.count, tie0 + b.count + one.count) * tie_weight;
    if (point >= from && point < from + width) out[r] = first + e - phase;
  }
  cluster.sync();   // no block leaves while its shared memory may still be read
}

template <typename T, int THREADS>
cudaError_t launch(const void* logits, int64_t row_stride, int n, int vocab, const float* temperature, const int32_t* top_k,
                   const float* top_p, const float* min_p, const float* uniform, int64_t* out, cudaStream_t s) {
  constexpr int kVec = Raw<T>::kVec;
  const int per = (vocab + kCluster * kVec - 1) / (kCluster * kVec);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n * kCluster); cfg.blockDim = dim3(THREADS); cfg.stream = s;
  cfg.dynamicSmemBytes = (size_t)(per + 1) * 16;     // one more piece: a slice that does not begin on a 16-byte boundary
  // The limit belongs to the kernel, not to the call: always that of the largest vocabulary, so that calls of several host threads
  // cannot lower it for one another between setting it and launching.
  constexpr int kMaxSlice = (kMaxVocab / (kCluster * kVec) + 1) * 16;
  if (cudaError_t e = cudaFuncSetAttribute(k_sample<T, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice)) return e;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kCluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_sample<T, THREADS>, (const T*)logits, row_stride, vocab, temperature, top_k, top_p, min_p, uniform,
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
  // 512 threads where a block has an SM to itself: few rows (8 of 151,936 bf16, top-p: 30 us, with 256 threads 36; 32 rows: 43
  // and 42), or slices of more than 95 KB (64 rows of 200,000 fp32, top-p: 172 and 211 us; of 151,936: 90 and 89, temperature
  // alone 39 and 31).
  const bool wide = n * kCluster <= 148 || (int64_t)vocab * (logits_f32 ? 4 : 2) > (int64_t)kCluster * 95 * 1024;
  const auto f = wide ? (logits_f32 ? launch<float, 512> : launch<__nv_bfloat16, 512>)
                                         : (logits_f32 ? launch<float, 256> : launch<__nv_bfloat16, 256>);
  const cudaError_t e = f(logits, row_stride, n, vocab, temperature, top_k, top_p, min_p, uniform, out, (cudaStream_t)stream);
  return e == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}
