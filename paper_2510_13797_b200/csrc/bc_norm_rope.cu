// Norms of the query and key heads with the rotation in the same pass, and the gradient of both.
//
// Models that normalise every query and key head before the rotation put, between the QKV projection and the
// attention, for each head x of D coordinates (bf16 in, fp32 arithmetic, ONE rounding to bf16 at the end):
//     y = x / sqrt(mean(x^2) + eps) * w                (w: D weights shared by all query heads, D by all key heads)
//     out = R(pos) y                                   (half-split rotation by pos * theta^(-2j/D), as bc_rope_split)
// and the gradient, with g = d loss / d out, r = 1 / sqrt(mean(x^2) + eps):
//     dy = R(pos)^T g,   dx = r (w dy - x r^2 mean(x w dy)),   dw = sum over rows and heads of x r dy.
// Everything is bound by memory: the packed rows are read once and q, k, v written once (the gradient reads x and
// g of the rotated heads and writes dx; v's gradient is a copy).
//
// A head is held by D / 16 lanes, each with 8 coordinates of the lower half and the 8 that they are paired with, so
// the rotation needs no exchange and the norm D / 16 lanes' shuffles; a warp works on 32 / (D / 16) heads at a time.
// A warp takes a whole row (or, while there are few rows, a share of its heads) and computes the row's D / 2 angles
// itself, D / 64 per lane: the position times the frequency in turns, reduced to a fraction of a turn in double
// precision (pos * theta^(-2j/D) reaches 10^5 radians, where single precision has lost the angle), then the sine and
// cosine of that fraction in fp32.
//
// Measured (32 / 8 heads of 128, bf16): 16384 rows 66 to 67 us in replays, 6.0 TB/s of the 403 MB moved (0.92 of a
// copy), 69 us as a call; the gradient with the weights' of 8192 rows 61 us, 4.6 TB/s, 63.5 us as a call (its sums over rows and the
// second launch, which adds the blocks' sums up, are what a copy does not have); 64 rows of 12 / 2 heads 2.5 us, a launch.
#include "bc_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Pairs of fp32 numbers in one register pair: one instruction for both (Blackwell's packed fp32 arithmetic).
typedef unsigned long long F2;
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
__device__ __forceinline__ void unpack8(const uint4& v, F2* f) {
  f[0] = pair(bf_lo(v.x), bf_hi(v.x)); f[1] = pair(bf_lo(v.y), bf_hi(v.y));
  f[2] = pair(bf_lo(v.z), bf_hi(v.z)); f[3] = pair(bf_lo(v.w), bf_hi(v.w));
}
__device__ __forceinline__ uint32_t pack_bf16(F2 v) {
  float a, b;
  split(v, &a, &b);
  return pack_bf16(a, b);
}
__device__ __forceinline__ uint4 pack8(const F2* f) { return make_uint4(pack_bf16(f[0]), pack_bf16(f[1]), pack_bf16(f[2]), pack_bf16(f[3])); }
__device__ __forceinline__ float sum_of(F2 v) {
  float a, b;
  split(v, &a, &b);
  return a + b;
}

// sum over the D / 16 lanes that hold a head
template <int D>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int d = D / 32; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

// Frequencies (in turns per position) of the angles this lane computes: D / 64 consecutive ones.
template <int D>
__device__ __forceinline__ void lane_frequencies(double log2_theta, double* f) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int j = (int)(threadIdx.x & 31) * (D / 64) + i;
    f[i] = exp2(-2.0 * (double)j / (double)D * log2_theta) * 0.15915494309189535;   // 1 / (2 pi)
  }
}
// cos and sin of the eight angles that belong to this lane's coordinates, for the position of the warp's row
template <int D>
__device__ __forceinline__ void row_angles(int pos, const double* f, F2* c2, F2* s2) {
  float c[8], s[8];
  float cs[D / 64], sn[D / 64];
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const double turns = (double)pos * f[i];
    sincospif(2.f * (float)(turns - rint(turns)), &sn[i], &cs[i]);
  }
  const int piece = (int)(threadIdx.x & 31) & (D / 16 - 1);
#pragma unroll
  for (int i = 0; i < 8; ++i) {   // angle piece * 8 + i was computed by lane (piece * 8 + i) / (D / 64)
    const int src = (piece * 8 + i) / (D / 64);
    c[i] = __shfl_sync(0xffffffffu, cs[i % (D / 64)], src);
    s[i] = __shfl_sync(0xffffffffu, sn[i % (D / 64)], src);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { c2[i] = pair(c[2 * i], c[2 * i + 1]); s2[i] = pair(s[2 * i], s[2 * i + 1]); }
}

struct NormRopeArgs {
  const uint8_t* qkv;
  int64_t row_bytes;
  const int32_t* positions;
  const uint4 *q_weight, *k_weight;   // NULL: ones
  uint4 *q_out, *k_out, *v_out;
  int64_t units;                      // rows * split
  int q_heads, kv_heads, split;       // split: warps that share a row's heads
  double log2_theta;
  float eps;
};

// The heads a warp has of a row are worked on in passes of kHeads; kAhead passes' loads are in flight at once (two blocks per SM
// of 4 KB per warp: 64 KB, a little more than the memory's latency times its rate takes), the row's angles are computed behind the
// first of them.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope(const NormRopeArgs a) {
  constexpr int kLanes = D / 16, kHeads = 32 / kLanes, kChunks = D / 8;   // lanes per head, heads per pass, 16-byte pieces per head
  constexpr int kAhead = 4;
  const int lane = threadIdx.x & 31, piece = lane & (kLanes - 1), sub = lane / kLanes;
  const uint4 ones = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  const uint4 wq0 = a.q_weight ? a.q_weight[piece] : ones, wq1 = a.q_weight ? a.q_weight[kLanes + piece] : ones;
  const uint4 wk0 = a.k_weight ? a.k_weight[piece] : ones, wk1 = a.k_weight ? a.k_weight[kLanes + piece] : ones;
  double freq[D / 64];
  lane_frequencies<D>(a.log2_theta, freq);
  const int rot = a.q_heads + a.kv_heads, heads = rot + a.kv_heads;
  const int64_t step = (int64_t)gridDim.x * kWarps;
  for (int64_t u = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); u < a.units; u += step) {
    const int64_t row = u / a.split;
    const int part = (int)(u - row * a.split);
    const int pos = a.positions[row];
    const uint4* in = reinterpret_cast<const uint4*>(a.qkv + row * a.row_bytes);
    F2 c[4], s[4];
    for (int h0 = part * kHeads; h0 < heads; h0 += kAhead * a.split * kHeads) {
      uint4 lo[kAhead], hi[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = h0 + k * a.split * kHeads + sub;
        lo[k] = hi[k] = make_uint4(0, 0, 0, 0);
        if (h < heads) { lo[k] = __ldcs(in + h * kChunks + piece); hi[k] = __ldcs(in + h * kChunks + kLanes + piece); }
      }
      if (h0 == part * kHeads) row_angles<D>(pos, freq, c, s);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = h0 + k * a.split * kHeads + sub;
        if (h0 + k * a.split * kHeads >= heads) break;             // uniform over the warp
        F2 x[4], y[4], sq = pair(0.f, 0.f);
        unpack8(lo[k], x); unpack8(hi[k], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) sq = fma2(x[i], x[i], fma2(y[i], y[i], sq));
        const float r = rsqrtf(head_sum<D>(sum_of(sq)) * (1.f / D) + a.eps);
        if (h < rot) {
          const bool is_q = h < a.q_heads;
          F2 w0[4], w1[4];
          unpack8(is_q ? wq0 : wk0, w0); unpack8(is_q ? wq1 : wk1, w1);
          const F2 r2 = pair(r, r), minus = pair(-1.f, -1.f);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const F2 p = mul2(mul2(x[i], r2), w0[i]), q = mul2(mul2(y[i], r2), w1[i]);
            x[i] = fma2(p, c[i], mul2(mul2(q, minus), s[i]));
            y[i] = fma2(q, c[i], mul2(p, s[i]));
          }
          uint4* dst = is_q ? a.q_out + (row * a.q_heads + h) * kChunks : a.k_out + (row * a.kv_heads + (h - a.q_heads)) * kChunks;
          dst[piece] = pack8(x);
          dst[kLanes + piece] = pack8(y);
        } else if (h < heads) {
          uint4* dst = a.v_out + (row * a.kv_heads + (h - rot)) * kChunks;
          dst[piece] = lo[k];
          dst[kLanes + piece] = hi[k];
        }
      }
    }
  }
}

struct NormRopeGradArgs {
  const uint8_t* qkv;
  int64_t row_bytes;
  const int32_t* positions;
  const __nv_bfloat16 *q_weight, *k_weight;
  const uint4 *dq, *dk, *dv;
  uint4* dqkv;          // [rows][q_heads + 2 kv_heads][D], contiguous
  float* partial;       // [blocks][2][D]
  int64_t units;
  int q_heads, kv_heads, split, fold;
  double log2_theta;
  float eps;
};

// The weight gradients: every lane adds up its 16 coordinates over the rows and heads it meets (fp32; the query heads' sums in
// registers, the key heads', which are fewer, in a place of the lane's own in shared memory).  After `fold` units, kFoldTerms terms or one
// unit's, the warp's lanes are joined into the warp's sums in shared memory and begin again, so that no chain of additions grows
// with the number of rows but that of the folds, a hundredth as long.  At the end the block's warps are joined and a second kernel adds
// the blocks', all in a fixed order, so that results are reproducible.
constexpr int kFoldTerms = 128;
template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope_grad(const NormRopeGradArgs a) {
  constexpr int kLanes = D / 16, kHeads = 32 / kLanes, kChunks = D / 8;
  constexpr int kAhead = 2;
  if (a.partial != nullptr) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the kernel that adds the blocks' sums waits for this one's end
  __shared__ __align__(16) float weights[2][D];
  __shared__ __align__(16) float dwk[kWarps][4][32][4];           // a lane's 16 sums: 16 bytes apart from its neighbours'
  __shared__ __align__(16) float sums[kWarps][2][D];
  const int lane = threadIdx.x & 31, piece = lane & (kLanes - 1), sub = lane / kLanes, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const __nv_bfloat16* w = i < D ? a.q_weight : a.k_weight;
    weights[i / D][i % D] = w ? __bfloat162float(w[i % D]) : 1.f;
  }
  for (int i = threadIdx.x; i < kWarps * 2 * D / 4; i += kThreads) reinterpret_cast<float4*>(sums)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(dwk[warp][i][lane]) = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  double freq[D / 64];
  lane_frequencies<D>(a.log2_theta, freq);
  const int rot = a.q_heads + a.kv_heads, heads = rot + a.kv_heads;
  F2 dwq[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dwq[i] = pair(0.f, 0.f);
  const int64_t step = (int64_t)gridDim.x * kWarps;
  int left = a.fold;
  for (int64_t u = (int64_t)blockIdx.x * kWarps + warp; u < a.units; u += step) {
    const int64_t row = u / a.split;
    const int part = (int)(u - row * a.split);
    const int pos = a.positions[row];
    const uint4* in = reinterpret_cast<const uint4*>(a.qkv + row * a.row_bytes);
    const uint4* gq = a.dq + row * a.q_heads * kChunks;               // + h: the gradient of head h of the row, of its kind
    const uint4* gk = a.dk + (row * a.kv_heads - a.q_heads) * kChunks;
    const uint4* gv = a.dv + (row * a.kv_heads - rot) * kChunks;
    uint4* out = a.dqkv + row * heads * kChunks;
    F2 c[4], s[4];
    for (int h0 = part * kHeads; h0 < heads; h0 += kAhead * a.split * kHeads) {
      uint4 xlo[kAhead], xhi[kAhead], glo[kAhead], ghi[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = h0 + k * a.split * kHeads + sub;
        xlo[k] = xhi[k] = glo[k] = ghi[k] = make_uint4(0, 0, 0, 0);
        if (h < rot) { xlo[k] = __ldcs(in + h * kChunks + piece); xhi[k] = __ldcs(in + h * kChunks + kLanes + piece); }
        if (h < heads) {
          const uint4* g = (h < a.q_heads ? gq : (h < rot ? gk : gv)) + h * kChunks;
          glo[k] = __ldcs(g + piece); ghi[k] = __ldcs(g + kLanes + piece);
        }
      }
      if (h0 == part * kHeads) row_angles<D>(pos, freq, c, s);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int h = h0 + k * a.split * kHeads + sub;
        if (h0 + k * a.split * kHeads >= heads) break;             // uniform over the warp
        const bool is_q = h < a.q_heads;
        F2 w0[4], w1[4];
        {
          const float4* w = reinterpret_cast<const float4*>(weights[is_q ? 0 : 1] + piece * 8);
          const float4 v0 = w[0], v1 = w[1], v2 = w[D / 8], v3 = w[D / 8 + 1];
          w0[0] = pair(v0.x, v0.y); w0[1] = pair(v0.z, v0.w); w0[2] = pair(v1.x, v1.y); w0[3] = pair(v1.z, v1.w);
          w1[0] = pair(v2.x, v2.y); w1[1] = pair(v2.z, v2.w); w1[2] = pair(v3.x, v3.y); w1[3] = pair(v3.z, v3.w);
        }
        F2 x[4], y[4], p[4], q[4], sq2 = pair(0.f, 0.f), dot2 = sq2;
        const F2 minus = pair(-1.f, -1.f);
        unpack8(xlo[k], x); unpack8(xhi[k], y); unpack8(glo[k], p); unpack8(ghi[k], q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const F2 d0 = fma2(p[i], c[i], mul2(q[i], s[i])), d1 = fma2(q[i], c[i], mul2(mul2(p[i], minus), s[i]));   // the rotation taken back
          p[i] = d0; q[i] = d1;
          sq2 = fma2(x[i], x[i], fma2(y[i], y[i], sq2));
          dot2 = fma2(mul2(x[i], w0[i]), d0, fma2(mul2(y[i], w1[i]), d1, dot2));
        }
        const float sq = head_sum<D>(sum_of(sq2)), dot = head_sum<D>(sum_of(dot2));
        const float r = rsqrtf(sq * (1.f / D) + a.eps), t = r * r * dot * (1.f / D);
        const F2 r2 = pair(r, r), t2 = pair(-t, -t);
        if (h < rot) {
          if (is_q) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { dwq[i] = fma2(mul2(x[i], r2), p[i], dwq[i]); dwq[4 + i] = fma2(mul2(y[i], r2), q[i], dwq[4 + i]); }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              ulonglong2* at = reinterpret_cast<ulonglong2*>(dwk[warp][j][lane]);
              ulonglong2 v = *at;
              const F2* xx = j < 2 ? x + 2 * j : y + 2 * (j - 2);
              const F2* pp = j < 2 ? p + 2 * j : q + 2 * (j - 2);
              v.x = fma2(mul2(xx[0], r2), pp[0], v.x);
              v.y = fma2(mul2(xx[1], r2), pp[1], v.y);
              *at = v;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = mul2(r2, fma2(x[i], t2, mul2(w0[i], p[i])));
            y[i] = mul2(r2, fma2(y[i], t2, mul2(w1[i], q[i])));
          }
          out[h * kChunks + piece] = pack8(x);
          out[h * kChunks + kLanes + piece] = pack8(y);
        } else if (h < heads) {
          out[h * kChunks + piece] = glo[k];
          out[h * kChunks + kLanes + piece] = ghi[k];
        }
      }
    }
    if (a.partial != nullptr && (--left == 0 || u + step >= a.units)) {   // the lanes' sums to the warp's
      left = a.fold;
#pragma unroll
      for (int j = 0; j < 4; ++j) {               // four coordinates of q and of k
        const float4 k4 = *reinterpret_cast<const float4*>(dwk[warp][j][lane]);
        float v[8] = {0.f, 0.f, 0.f, 0.f, k4.x, k4.y, k4.z, k4.w};
        split(dwq[2 * j], v, v + 1);
        split(dwq[2 * j + 1], v + 2, v + 3);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int d = kLanes; d < 32; d <<= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        if (sub < 2) {                            // one lane of each piece keeps the query heads' sums, one the key heads'
          float4* at = reinterpret_cast<float4*>(&sums[warp][sub][(j >> 1) * (D / 2) + piece * 8 + (j & 1) * 4]);
          const float4 s4 = *at;
          *at = sub == 0 ? make_float4(s4.x + v[0], s4.y + v[1], s4.z + v[2], s4.w + v[3])
                         : make_float4(s4.x + v[4], s4.y + v[5], s4.z + v[6], s4.w + v[7]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) dwq[i] = pair(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(dwk[warp][i][lane]) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  if (a.partial == nullptr) return;
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const float* col = &sums[0][0][0] + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int v = 0; v < kWarps; ++v) t += col[v * 2 * D];
    a.partial[(int64_t)blockIdx.x * 2 * D + threadIdx.x] = t;
  }
}

// Adds the blocks' sums: a block has 32 of the 2 D columns, 32 threads per column.
__global__ void __launch_bounds__(1024) k_norm_rope_weights(const float* __restrict__ partial, int blocks, int D, float* __restrict__ dq_weight,
                                                           float* __restrict__ dk_weight) {
  asm volatile("griddepcontrol.wait;" ::: "memory");           // the launch may begin while the kernel ahead ends
  __shared__ float sh[32][33];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5, col = (int)blockIdx.x * 32 + lane;
  float t = 0.f;
#pragma unroll 10
  for (int b = grp; b < blocks; b += 32) t += partial[(int64_t)b * 2 * D + col];
  sh[grp][lane] = t;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int g = 1; g < 32; ++g) t += sh[g][lane];
    float* dst = col < D ? dq_weight : dk_weight;
    if (dst != nullptr) dst[col % D] = t;
  }
}

constexpr int kMaxGradBlocks = 148 * 2;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Few rows: several warps share a row's heads, down to one pass each, until there is a unit for each of the 16 warps per SM;
// and while that leaves `ahead` passes per unit, until there are about six, so that the last round of units is a small part
// of the whole (8192 rows of 48 heads, the gradient: 63.7 us in 3.5 rounds, 60.8 us in 6.9).
int row_split(int64_t n, int heads, int head_dim, int ahead) {
  const int passes = (heads * (head_dim / 16) + 31) / 32;
  int split = 1;
  while (split < passes && (n * split < 148 * 16 || (n * split < 148 * 16 * 6 && passes >= 2 * split * ahead))) split *= 2;
  return split < passes ? split : passes;
}

bc_status check(int64_t n, int q_heads, int kv_heads, int head_dim, const void* qkv, int64_t row_stride, const int32_t* positions,
                float theta, const void* q_weight, const void* k_weight, float eps) {
  if (n <= 0 || q_heads < 1 || kv_heads < 1 || !qkv || !positions || !(theta > 1.f) || !(eps >= 0.f)) return BC_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return BC_ERR_UNSUPPORTED;
  if ((int64_t)q_heads + 2 * (int64_t)kv_heads > (1 << 20)) return BC_ERR_UNSUPPORTED;
  if (row_stride < (int64_t)(q_heads + 2 * kv_heads) * head_dim || row_stride % 8) return BC_ERR_INVALID_ARG;
  if (!aligned16(qkv) || (reinterpret_cast<uintptr_t>(positions) & 3) || !aligned16(q_weight) || !aligned16(k_weight)) return BC_ERR_INVALID_ARG;
  return BC_OK;
}

}  // namespace

extern "C" {

bc_status bc_norm_rope_split(int32_t n, int32_t q_heads, int32_t kv_heads, int32_t head_dim, const void* qkv, int64_t row_stride,
                             const int32_t* positions, float theta, const void* q_weight, const void* k_weight, float eps,
                             void* q_out, void* k_out, void* v_out, void* stream) {
  const bc_status st = check(n, q_heads, kv_heads, head_dim, qkv, row_stride, positions, theta, q_weight, k_weight, eps);
  if (st) return st;
  if (!q_out || !k_out || !v_out || !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out)) return BC_ERR_INVALID_ARG;
  NormRopeArgs a;
  a.qkv = (const uint8_t*)qkv; a.row_bytes = row_stride * 2; a.positions = positions;
  a.q_weight = (const uint4*)q_weight; a.k_weight = (const uint4*)k_weight;
  a.q_out = (uint4*)q_out; a.k_out = (uint4*)k_out; a.v_out = (uint4*)v_out;
  a.q_heads = q_heads; a.kv_heads = kv_heads; a.split = row_split(n, q_heads + 2 * kv_heads, head_dim, 4);
  a.units = (int64_t)n * a.split; a.log2_theta = log2((double)theta); a.eps = eps;
  const int64_t want = (a.units + kWarps - 1) / kWarps;
  const int blocks = (int)(want < 148 * 2 ? want : 148 * 2);   // two resident blocks per SM
  if (head_dim == 64) k_norm_rope<64><<<blocks, kThreads, 0, (cudaStream_t)stream>>>(a);
  else k_norm_rope<128><<<blocks, kThreads, 0, (cudaStream_t)stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}

bc_status bc_norm_rope_query_bytes(int32_t head_dim, size_t* workspace_bytes) {
  if (!workspace_bytes) return BC_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return BC_ERR_UNSUPPORTED;
  *workspace_bytes = (size_t)kMaxGradBlocks * 2 * head_dim * sizeof(float);
  return BC_OK;
}

bc_status bc_norm_rope_split_backward(int32_t n, int32_t q_heads, int32_t kv_heads, int32_t head_dim, const void* qkv,
                                      int64_t row_stride, const int32_t* positions, float theta, const void* q_weight,
                                      const void* k_weight, float eps, const void* dq, const void* dk, const void* dv, void* dqkv,
                                      float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  const bc_status st = check(n, q_heads, kv_heads, head_dim, qkv, row_stride, positions, theta, q_weight, k_weight, eps);
  if (st) return st;
  if (!dq || !dk || !dv || !dqkv || !workspace || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(dqkv) ||
      !aligned16(workspace) || ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 3))
    return BC_ERR_INVALID_ARG;
  if (workspace_bytes < (size_t)kMaxGradBlocks * 2 * head_dim * sizeof(float)) return BC_ERR_INVALID_ARG;
  NormRopeGradArgs a;
  a.qkv = (const uint8_t*)qkv; a.row_bytes = row_stride * 2; a.positions = positions;
  a.q_weight = (const __nv_bfloat16*)q_weight; a.k_weight = (const __nv_bfloat16*)k_weight;
  a.dq = (const uint4*)dq; a.dk = (const uint4*)dk; a.dv = (const uint4*)dv; a.dqkv = (uint4*)dqkv;
  const bool weights = dq_weight != nullptr || dk_weight != nullptr;
  a.partial = weights ? (float*)workspace : nullptr;
  a.q_heads = q_heads; a.kv_heads = kv_heads; a.log2_theta = log2((double)theta); a.eps = eps;
  a.split = row_split(n, q_heads + 2 * kv_heads, head_dim, 2);
  a.units = (int64_t)n * a.split;
  const int per_pass = 32 / (head_dim / 16) * a.split, terms = (q_heads + 2 * kv_heads + per_pass - 1) / per_pass;   // of a lane, per unit, at most
  a.fold = terms < kFoldTerms ? kFoldTerms / terms : 1;
  const int64_t want = (a.units + kWarps - 1) / kWarps;
  const int blocks = (int)(want < kMaxGradBlocks ? want : kMaxGradBlocks);
  cudaStream_t s = (cudaStream_t)stream;
  if (head_dim == 64) k_norm_rope_grad<64><<<blocks, kThreads, 0, s>>>(a);
  else k_norm_rope_grad<128><<<blocks, kThreads, 0, s>>>(a);
  if (cudaGetLastError() != cudaSuccess) return BC_ERR_CUDA;
  if (!weights) return BC_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * head_dim / 32)); cfg.blockDim = dim3(1024); cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_norm_rope_weights, (const float*)a.partial, blocks, (int)head_dim, dq_weight, dk_weight);
  return e == cudaSuccess ? BC_OK : BC_ERR_CUDA;
}

}  // extern "C"
