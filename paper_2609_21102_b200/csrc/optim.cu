// The optimizer step of what Muon does not take: AdamW over a list of tensors in one launch per type, moments in 32 or in
// 8 bits, and the global norm of a list of gradients with the clipping factor kept on the device.
//
// Tables. A call's list of tensors travels in the kernel's parameters (up to 32 KB), not in device memory: no buffer to
// keep alive, no copy before the launch, and a captured graph holds its own list. A list that does not fit goes through in
// several launches.
#include "../../include/defl.h"
#include "ctx.cuh"
#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

namespace defl {
namespace {

constexpr int OPT_THREADS = 256;
constexpr int CHUNK = 2048;                       // elements of one CTA's trip: 8 a thread, a block of 256 a warp
// Tensors a launch. The largest tables stay within the 32,764 bytes that a launch's parameters may take (31.7 and 31.2 KB); a launch copies its
// parameters whole, which the smaller ones save (us on the host with the largest table, the middle one and the smallest; graphs do not care:
// AdamW 4 tensors 4.7 3.8 3.3, 48 tensors 6.6 5.6 5.2, 160 tensors 10.8 9.8; norm 4 tensors 6.9 5.8 5.1, 48 7.5 6.4 5.9, 386 12.1 10.8).
constexpr int ADAM_CAP = 438, ADAM_CAP_SMALL = 48, ADAM_CAP_MID = 160;
constexpr int NORM_CAP = 1300, NORM_CAP_MID = 440, NORM_CAP_SMALL = 48;
constexpr int NORM_BLOCKS = 592;                  // four CTAs on each of 148 SMs
constexpr int NORM_CHUNK = 4 * CHUNK;

struct AdamTensor {
  void* p; const void* g; void* m; void* v; float* ms; float* vs; void* copy;
  long long n;
  unsigned int first;          // number of chunks before this tensor
  int index;                   // its place in the caller's list; the sign bit: all rows start on 16-byte boundaries
};
struct AdamHyper {
  double beta1, beta2, lr, decay;
  long long step;
  const long long* step_dev; const float* lr_dev; const float* grad_scale;
  unsigned long long seed;     // the generator's h(seed)
  float b1, ob1, b2, ob2, eps;
  int known;                   // step and learning rate came from the host: what follows from them is here already
  float size, rc2, keep;
  unsigned long long key_base;
};
template <int CAP>
struct AdamTable {
  AdamHyper h;
  int count;
  unsigned int chunks;
  AdamTensor t[CAP];
};
static_assert(sizeof(AdamTable<ADAM_CAP>) <= 32764, "kernel parameters");

// The last tensor, from number i on, that starts at or before this chunk. (Mostly number i itself; else by halves: a walk through
// hundreds of small tensors behind a large one took 20 us.)
template <typename Table>
__device__ __forceinline__ int find_tensor(const Table& tb, int i, unsigned int chunk) {
  int hi = tb.count - 1;
  if (i >= hi || tb.t[i + 1].first > chunk) return i;
  for (++i; i < hi;) {
    const int mid = (i + hi + 1) >> 1;
    if (tb.t[mid].first <= chunk) i = mid; else hi = mid - 1;
  }
  return i;
}

// the mixing function of defl_fill_gaussian's generator
__host__ __device__ __forceinline__ unsigned long long mix64(unsigned long long x) {
  x += 0x9E3779B97F4A7C15ull;
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

// beta^t by squaring: 2 log2(t) products, each good to 2^-53
__host__ __device__ inline double power_of(double b, long long t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

struct Scalars { float size, rc2, keep, c; };     // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), 1 - lr * decay, gradient factor

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// eight consecutive values, 16-byte accesses
template <typename T> __device__ __forceinline__ void load8(const T* s, float* x);
template <> __device__ __forceinline__ void load8<float>(const float* s, float* x) {
  const float4 a = reinterpret_cast<const float4*>(s)[0], b = reinterpret_cast<const float4*>(s)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* s, float* x) {
  const uint4 a = *reinterpret_cast<const uint4*>(s);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
}
__device__ __forceinline__ void store8(float* d, const float* x) {
  reinterpret_cast<float4*>(d)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(d)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* d, const float* x) {
  uint4 q;
  q.x = pack16x2(x[0], x[1], false); q.y = pack16x2(x[2], x[3], false);
  q.z = pack16x2(x[4], x[5], false); q.w = pack16x2(x[6], x[7], false);
  *reinterpret_cast<uint4*>(d) = q;
}

__device__ __forceinline__ float2 e4m3x2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(__half2(h));
}
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// y >= 0 to a neighbouring e4m3 value, up with the probability of the part that is cut off. y * 2^-120 has e4m3's exponents in fp32's
// exponent field, and what is subnormal there is subnormal here: the bits above the 20 lowest are the code, in both ranges, and 16 random bits
// are added below them. (A block's largest y is 448 give or take two units of fp32: with those and all 16 bits set it still does
// not reach the next spacing, so 448 stays 448.) Returns the code at bit 20.
__device__ __forceinline__ uint32_t e4m3_stochastic(float y, uint32_t bits16) {
  return __float_as_uint(y * 7.52316384526264e-37f) + (bits16 << 4);
}

// fp32 to bf16 by 16 random bits, kept as fp32; Inf and NaN stay what they are
__device__ __forceinline__ float bf16_stochastic(float x, uint32_t bits16) {
  const uint32_t z = (__float_as_uint(x) + bits16) & 0xFFFF0000u;
  return fabsf(x) < __int_as_float(0x7f800000) ? __uint_as_float(z) : x;
}

// One element: m, v and p in fp32, root <- sqrt(v). Every operation of the moments rounds by itself (no fused multiply-add), so
// that what is held in 8 bits is the same to the bit wherever the step is computed in fp32: a value that lands on another
// code moves its block's scale in a later step.
__device__ __forceinline__ void adam_one(const AdamHyper& h, const Scalars& s, float g, float& p, float& m, float& v, float& root) {
  g = __fmul_rn(g, s.c);
  m = __fadd_rn(__fmul_rn(h.b1, m), __fmul_rn(h.ob1, g));
  v = __fadd_rn(__fmul_rn(h.b2, v), __fmul_rn(h.ob2, __fmul_rn(g, g)));
  root = sqrtf(v);
  // the reciprocal of a subnormal is taken as that of zero: a root is 0 or above 2^-75, so that only an eps below fp32's normal numbers
  // counts as zero. (80M elements in 8 bits 242 -> 232 us against a division that minds the ends of the range.)
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(fmaf(root, s.rc2, h.eps)));
  p = fmaf(-s.size, m * inv, p * s.keep);
}

// the largest magnitude of three; a NaN is the largest
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// What is held of a block of 256 values in 8 bits: the factor that brings its largest magnitude to 448, and the scale. (Below
// 2^-100 a block counts as zero: the factor would leave fp32. A NaN or Inf makes the scale NaN, and the block with it.) Both moments at
// once, the first's in the lower lanes and the second's in the upper ones: the divisions are paid once.
__device__ __forceinline__ void block_scales(float big_m, float big_r, int lane, float& inv_m, float& inv_r, float* ms, float* vs) {
  const uint32_t bm = __reduce_max_sync(0xffffffffu, __float_as_uint(big_m) & 0x7fffffffu);     // magnitudes order as their bits, NaN above all
  const uint32_t br = __reduce_max_sync(0xffffffffu, __float_as_uint(big_r) & 0x7fffffffu);
  const uint32_t bits = lane < 16 ? bm : br;
  const float b = __uint_as_float(bits);
  const bool some = b > 7.888609052210118e-31f;
  const float inv = some ? 448.f / b : 0.f;
  float scale = some ? b / 448.f : 0.f;
  if (bits >= 0x7f800000u) scale = __int_as_float(0x7fffffff);
  inv_m = __shfl_sync(0xffffffffu, inv, 0);
  inv_r = __shfl_sync(0xffffffffu, inv, 16);
  if ((lane & 15) == 0) *(lane ? vs : ms) = scale;
}

// One block of 256 elements (`left` of them exist) by one warp. VEC: all of them exist and everything starts on 16-byte
// boundaries, a lane has 8 consecutive ones; else it has one in 32, so that the single accesses of a warp touch as few lines.
template <typename P, typename G, bool EIGHT, bool SR, bool VEC>
__device__ __forceinline__ void adam_block(const AdamTensor& t, const AdamHyper& h, const Scalars& s, unsigned long long key,
                                           long long base, long long left, int lane) {
  P* const pp = reinterpret_cast<P*>(t.p) + base;
  const G* const gp = reinterpret_cast<const G*>(t.g) + base;
  uint8_t* const m8 = reinterpret_cast<uint8_t*>(t.m) + base;
  uint8_t* const v8 = reinterpret_cast<uint8_t*>(t.v) + base;
  float* const m32 = reinterpret_cast<float*>(t.m) + base;
  float* const v32 = reinterpret_cast<float*>(t.v) + base;
  const long long block = base >> 8;
  const float s_m = EIGHT ? t.ms[block] : 0.f, s_v = EIGHT ? t.vs[block] : 0.f;
  float p[8], g[8], m[8], v[8], big_m = 0.f, big_r = 0.f;
  if (VEC) {
    load8(pp + 8 * lane, p);
    load8(gp + 8 * lane, g);
    if (EIGHT) {
      const uint2 qm = reinterpret_cast<const uint2*>(m8)[lane], qv = reinterpret_cast<const uint2*>(v8)[lane];
      const uint32_t wm[2] = {qm.x, qm.y}, wv[2] = {qv.x, qv.y};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 a = e4m3x2((wm[j >> 1] >> (16 * (j & 1))) & 0xFFFFu), b = e4m3x2((wv[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
        m[2 * j] = a.x; m[2 * j + 1] = a.y; v[2 * j] = b.x; v[2 * j + 1] = b.y;
      }
    } else {
      load8(m32 + 8 * lane, m);
      load8(v32 + 8 * lane, v);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = lane + 32 * j;
      const bool on = e < left;
      p[j] = on ? to_f(pp[e]) : 0.f;
      g[j] = on ? to_f(gp[e]) : 0.f;
      m[j] = !on ? 0.f : EIGHT ? e4m3x2(m8[e]).x : m32[e];
      v[j] = !on ? 0.f : EIGHT ? e4m3x2(v8[e]).x : v32[e];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (EIGHT) { m[j] *= s_m; v[j] *= s_v; v[j] *= v[j]; }
    float root;
    adam_one(h, s, g[j], p[j], m[j], v[j], root);
    if (EIGHT) {
      v[j] = root;                                 // what is held
      if (j & 1) {
        big_m = max_abs3(big_m, m[j - 1], m[j]);
        big_r = max_abs3(big_r, v[j - 1], v[j]);
      }
    }
  }
  float inv_m = 0.f, inv_r = 0.f;
  if (EIGHT) {
    block_scales(big_m, big_r, lane, inv_m, inv_r, t.ms + block, t.vs + block);
  }
  uint32_t cm[4], cv[4];                           // two codes each
  const unsigned long long lane_key = key ^ (unsigned long long)((base >> 1) + (VEC ? 4 * lane : lane >> 1));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t bits[2] = {0, 0};
    if (SR) {
      if (VEC) {
        const unsigned long long w = mix64(lane_key ^ (unsigned long long)j);      // (base / 2 + 4 lane is a multiple of four)
        bits[0] = (uint32_t)w; bits[1] = (uint32_t)(w >> 32);
      } else {
        // two neighbouring lanes hold the halves of a pair: the even lane makes the word of their pair 2 j, the odd one of 2 j + 1
        const int odd = lane & 1;
        const unsigned long long w = mix64(lane_key ^ (unsigned long long)(16 * (2 * j + odd)));
        const uint32_t mine = odd ? (uint32_t)(w >> 32) : (uint32_t)w;
        const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? (uint32_t)w : (uint32_t)(w >> 32), 1);
        bits[0] = odd ? other : mine; bits[1] = odd ? mine : other;
      }
    }
    uint32_t qm[2], qv[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = 2 * j + k;
      if (SR && sizeof(P) == 2) p[i] = bf16_stochastic(p[i], bits[k] >> 16);
      if (EIGHT) {
        const float a = fabsf(m[i]) * inv_m, b = v[i] * inv_r;
        // the root of what is not zero does not become zero: the moment beside it may be larger than its step's gradient,
        // and would be divided by eps alone. (A root that is not zero is above 2^-75.)
        if (SR) {
          qm[k] = e4m3_stochastic(a, bits[k] & 0xFFFFu);
          qv[k] = max(e4m3_stochastic(b, bits[k] >> 16), min(__float_as_uint(v[i]), 1u << 20));
        } else {
          m[i] = copysignf(a, m[i]);
          v[i] = b > 0.f ? fmaxf(b, 0.001953125f) : b;
        }
      }
    }
    if (EIGHT && SR) {
      cm[j] = (qm[0] >> 20 | (qm[1] >> 20) << 8) | (__byte_perm(__float_as_uint(m[2 * j]), __float_as_uint(m[2 * j + 1]), 0x73) & 0x8080u);
      cv[j] = qv[0] >> 20 | (qv[1] >> 20) << 8;
    } else if (EIGHT) {
      cm[j] = to_e4m3x2(m[2 * j], m[2 * j + 1]);
      cv[j] = to_e4m3x2(v[2 * j], v[2 * j + 1]);
    }
  }
  if (VEC) {
    store8(pp + 8 * lane, p);
    if (t.copy) store8(reinterpret_cast<__nv_bfloat16*>(t.copy) + base + 8 * lane, p);
    if (EIGHT) {
      reinterpret_cast<uint2*>(m8)[lane] = make_uint2(cm[0] | (cm[1] << 16), cm[2] | (cm[3] << 16));
      reinterpret_cast<uint2*>(v8)[lane] = make_uint2(cv[0] | (cv[1] << 16), cv[2] | (cv[3] << 16));
    } else {
      store8(m32 + 8 * lane, m);
      store8(v32 + 8 * lane, v);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = lane + 32 * j;
      if (e < left) {
        pp[e] = (P)p[j];
        if (t.copy) reinterpret_cast<__nv_bfloat16*>(t.copy)[base + e] = __float2bfloat16_rn(p[j]);
        if (EIGHT) {
          m8[e] = (uint8_t)(cm[j >> 1] >> (8 * (j & 1)));
          v8[e] = (uint8_t)(cv[j >> 1] >> (8 * (j & 1)));
        } else {
          m32[e] = m[j];
          v32[e] = v[j];
        }
      }
    }
  }
}

// Bytes an element with fp32 weights and bf16 gradients: 26 with 32-bit moments, 14.1 with 8-bit ones; what HBM can bring of
// that in a second leaves 150 and 77 instructions an element. 80M elements on a B200: 313 us with 32-bit moments (6.7 TB/s: bound by HBM; bf16
// weights 264, to nearest or random), with 8-bit ones 191 to nearest and 231 with random bits, which are bound by the issue of instructions (84
// an element, 82 % of the slots taken; under the power cap of half a second without a pause 257): the generator's two 64-bit products and shifts
// take 28 us of that, the exact square root 14. Two blocks a trip take registers that spill (276; as it is, 16 bytes do), three CTAs an SM
// leave too little to hide (255).
template <typename P, typename G, bool EIGHT, bool SR, int CAP>
__global__ void __launch_bounds__(OPT_THREADS, 4) adamw_kernel(const __grid_constant__ AdamTable<CAP> tb) {
  __shared__ Scalars sc;
  __shared__ unsigned long long shared_key;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const AdamHyper& h = tb.h;
  unsigned int chunk = blockIdx.x;
  int i = find_tensor(tb, 0, chunk);
  pdl_wait();
  Scalars s = {h.size, h.rc2, h.keep, h.grad_scale ? *h.grad_scale : 1.f};
  unsigned long long key_base = h.key_base;
  if (!h.known) {
    if (warp == 0) {
      const long long t0 = h.step_dev ? *h.step_dev : h.step, t = t0 > 0 ? t0 : 1;
      // two lanes, one correction each
      const double corr = 1.0 - power_of(lane == 0 ? h.beta1 : h.beta2, t);
      const double lr = h.lr_dev ? (double)*h.lr_dev : h.lr;
      if (lane == 0) {
        sc.size = (float)(lr / corr);
        sc.keep = (float)(1.0 - lr * h.decay);
        shared_key = mix64(h.seed ^ (unsigned long long)t);
      } else if (lane == 1) {
        sc.rc2 = (float)(1.0 / sqrt(corr));
      }
    }
    __syncthreads();
    s.size = sc.size; s.rc2 = sc.rc2; s.keep = sc.keep;
    key_base = shared_key;
  }
  if (s.c == 0.f) return;                          // gradients that were not finite: the step is left out
  for (; chunk < tb.chunks; chunk += gridDim.x) {
    i = find_tensor(tb, i, chunk);
    const AdamTensor& t = tb.t[i];
    const long long base = (long long)(chunk - t.first) * CHUNK + warp * 256, left = t.n - base;      // this warp's block
    if (left <= 0) continue;
    const unsigned long long key = SR ? mix64(key_base ^ (unsigned long long)(t.index & 0x7fffffff)) : 0ull;
    if (t.index < 0 && left >= 256) adam_block<P, G, EIGHT, SR, true>(t, tb.h, s, key, base, left, lane);
    else adam_block<P, G, EIGHT, SR, false>(t, tb.h, s, key, base, left, lane);
  }
}

// ---------------------------------------------------------------------------------------------
struct NormTensor {
  const void* x;
  long long n;
  unsigned int first;
  int dtype;                   // DEFL_F32 or DEFL_BF16; the sign bit: starts on a 16-byte boundary
};
template <int CAP>
struct NormTable {
  double* partial;             // one slot a CTA
  int count;
  unsigned int chunks;
  NormTensor t[CAP];
};
static_assert(sizeof(NormTable<NORM_CAP>) <= 32764, "kernel parameters");

// Eight squares are summed in fp32 and the sums in fp64: a conversion an element would cost as much as the loads (16 a cycle
// and SM). Sums that left fp32's range at either end are formed again in fp64.
__device__ __forceinline__ double squares8(const float* x) {
  float a = x[0] * x[0], b = x[1] * x[1];
#pragma unroll
  for (int j = 2; j < 8; j += 2) { a = fmaf(x[j], x[j], a); b = fmaf(x[j + 1], x[j + 1], b); }
  const float q = a + b;
  if (q > 1e-30f && q < 1e38f) return (double)q;
  double d = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) d = fma((double)x[j], (double)x[j], d);
  return d;
}

__device__ __forceinline__ double block_sum(double acc, double* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = acc;
  __syncthreads();
  double d = 0.0;
  for (int w = 0; w < OPT_THREADS / 32; ++w) d += part[w];
  return d;
}

// Reads 2 or 4 bytes an element and writes nothing, so four loads of a thread are in flight. bf16: 80M elements 44 us, the 1.47G of a model 717:
// 4.1 of the 6.5 TB/s that HBM brings; what keeps it there has not been taken apart.
template <int CAP>
__global__ void __launch_bounds__(OPT_THREADS) grad_norm_kernel(const __grid_constant__ NormTable<CAP> tb) {
  __shared__ double part[OPT_THREADS / 32];
  pdl_wait();
  double acc = 0.0;
  int i = 0;
  for (unsigned int chunk = blockIdx.x; chunk < tb.chunks; chunk += gridDim.x) {
    i = find_tensor(tb, i, chunk);
    const NormTensor& t = tb.t[i];
    const long long base = (long long)(chunk - t.first) * NORM_CHUNK + threadIdx.x * 8;
    const long long left = t.n - base;
    float x[NORM_CHUNK / CHUNK][8];
    const bool bf16 = (t.dtype & 0xFF) == BF16, vec = t.dtype < 0;
#pragma unroll
    for (int u = 0; u < NORM_CHUNK / CHUNK; ++u) {
      const long long at = base + u * CHUNK, rest = left - u * CHUNK;
      if (vec && rest >= 8) {
        if (bf16) load8(reinterpret_cast<const __nv_bfloat16*>(t.x) + at, x[u]); else load8(reinterpret_cast<const float*>(t.x) + at, x[u]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[u][j] = j < rest ? (bf16 ? to_f(reinterpret_cast<const __nv_bfloat16*>(t.x)[at + j]) : reinterpret_cast<const float*>(t.x)[at + j]) : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < NORM_CHUNK / CHUNK; ++u) acc += squares8(x[u]);
  }
  acc = block_sum(acc, part);
  if (threadIdx.x == 0) tb.partial[blockIdx.x] = acc;
}

// All partial sums in a fixed order, then the factor. (A launch of its own and not the work of the CTA that ends last: that
// would need a counter that is zero beforehand, which a buffer given for one call is not.)
__global__ void __launch_bounds__(OPT_THREADS) grad_norm_finish_kernel(const double* partial, int slots, float max_norm, float* out, long long* step) {
  __shared__ double part[OPT_THREADS / 32];
  pdl_wait();
  double acc = 0.0;
  for (int k = threadIdx.x; k < slots; k += OPT_THREADS) acc += partial[k];
  acc = block_sum(acc, part);
  if (threadIdx.x == 0) {
    const double norm = sqrt(acc);
    const float nf = (float)norm;
    const bool finite = nf < __int_as_float(0x7f800000);
    double f = 1.0;
    if (max_norm > 0.f) { f = (double)max_norm / (norm + 1e-6); if (f > 1.0) f = 1.0; }
    out[0] = nf;
    out[1] = finite ? (float)f : 0.f;
    if (step && finite) *step += 1;
  }
}

bool on16(const void* p) { return on(p, 16); }

template <typename P, typename G, bool EIGHT, bool SR, int CAP>
cudaError_t adamw_launch(const AdamTable<ADAM_CAP>& tb, int num_sms, cudaStream_t st) {
  AdamTable<CAP> small;
  const AdamTable<CAP>* arg;
  if (CAP == ADAM_CAP) {
    arg = reinterpret_cast<const AdamTable<CAP>*>(&tb);
  } else {
    small.h = tb.h; small.count = tb.count; small.chunks = tb.chunks;
    memcpy(small.t, tb.t, sizeof(AdamTensor) * tb.count);
    arg = &small;
  }
  // (sixty-four CTAs an SM, of which four at a time: with eight, or with four that stay, 80M elements took 366 and 379 us in 32 bits, now 312)
  const unsigned int most = (unsigned int)num_sms * 64u;
  return launch_kernel(adamw_kernel<P, G, EIGHT, SR, CAP>, dim3(tb.chunks < most ? tb.chunks : most), dim3(OPT_THREADS), 0, st, *arg);
}
template <typename P, typename G, int CAP>
cudaError_t adamw_pick(const AdamTable<ADAM_CAP>& tb, bool eight, bool sr, int sms, cudaStream_t st) {
  if (eight) return sr ? adamw_launch<P, G, true, true, CAP>(tb, sms, st) : adamw_launch<P, G, true, false, CAP>(tb, sms, st);
  if constexpr (sizeof(P) == 2)                   // (with fp32 weights and 32-bit moments nothing is left to round)
    if (sr) return adamw_launch<P, G, false, true, CAP>(tb, sms, st);
  return adamw_launch<P, G, false, false, CAP>(tb, sms, st);
}
template <int CAP>
cudaError_t adamw_type(const AdamTable<ADAM_CAP>& tb, int cls, bool sr, int sms, cudaStream_t st) {
  const bool eight = (cls & 1) != 0;
  switch (cls >> 1) {
    case 0: return adamw_pick<float, float, CAP>(tb, eight, sr, sms, st);
    case 1: return adamw_pick<float, __nv_bfloat16, CAP>(tb, eight, sr, sms, st);
    case 2: return adamw_pick<__nv_bfloat16, float, CAP>(tb, eight, sr, sms, st);
    default: return adamw_pick<__nv_bfloat16, __nv_bfloat16, CAP>(tb, eight, sr, sms, st);
  }
}

template <int CAP>
cudaError_t norm_launch(const NormTable<NORM_CAP>& tb, int grid, cudaStream_t st) {
  NormTable<CAP> small;
  const NormTable<CAP>* arg;
  if (CAP == NORM_CAP) {
    arg = reinterpret_cast<const NormTable<CAP>*>(&tb);
  } else {
    memcpy(&small, &tb, sizeof(small));             // the head and the first CAP tensors
    arg = &small;
  }
  return launch_kernel(grad_norm_kernel<CAP>, dim3(grid), dim3(OPT_THREADS), 0, st, *arg);
}

constexpr long long MAX_ELEMENTS = 1ll << 40;

// types of weights, gradient and moments as one number
int type_class(const defl_adamw_tensor& x) {
  return (x.p_dtype == DEFL_BF16 ? 4 : 0) + (x.g_dtype == DEFL_BF16 ? 2 : 0) + (x.state_bits == 8 ? 1 : 0);
}

}  // namespace

}  // namespace defl

using namespace defl;

extern "C" {

int defl_adamw_step(defl_ctx* c, const defl_adamw_tensor* t, int count, const defl_adamw_opts* o) {
  if (!c || count < 0 || (count > 0 && !t) || !o) return DEFL_ERR_ARG;
  if (!(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0) || !(o->eps >= 0.0) || !isfinite(o->eps) ||
      !isfinite(o->lr) || !isfinite(o->weight_decay)) return DEFL_ERR_ARG;
  if (!o->step_dev && o->step < 1) return DEFL_ERR_ARG;
  if (!on(o->step_dev, 8) || !on(o->lr_dev, 4) || !on(o->grad_scale, 4)) return DEFL_ERR_ARG;
  unsigned long long total = 0;
  unsigned int present = 0;                       // the combinations of types that the list holds
  AdamTable<ADAM_CAP> tb;
  auto start = [&] { tb.count = 0; tb.chunks = 0; };
  auto put = [&](int i) {
    const defl_adamw_tensor& x = t[i];
    AdamTensor& d = tb.t[tb.count++];
    d.p = x.p; d.g = x.g; d.m = x.m; d.v = x.v; d.ms = x.m_scale; d.vs = x.v_scale; d.copy = x.copy; d.n = x.n;
    d.first = tb.chunks;
    const bool aligned = on16(x.p) && on16(x.g) && on16(x.m) && on16(x.v) && on16(x.copy);
    d.index = (int)((unsigned int)i | (aligned ? 0x80000000u : 0u));
    tb.chunks += (unsigned int)((x.n + CHUNK - 1) / CHUNK);
  };
  // the usual list, of one combination of types and no longer than a table, is put down while it is looked through
  bool whole = true;
  start();
  for (int i = 0; i < count; ++i) {
    const defl_adamw_tensor& x = t[i];
    if (x.n < 0 || x.n > MAX_ELEMENTS) return DEFL_ERR_ARG;
    if (x.n == 0 || !x.g) continue;
    if (!x.p || !x.m || !x.v) return DEFL_ERR_ARG;
    if ((x.p_dtype != DEFL_F32 && x.p_dtype != DEFL_BF16) || (x.g_dtype != DEFL_F32 && x.g_dtype != DEFL_BF16)) return DEFL_ERR_ARG;
    if (x.state_bits != 32 && x.state_bits != 8) return DEFL_ERR_ARG;
    if (x.state_bits == 8 && (!x.m_scale || !x.v_scale || !on(x.m_scale, 4) || !on(x.v_scale, 4))) return DEFL_ERR_ARG;
    if (!on(x.p, (unsigned)dtype_size(x.p_dtype)) || !on(x.g, (unsigned)dtype_size(x.g_dtype)) || !on(x.copy, 2)) return DEFL_ERR_ARG;
    if (x.state_bits == 32 && (!on(x.m, 4) || !on(x.v, 4))) return DEFL_ERR_ARG;
    present |= 1u << type_class(x);
    whole = whole && (present & (present - 1)) == 0 && tb.count < ADAM_CAP;
    if (whole) put(i);
    total += (unsigned long long)((x.n + CHUNK - 1) / CHUNK);
  }
  if (total > 0x7fffffffull) return DEFL_ERR_RANK;
  DeviceScope scope(c->device);
  c->err[0] = 0;
  AdamHyper& h = tb.h;
  h.beta1 = o->beta1; h.beta2 = o->beta2; h.lr = o->lr; h.decay = o->weight_decay;
  h.step = o->step; h.step_dev = reinterpret_cast<const long long*>(o->step_dev); h.lr_dev = o->lr_dev; h.grad_scale = o->grad_scale;
  h.seed = mix64(o->seed);
  h.known = !o->step_dev && !o->lr_dev;
  h.size = h.rc2 = h.keep = 0.f;
  h.key_base = 0;
  if (h.known) {
    h.size = (float)(o->lr / (1.0 - power_of(o->beta1, o->step)));
    h.rc2 = (float)(1.0 / sqrt(1.0 - power_of(o->beta2, o->step)));
    h.keep = (float)(1.0 - o->lr * o->weight_decay);
    h.key_base = mix64(h.seed ^ (unsigned long long)o->step);
  }
  h.b1 = (float)o->beta1; h.ob1 = (float)(1.0 - o->beta1); h.b2 = (float)o->beta2; h.ob2 = (float)(1.0 - o->beta2); h.eps = (float)o->eps;
  for (int cls = 0; cls < 8; ++cls) {
    if (!(present >> cls & 1u)) continue;
    for (int i = 0; i < count;) {
      if (whole) {
        i = count;
      } else {
        start();
        for (; i < count && tb.count < ADAM_CAP; ++i)
          if (t[i].n != 0 && t[i].g && type_class(t[i]) == cls) put(i);
      }
      if (tb.count == 0) break;
      const bool sr = o->stochastic != 0;
      const cudaError_t e = tb.count <= ADAM_CAP_SMALL ? adamw_type<ADAM_CAP_SMALL>(tb, cls, sr, c->num_sms, c->stream)
                            : tb.count <= ADAM_CAP_MID ? adamw_type<ADAM_CAP_MID>(tb, cls, sr, c->num_sms, c->stream)
                                                       : adamw_type<ADAM_CAP>(tb, cls, sr, c->num_sms, c->stream);
      ++c->launches;
      if (ctx_fail(c, e, "adamw")) return DEFL_ERR_CUDA;
    }
  }
  return DEFL_OK;
}

size_t defl_grad_norm_work_bytes(int count) {
  return count < 0 ? 0 : sizeof(double) * NORM_BLOCKS * (size_t)(count <= NORM_CAP ? 1 : (count + NORM_CAP - 1) / NORM_CAP);
}

int defl_grad_norm(defl_ctx* c, const defl_norm_tensor* t, int count, float max_norm, float* out, int64_t* step, void* work) {
  if (!c || count < 0 || (count > 0 && !t) || !out || !work || !on(work, 8) || !on(out, 4) || !on(step, 8) || isnan(max_norm)) return DEFL_ERR_ARG;
  unsigned long long total = 0;
  NormTable<NORM_CAP> tb;
  auto start = [&] { tb.count = 0; tb.chunks = 0; };
  auto put = [&](int i) {
    NormTensor& d = tb.t[tb.count++];
    d.x = t[i].x; d.n = t[i].n; d.first = tb.chunks;
    d.dtype = (int)((unsigned int)t[i].dtype | (on16(t[i].x) ? 0x80000000u : 0u));
    tb.chunks += (unsigned int)((t[i].n + NORM_CHUNK - 1) / NORM_CHUNK);
  };
  bool whole = true;                              // as in defl_adamw_step
  start();
  for (int i = 0; i < count; ++i) {
    if (t[i].n < 0 || t[i].n > MAX_ELEMENTS) return DEFL_ERR_ARG;
    if (t[i].n == 0) continue;
    if (!t[i].x || (t[i].dtype != DEFL_F32 && t[i].dtype != DEFL_BF16) || !on(t[i].x, (unsigned)dtype_size(t[i].dtype))) return DEFL_ERR_ARG;
    whole = whole && tb.count < NORM_CAP;
    if (whole) put(i);
    total += (unsigned long long)((t[i].n + NORM_CHUNK - 1) / NORM_CHUNK);
  }
  if (total > 0x7fffffffull) return DEFL_ERR_RANK;
  DeviceScope scope(c->device);
  c->err[0] = 0;
  double* const partial = reinterpret_cast<double*>(work);
  int slots = 0;
  for (int i = 0; i < count;) {
    if (whole) {
      i = count;
    } else {
      start();
      for (; i < count && tb.count < NORM_CAP; ++i)
        if (t[i].n != 0) put(i);
    }
    if (tb.count == 0) break;
    const int grid = tb.chunks < (unsigned int)NORM_BLOCKS ? (int)tb.chunks : NORM_BLOCKS;
    tb.partial = partial + slots;
    slots += grid;
    const cudaError_t e = tb.count <= NORM_CAP_SMALL ? norm_launch<NORM_CAP_SMALL>(tb, grid, c->stream)
                          : tb.count <= NORM_CAP_MID ? norm_launch<NORM_CAP_MID>(tb, grid, c->stream) : norm_launch<NORM_CAP>(tb, grid, c->stream);
    ++c->launches;
    if (ctx_fail(c, e, "grad norm")) return DEFL_ERR_CUDA;
  }
  ++c->launches;
  if (ctx_fail(c, launch_kernel(grad_norm_finish_kernel, dim3(1), dim3(OPT_THREADS), 0, c->stream, (const double*)partial, slots, max_norm,
                                out, reinterpret_cast<long long*>(step)), "grad norm"))
    return DEFL_ERR_CUDA;
  return DEFL_OK;
}

}  // extern "C"
