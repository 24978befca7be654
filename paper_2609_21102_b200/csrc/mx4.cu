// Microscaled 4-bit floating point: quantisation in one or both block directions from one read, the way back, and the
// products' entry point. Definitions and layout are in include/defl.h.
#include "../../include/defl.h"
#include "ctx.cuh"
#include "mx4.cuh"
#include <cuda_fp8.h>
#include <math.h>
#include <type_traits>

namespace defl {
namespace {

constexpr int TILE = 128;                  // a CTA takes 128 x 128 values: a whole tile of scales in either direction
constexpr int Q_THREADS = 256;
constexpr int MAX_PARTIALS = 592;          // partial maxima a call (four CTAs an SM), at least one a matrix

struct QuantParams {
  const void* X;
  long long ld, batch_stride;
  int b, rows, cols;
  int tiles_c;
  uint8_t* rc; uint8_t* rs; float* rscale;     // blocks along the rows (null: not wanted)
  uint8_t* cc; uint8_t* cs; float* cscale;     // blocks along the columns
  const float* partial;                        // largest finite magnitudes of parts of each matrix (nvfp4)
  int nper;                                    // partial maxima a matrix; 0: the matrix is small, look at it here
};

template <typename T> __device__ __forceinline__ uint32_t magnitude_bits(T x);           // as those of a float
template <> __device__ __forceinline__ uint32_t magnitude_bits<float>(float x) { return __float_as_uint(x) & 0x7fffffffu; }
template <> __device__ __forceinline__ uint32_t magnitude_bits<__nv_bfloat16>(__nv_bfloat16 x) {
  return ((uint32_t)__bfloat16_as_ushort(x) & 0x7fffu) << 16;
}
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t bits) { return bits < 0x7f800000u ? bits : 0u; }

// Eight values to eight e2m1 codes, the first in the low bits: to nearest, ties to even, magnitudes above 6 to 6.
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

// exponent byte of the power of two of an nvfp4 matrix whose largest magnitude has these bits: the smallest with
// largest <= 448 * 6 * 2^w (2688 = 1.3125 * 2^11), at least 2^-100 (so that a block's scale and its reciprocal stay ordinary
// numbers); 1 for a matrix of zeros
__device__ __forceinline__ int whole_exponent(uint32_t top) {
  if (top == 0u) return 127;
  const int e = (int)((top + 0x57ffffu) >> 23) - 11;
  return e > 27 ? e : 27;
}

// A block's scale byte and what its values are multiplied by.
struct BlockScale {
  float r, lo, s;         // mxfp4: value * r. nvfp4: the quotient value / s with r (+ lo) = 1 / s
  uint32_t byte;
};
// `whole` = 2^w, `unit` = 2^-w
template <int FMT, bool SHORT>
__device__ __forceinline__ BlockScale block_scale(uint32_t big, float whole, float unit) {
  BlockScale q;
  q.lo = q.s = 0.f;
  if (FMT == MXFP4) {
    // the smallest power of two with big <= 6 * 2^e = 1.5 * 2^(e + 2). (The usual rule 2^(floor(log2 big) - 2) clips whatever
    // lies above 6 of 8, up to a quarter of the block's largest value.)
    const int byte = (int)((big + 0x3fffffu) >> 23) - 2;
    q.byte = byte > 0 ? (uint32_t)byte : 0u;
    q.r = __uint_as_float((254u - q.byte) << 23);
    if (big >= 0x7f800000u) q.byte = 255u;                    // NaN: Inf and NaN have no place in a block
  } else {
    // big * 2^-w / 6 correctly rounded: the product with the rounded reciprocal, and one correction by its exact remainder
    // (Markstein 1990)
    const float x = __uint_as_float(big) * unit, sixth = 1.f / 6.f, t = x * sixth, a = fmaf(fmaf(-t, 6.f, x), sixth, t);
    q.byte = (uint32_t)__nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3);
    q.s = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)q.byte, __NV_E4M3))) * whole;
    if (SHORT) {
      // 1 / s in two parts, the first of 16 bits, the second from its exact remainder (for that an approximate 1 / s is enough)
      float r;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(q.s));
      if (!(q.s > 0.f)) r = 0.f;
      q.r = __uint_as_float(__float_as_uint(r) & 0xffffff00u);
      q.lo = fmaf(-q.r, q.s, 1.f) * r;
    } else {
      q.r = q.s > 0.f ? __frcp_rn(q.s) : 0.f;
    }
    // NaN; what is finite in such a block, the padding too, becomes zero (a factor made of NaN turned the padding's zeros into sixes)
    if (big >= 0x7f800000u) { q.byte = 0x7fu; q.r = q.lo = q.s = 0.f; }
  }
  return q;
}
// The quotient value / s correctly rounded, so that the ties between two codes, which values of few bits often hit, are ties.
// SHORT (values of 8 bits): value * r.hi is exact and value * r.lo brings the sum to 2^-39 of the quotient, far nearer than any
// quotient that is not a tie comes to one. Else the rounded product and one correction by its exact remainder (Markstein 1990).
// Two values at a time: one instruction multiplies both (8192 x 6400 bf16 to nvfp4 60.5 -> 58.3 us).
template <int FMT, bool SHORT>
__device__ __forceinline__ void scaled2(float x0, float x1, const BlockScale& q, float* v) {
  if (FMT == MXFP4) {
    v[0] = x0 * q.r;
    v[1] = x1 * q.r;
  } else if (SHORT) {
    asm("{\n\t.reg .b64 x, r, l, a;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 r, {%4, %4};\n\tmov.b64 l, {%5, %5};\n\t"
        "mul.rn.f32x2 a, x, r;\n\tfma.rn.f32x2 a, x, l, a;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(v[0]), "=f"(v[1]) : "f"(x0), "f"(x1), "f"(q.r), "f"(q.lo));
  } else {
    asm("{\n\t.reg .b64 x, r, n, a, e;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 r, {%4, %4};\n\tmov.b64 n, {%5, %5};\n\t"
        "mul.rn.f32x2 a, x, r;\n\tfma.rn.f32x2 e, a, n, x;\n\tfma.rn.f32x2 a, e, r, a;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(v[0]), "=f"(v[1]) : "f"(x0), "f"(x1), "f"(q.r), "f"(-q.s));
  }
}

// the larger magnitudes of two pairs of bf16 (signs mean nothing), NaN above all
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b) {
  asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  return a;
}
// the two bf16 of a word times a power of two, in fp32
__device__ __forceinline__ void widen(uint32_t w, uint16_t power, float& lo, float& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tfma.rn.f32.bf16 %0, l, %3, 0f00000000;\n\tfma.rn.f32.bf16 %1, h, %3, 0f00000000;\n\t}"
      : "=f"(lo), "=f"(hi) : "r"(w), "h"(power));
}

// Where a row of the tile starts in shared memory, in words: rows of 32 columns further on are shifted by 8 words, so that the
// column pass (four row blocks x eight columns a warp) meets no bank twice.
template <typename T> __device__ __forceinline__ int row_word(int r) { return r * (TILE * (int)sizeof(T) / 4) + 8 * (r >> 5); }
template <typename T> __host__ __device__ constexpr int tile_bytes() { return (TILE * TILE * (int)sizeof(T) / 4 + 32) * 4; }

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Reads 2 or 4 bytes a value and writes half a byte and 1/32 or 1/16 a direction: HBM leaves some fifteen instructions a value, which mxfp4
// stays below (8192 x 6400 bf16 in both directions 28 us, 5.8 TB/s) and nvfp4, about twenty, does not (39 us behind 18 of the search for
// the largest magnitude). The tile goes through shared memory once; both passes read it from there.
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(Q_THREADS) mx4_quantize_kernel(const QuantParams p) {
  constexpr int BLK = FMT == MXFP4 ? 32 : 16, SBYTES = TILE / BLK * TILE, ES = (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* const s_row = smem + tile_bytes<T>();
  uint8_t* const s_col = s_row + SBYTES;
  __shared__ uint32_t s_top[Q_THREADS / 32];
  uint32_t* const words = reinterpret_cast<uint32_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int bz = blockIdx.y;
  // (nvfp4: the last tiles first, since the search for the largest magnitude has just left them in L2: 8192 x 6400 in bf16 64 -> 60 us)
  const unsigned int tile = FMT == NVFP4 ? gridDim.x - 1u - blockIdx.x : blockIdx.x;
  const int tr = (int)(tile / (unsigned)p.tiles_c), tc = (int)(tile - (unsigned)tr * (unsigned)p.tiles_c);
  const int row0 = tr * TILE, col0 = tc * TILE;
  const T* const X = reinterpret_cast<const T*>(p.X) + (long long)bz * p.batch_stride;
  pdl_wait();
  if (VEC) {
    constexpr int PER = TILE * ES / 16;          // 16-byte pieces a row
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
    constexpr int ROWS = Q_THREADS / PER;        // rows a pass of the CTA covers
    const int r0 = tid / PER, c = (tid % PER) * (16 / ES);
    const uint32_t dst = base + 4 * row_word<T>(r0) + (tid % PER) * 16;
    const T* src = X + (long long)(row0 + r0) * p.ld + col0 + c;
    if (row0 + TILE <= p.rows && col0 + TILE <= p.cols) {
#pragma unroll
      for (int i = 0; i < TILE / ROWS; ++i, src += (long long)ROWS * p.ld) copy16(dst + 4 * row_word<T>(ROWS * i), src, 16u);
    } else {
#pragma unroll
      for (int i = 0; i < TILE / ROWS; ++i, src += (long long)ROWS * p.ld) {
        int left = row0 + r0 + ROWS * i < p.rows ? (p.cols - col0 - c) * ES : 0;
        left = left < 0 ? 0 : left > 16 ? 16 : left;
        copy16(dst + 4 * row_word<T>(ROWS * i), left ? src : X, (uint32_t)left);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  } else if (ES == 4) {
    // rows that start anywhere: value by value, all on their way at once
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
    const int r0 = tid / TILE, c = tid % TILE;
    const T* src = X + (long long)(row0 + r0) * p.ld + col0 + c;
#pragma unroll 8
    for (int i = 0; i < TILE * TILE / Q_THREADS; ++i, src += 2 * p.ld) {
      const int r = r0 + 2 * i;
      const bool on = row0 + r < p.rows && col0 + c < p.cols;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(base + 4 * (row_word<T>(r) + c)), "l"(on ? src : X), "r"(on ? 4u : 0u) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  } else {
    // rows that start anywhere, 2 bytes a value
    if (col0 > 0 && col0 + TILE + 4 <= p.cols && row0 + TILE <= p.rows) {
      // inside the matrix: a warp a row, in the aligned 8-byte pieces that cover it, shifted into place with the next lane's (1600 x 50257,
      // both directions, 82 -> 66 us; 43 where rows are aligned). Guards at each piece, for all tiles, took 84.
      constexpr int ROWS = 8;
#pragma unroll 1
      for (int r0 = warp; r0 < TILE; r0 += ROWS * (Q_THREADS / 32)) {
        uint64_t w[ROWS], end[ROWS];
        const T* row = X + (long long)(row0 + r0) * p.ld + col0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const uint64_t* const src = reinterpret_cast<const uint64_t*>(reinterpret_cast<uintptr_t>(row + i * (Q_THREADS / 32) * p.ld) & ~(uintptr_t)7);
          w[i] = src[lane];
          end[i] = src[TILE / 4];
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const int bits = (int)(reinterpret_cast<uintptr_t>(row + i * (Q_THREADS / 32) * p.ld) & 7u) * 8;
          uint64_t next = __shfl_down_sync(0xffffffffu, w[i], 1);
          if (lane == 31) next = end[i];
          *reinterpret_cast<uint64_t*>(words + row_word<T>(r0 + i * (Q_THREADS / 32)) + 2 * lane) = bits ? w[i] >> bits | next << (64 - bits) : w[i];
        }
      }
    } else {
#pragma unroll 16
      for (int i = 0; i < TILE * TILE / Q_THREADS; ++i) {
        const int u = tid + Q_THREADS * i, r = u / TILE, c = u % TILE;
        const bool on = row0 + r < p.rows && col0 + c < p.cols;
        const T x = on ? X[(long long)(row0 + r) * p.ld + col0 + c] : (T)0.f;
        reinterpret_cast<T*>(words + row_word<T>(r))[c] = x;
      }
    }
  }
  float whole = 1.f, unit = 1.f;
  if (FMT == NVFP4) {
    uint32_t top = 0;
    if (p.nper > 0) {
      for (int i = tid; i < p.nper; i += Q_THREADS) top = max(top, __float_as_uint(p.partial[(long long)bz * p.nper + i]));
    } else {
      constexpr int V = 16 / ES;
      int done = 0;
      if (VEC && (p.ld == p.cols || p.rows == 1)) {
        done = p.rows * p.cols / V * V;
#pragma unroll 4
        for (int u = tid; u < done / V; u += Q_THREADS) {
          const uint4 q = reinterpret_cast<const uint4*>(X)[u];
          const uint32_t x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (ES == 4) top = max(top, finite_or_zero(x[j] & 0x7fffffffu));
            else top = max(top, max(finite_or_zero((x[j] << 16) & 0x7fff0000u), finite_or_zero(x[j] & 0x7fff0000u)));
          }
        }
      }
#pragma unroll 4
      for (int u = done + tid; u < p.rows * p.cols; u += Q_THREADS) {
        const int r = u / p.cols;
        top = max(top, finite_or_zero(magnitude_bits(X[(long long)r * p.ld + (u - r * p.cols)])));
      }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s_top[warp] = top;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  if (FMT == NVFP4) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < Q_THREADS / 32; ++i) top = max(top, s_top[i]);
    const uint32_t e = (uint32_t)whole_exponent(top);
    whole = __uint_as_float(e << 23);
    unit = __uint_as_float((254u - e) << 23);
    if (blockIdx.x == 0 && tid == 0) {
      if (p.rscale) p.rscale[bz] = whole;
      if (p.cscale) p.cscale[bz] = whole;
    }
  }

  if (p.rc) {
    // A lane takes 32 values of a row, in four pieces of eight codes. Its first piece is number `rot`, so that the eight lanes of a
    // shared-memory access meet all banks (fp32: and the second half of a piece first in every other lane).
    const int width = mx4_width(p.cols), rot = (lane >> 1) & 3, odd = lane & 1;
    uint8_t* const out = p.rc + (long long)bz * p.rows * (width / 2);
#pragma unroll 1
    for (int i = 0; i < TILE * TILE / 32 / Q_THREADS; ++i) {
      const int u = tid + Q_THREADS * i, r = u >> 2, g = u & 3;
      const uint32_t* const src = words + row_word<T>(r) + g * (8 * ES);
      uint32_t w[8 * ES], big[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int piece = (k + rot) & 3;
        if (ES == 2) {
          const uint4 q = *reinterpret_cast<const uint4*>(src + 4 * piece);
          w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
          const uint32_t m = max_magnitudes(max_magnitudes(q.x, q.y), max_magnitudes(q.z, q.w)) & 0x7fff7fffu;
          big[k] = max(m << 16, m & 0xffff0000u);
        } else {
          uint32_t m = 0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 q = *reinterpret_cast<const uint4*>(src + 8 * piece + 4 * (h ^ odd));
            w[8 * k + 4 * h] = q.x; w[8 * k + 4 * h + 1] = q.y; w[8 * k + 4 * h + 2] = q.z; w[8 * k + 4 * h + 3] = q.w;
#pragma unroll
            for (int j = 0; j < 4; ++j) m = max(m, w[8 * k + 4 * h + j] & 0x7fffffffu);
          }
          big[k] = m;
        }
      }
      // blocks of 16: which pieces are the first block's depends on the lane (the pair that starts at piece 0 or 2, or one of each)
      BlockScale q[2];
      if (FMT == MXFP4) {
        q[0] = block_scale<FMT, ES == 2>(max(max(big[0], big[1]), max(big[2], big[3])), whole, unit);
        q[1] = q[0];
      } else {
        const uint32_t even = max(big[0], big[1]), mid = max(big[1], big[2]), last = max(big[2], big[3]), ends = max(big[3], big[0]);
        const uint32_t b0 = rot == 0 ? even : rot == 1 ? ends : rot == 2 ? last : mid, b1 = rot == 0 ? last : rot == 1 ? mid : rot == 2 ? even : ends;
        q[0] = block_scale<FMT, ES == 2>(b0, whole, unit);
        q[1] = block_scale<FMT, ES == 2>(b1, whole, unit);
      }
      uint32_t codes[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        BlockScale c = q[0];
        if (FMT == NVFP4) {
          const bool second = ((k + rot) & 2) != 0;
          c.r = second ? q[1].r : q[0].r; c.lo = second ? q[1].lo : q[0].lo; c.s = second ? q[1].s : q[0].s;
        }
        float v[8];
        if (ES == 2) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t x = w[4 * k + j];
            if (FMT == MXFP4) {
              widen(x, (uint16_t)(__float_as_uint(c.r) >> 16), v[2 * j], v[2 * j + 1]);
            } else {
              scaled2<FMT, true>(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u), c, v + 2 * j);
            }
          }
          codes[k] = e2m1x8(v);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j += 2) scaled2<FMT, false>(__uint_as_float(w[8 * k + j]), __uint_as_float(w[8 * k + j + 1]), c, v + j);
          const uint32_t x = e2m1x8(v);
          codes[k] = odd ? __byte_perm(x, x, 0x1032) : x;
        }
      }
      // the pieces back in their places
      if (rot & 1) { const uint32_t x = codes[3]; codes[3] = codes[2]; codes[2] = codes[1]; codes[1] = codes[0]; codes[0] = x; }
      if (rot & 2) { uint32_t x = codes[0]; codes[0] = codes[2]; codes[2] = x; x = codes[1]; codes[1] = codes[3]; codes[3] = x; }
      if (row0 + r < p.rows && col0 + 32 * g < width)
        *reinterpret_cast<uint4*>(out + (long long)(row0 + r) * (width / 2) + (col0 + 32 * g) / 2) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
      uint8_t* const sb = s_row + (r & 31) * 16 + (r >> 5) * 4;
      if (FMT == MXFP4) sb[g] = (uint8_t)q[0].byte;
      else *reinterpret_cast<uint16_t*>(sb + (g >> 1) * 512 + (g & 1) * 2) = (uint16_t)(q[0].byte | q[1].byte << 8);
    }
  }

  if (p.cc) {
    const int width = mx4_width(p.rows);         // codes a column
    uint8_t* const out = p.cc + (long long)bz * p.cols * (width / 2);
    const int rb = lane & 3;                     // rows 32 rb ..
    constexpr int COLS = ES == 2 ? 2 : 1;        // columns of a word
#pragma unroll 1
    for (int i = 0; i < 2 / COLS; ++i) {
      const int cw = (lane >> 2) + 8 * warp + 64 * i;
      uint32_t w[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) w[j] = words[row_word<T>(32 * rb) + j * (TILE * ES / 4) + cw];
      uint32_t big[32 / BLK];
#pragma unroll
      for (int h = 0; h < 32 / BLK; ++h) {
        uint32_t m = ES == 4 ? w[BLK * h] & 0x7fffffffu : w[BLK * h];
#pragma unroll
        for (int j = 1; j < BLK; ++j) m = ES == 4 ? max(m, w[BLK * h + j] & 0x7fffffffu) : max_magnitudes(m, w[BLK * h + j]);
        big[h] = m;
      }
#pragma unroll
      for (int k = 0; k < COLS; ++k) {
        const int c = cw * COLS + k;
        uint32_t codes[4];
#pragma unroll
        for (int h = 0; h < 32 / BLK; ++h) {
          const uint32_t m = ES == 4 ? big[h] : (k == 0 ? big[h] << 16 : big[h]) & 0x7fff0000u;
          const BlockScale q = block_scale<FMT, ES == 2>(m, whole, unit);
#pragma unroll
          for (int o = 0; o < BLK / 8; ++o) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t x = w[BLK * h + 8 * o + j];
              if (ES == 2 && FMT == MXFP4) {
                float lo, hi;
                widen(x, (uint16_t)(__float_as_uint(q.r) >> 16), lo, hi);
                v[j] = k == 0 ? lo : hi;
              } else {
                v[j] = __uint_as_float(ES == 4 ? x : k == 0 ? x << 16 : x & 0xffff0000u);
                if (j & 1) scaled2<FMT, ES == 2>(v[j - 1], v[j], q, v + j - 1);
              }
            }
            codes[(BLK / 8) * h + o] = e2m1x8(v);
          }
          const int blk = rb * (32 / BLK) + h;
          s_col[(blk >> 2) * 512 + (c & 31) * 16 + (c >> 5) * 4 + (blk & 3)] = (uint8_t)q.byte;
        }
        if (col0 + c < p.cols && row0 + 32 * rb < width)
          *reinterpret_cast<uint4*>(out + (long long)(col0 + c) * (width / 2) + (row0 + 32 * rb) / 2) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
      }
    }
  }

  __syncthreads();
  // the tiles of scales, whole: rows and blocks that do not exist have zeros
  constexpr int NT = SBYTES / 512;
  if (p.rc) {
    const int kt = mx4_scale_tiles(p.cols, FMT), first = tc * NT;
    if (tid * 4 < min(NT, kt - first) * 512)
      reinterpret_cast<uint32_t*>(p.rs + (((long long)bz * mx4_row_tiles(p.rows) + tr) * kt + first) * 512)[tid] = reinterpret_cast<uint32_t*>(s_row)[tid];
  }
  if (p.cc) {
    const int kt = mx4_scale_tiles(p.rows, FMT), first = tr * NT;
    if (tid * 4 < min(NT, kt - first) * 512)
      reinterpret_cast<uint32_t*>(p.cs + (((long long)bz * mx4_row_tiles(p.cols) + tc) * kt + first) * 512)[tid] = reinterpret_cast<uint32_t*>(s_col)[tid];
  }
}

// Largest finite magnitude of a part of each matrix (nvfp4): its 16-byte pieces are dealt to the CTAs of a matrix. Bound by HBM
// (or L2): four pieces of a thread are on their way at a time. A thread that has met Inf or NaN looks again without them.
template <typename T, bool VEC>
__global__ void __launch_bounds__(Q_THREADS) mx4_amax_kernel(const void* Xv, long long ld, long long batch_stride, int rows, int cols, float* partial) {
  __shared__ uint32_t s_top[Q_THREADS / 32];
  pdl_wait();
  const T* const X = reinterpret_cast<const T*>(Xv) + (long long)blockIdx.y * batch_stride;
  constexpr int V = 16 / (int)sizeof(T);
  uint32_t top = 0;
  for (int pass = 0; pass < 2; ++pass) {
    top = 0;
    const bool fine = pass == 1;
    auto take = [&](const uint4& q) {
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 4) top = max(top, fine ? finite_or_zero(w[j] & 0x7fffffffu) : w[j] & 0x7fffffffu);
        else if (!fine) top = __vmaxu2(top, w[j] & 0x7fff7fffu);
        else top = max(top, max(finite_or_zero((w[j] << 16) & 0x7fff0000u), finite_or_zero(w[j] & 0x7fff0000u)));
      }
    };
    auto one = [&](T x) {
      const uint32_t m = fine ? finite_or_zero(magnitude_bits(x)) : magnitude_bits(x);
      if (sizeof(T) == 2 && !fine) top = __vmaxu2(top, m); else top = max(top, m);
    };
    const long long step = (long long)gridDim.x * Q_THREADS, u0 = (long long)blockIdx.x * Q_THREADS + threadIdx.x;
    if (ld == cols || rows == 1) {
      // one run of values: whole 32-byte pieces (16-byte ones: 8192 x 1600 quantised in 16.9 us, not 16.0), and those before and after them
      constexpr int V2 = 2 * V;
      const long long n = (long long)rows * cols;
      const long long skip = (long long)((32u - (uint32_t)(reinterpret_cast<uintptr_t>(X) & 31u)) & 31u) / (long long)sizeof(T), head = skip < n ? skip : n;
      const long long nv = (n - head) / V2, tail = head + nv * V2;
      const T* const P = X + head;
      long long u = u0;
      auto load = [&](long long at, uint4& a, uint4& b) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(P + at * V2));
      };
      for (; u + 3 * step < nv; u += 4 * step) {
        uint4 q[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) load(u + k * step, q[2 * k], q[2 * k + 1]);
#pragma unroll
        for (int k = 0; k < 8; ++k) take(q[k]);
      }
      for (; u < nv; u += step) {
        uint4 x, y;
        load(u, x, y);
        take(x); take(y);
      }
      if (u0 < head) one(X[u0]);
      if (u0 < n - tail) one(X[tail + u0]);
    } else {
      const long long per = VEC ? (cols + V - 1) / V : cols;
      // (row and column are carried along: the step is a fixed number of rows and columns)
      long long r = u0 / per, c = u0 - r * per;
      const long long dr = step / per, dc = step - dr * per;
      for (; r < rows;) {
        if (VEC && c * V + V <= cols) {
          take(*reinterpret_cast<const uint4*>(X + r * ld + c * V));
        } else {
          const int n = VEC ? V : 1;
          for (int j = 0; j < n; ++j)
            if (c * n + j < cols) one(X[r * ld + c * n + j]);
        }
        r += dr; c += dc;
        if (c >= per) { c -= per; ++r; }
      }
    }
    if (sizeof(T) == 2 && !fine) top = max(top << 16, top & 0xffff0000u);
    if (top < 0x7f800000u) break;
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < Q_THREADS / 32; ++i) top = max(top, s_top[i]);
    partial[(long long)blockIdx.y * gridDim.x + blockIdx.x] = __uint_as_float(top);
  }
}

__device__ __forceinline__ float2 e2m1x2(uint32_t two) {
  uint32_t h;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(two));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

constexpr int SEG = 64;                    // 32-byte pieces of a row of the result that a warp takes
// A warp 2 KB of a row of the result (256 values where the rows do not start on 16-byte boundaries), all its loads on their way at once. Bound by HBM:
// half a byte in, 2 or 4 out.
template <int FMT, typename O>
__global__ void __launch_bounds__(Q_THREADS) mx4_dequantize_kernel(Mx4View a, int b, int rows, int cols, O* out, int vec) {
  constexpr int BLK = FMT == MXFP4 ? 32 : 16;
  pdl_wait();
  const long long id = (long long)blockIdx.x * (Q_THREADS / 32) + (threadIdx.x >> 5);
  if (id >= (long long)b * rows) return;
  const int lane = threadIdx.x & 31, bz = (int)(id / rows), r = (int)(id - (long long)bz * rows);
  const int width = mx4_width(cols), kt = mx4_scale_tiles(cols, FMT);
  const uint32_t* const codes = reinterpret_cast<const uint32_t*>(a.codes + id * (width / 2));
  const uint8_t* const sc = a.scales + ((long long)bz * mx4_row_tiles(rows) + (r >> 7)) * kt * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4;
  const float whole = FMT == NVFP4 ? a.scale[bz] : 1.f;
  O* const dst = out + id * cols;
  auto scale_of = [&](int blk) {
    const uint32_t byte = sc[(long long)(blk >> 2) * 512 + (blk & 3)];
    return FMT == MXFP4 ? scale_value<FMT>(byte) : scale_value<FMT>(byte) * whole;
  };
  if (!vec) {
    // rows that do not start on 16-byte boundaries: a value a lane, side by side
    const int first = 256 * blockIdx.y, end = min(cols, first + 256);
#pragma unroll 8
    for (int c = first + lane; c < end; c += 32) {
      const float2 f = e2m1x2(codes[c >> 3] >> (4 * (c & 6)));
      dst[c] = (O)((c & 1 ? f.y : f.x) * scale_of(c / BLK));
    }
    return;
  }
  // a lane writes 32 bytes, a whole sector, in one store where rows start on such boundaries (8192 x 6400 to bf16 32 -> 25 us, to fp32
  // 58 -> 42, against 16 bytes at a time; one or four pieces a lane in place of two gain nothing)
  constexpr int PER = 32 / (int)sizeof(O);
  const int end = min((cols + PER - 1) / PER, SEG * ((int)blockIdx.y + 1));
#pragma unroll 2
  for (int u = SEG * blockIdx.y + lane; u < end; u += 32) {
    uint32_t q[PER / 8];
    if (PER == 16) { const uint2 two = reinterpret_cast<const uint2*>(codes)[u]; q[0] = two.x; q[PER / 8 - 1] = two.y; } else { q[0] = codes[u]; }
    const float s = scale_of(u * PER / BLK);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < PER / 2; ++j) {
      const float2 f = e2m1x2(q[j / 4] >> (8 * (j & 3)));
      if (PER == 16) { w[j & 7] = pack16x2(f.x * s, f.y * s, false); }
      else { w[(2 * j) & 7] = __float_as_uint(f.x * s); w[(2 * j + 1) & 7] = __float_as_uint(f.y * s); }
    }
    O* const d = dst + (long long)PER * u;
    if (vec == 2) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(d), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
      reinterpret_cast<uint4*>(d)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      if (PER == 8 || 16 * u + 8 < cols) reinterpret_cast<uint4*>(d)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}

template <typename T, int FMT>
constexpr int quantize_smem() { return tile_bytes<T>() + 2 * (TILE / (FMT == MXFP4 ? 32 : 16) * TILE); }

template <typename T, int FMT>
cudaError_t quantize_launch(const QuantParams& p, bool vec, cudaStream_t st) {
  const dim3 grid((unsigned)p.tiles_c * (unsigned)((p.rows + TILE - 1) / TILE), (unsigned)p.b);
  return vec ? launch_kernel(mx4_quantize_kernel<T, FMT, true>, grid, dim3(Q_THREADS), quantize_smem<T, FMT>(), st, p)
             : launch_kernel(mx4_quantize_kernel<T, FMT, false>, grid, dim3(Q_THREADS), quantize_smem<T, FMT>(), st, p);
}
template <typename T>
cudaError_t amax_launch(const void* X, long long ld, long long batch_stride, int rows, int cols, int b, int nper, float* partial, bool vec, cudaStream_t st) {
  const dim3 grid((unsigned)nper, (unsigned)b);
  return vec ? launch_kernel(mx4_amax_kernel<T, true>, grid, dim3(Q_THREADS), 0, st, X, ld, batch_stride, rows, cols, partial)
             : launch_kernel(mx4_amax_kernel<T, false>, grid, dim3(Q_THREADS), 0, st, X, ld, batch_stride, rows, cols, partial);
}
template <typename T, int FMT>
cudaError_t quantize_limit() {
  cudaError_t e = cudaFuncSetAttribute(mx4_quantize_kernel<T, FMT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, quantize_smem<T, FMT>());
  return e != cudaSuccess ? e : cudaFuncSetAttribute(mx4_quantize_kernel<T, FMT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, quantize_smem<T, FMT>());
}

int partials_of(int b) { return b >= MAX_PARTIALS ? 1 : MAX_PARTIALS / b; }

bool matrix_ok(const defl_mx4* m, int fmt) {
  return m->codes && m->scales && on(m->codes, 16) && on(m->scales, 16) && (fmt == DEFL_MXFP4 || (m->scale && on(m->scale, 4)));
}

}  // namespace

cudaError_t mx4_quantize_prepare() {
  cudaError_t e;
  if ((e = quantize_limit<float, MXFP4>()) != cudaSuccess) return e;
  if ((e = quantize_limit<float, NVFP4>()) != cudaSuccess) return e;
  if ((e = quantize_limit<__nv_bfloat16, MXFP4>()) != cudaSuccess) return e;
  return quantize_limit<__nv_bfloat16, NVFP4>();
}

}  // namespace defl

using namespace defl;

extern "C" {

size_t defl_mx4_codes_bytes(int b, int rows, int cols) {
  return b <= 0 || rows <= 0 || cols <= 0 ? 0 : (size_t)b * rows * (mx4_width(cols) / 2);
}
size_t defl_mx4_scales_bytes(int b, int rows, int cols, int fmt) {
  if (b <= 0 || rows <= 0 || cols <= 0 || (fmt != DEFL_MXFP4 && fmt != DEFL_NVFP4)) return 0;
  return (size_t)b * mx4_row_tiles(rows) * mx4_scale_tiles(cols, fmt) * 512;
}
size_t defl_mx4_work_bytes(int b) { return b <= 0 ? 0 : (size_t)b * partials_of(b) * sizeof(float); }

int defl_mx4_quantize(defl_ctx* c, const void* X, int dtype, int b, int rows, int cols, int64_t ld, int64_t batch_stride, int fmt,
                      const defl_mx4* by_rows, const defl_mx4* by_cols, void* work) {
  if (!c || !X || b <= 0 || rows <= 0 || cols <= 0 || ld < cols || (b > 1 && batch_stride < 0)) return DEFL_ERR_ARG;
  if ((dtype != DEFL_BF16 && dtype != DEFL_F32) || (fmt != DEFL_MXFP4 && fmt != DEFL_NVFP4)) return DEFL_ERR_ARG;
  if ((!by_rows && !by_cols) || (by_rows && !matrix_ok(by_rows, fmt)) || (by_cols && !matrix_ok(by_cols, fmt))) return DEFL_ERR_ARG;
  const unsigned es = (unsigned)dtype_size(dtype);
  if (!on(X, es)) return DEFL_ERR_ARG;
  if (rows > DEFL_MX4_MAX_SIDE || cols > DEFL_MX4_MAX_SIDE || b > 65535) return DEFL_ERR_RANK;
  // nvfp4: up to this size every CTA finds the largest magnitude by itself, which saves a launch. us that way and with the launch, blocks along the
  // rows: bf16 8192 values 2.9 5.0, 32000 4.2 4.9, 64000 5.7 4.9, 131072 8.1 4.3; fp32 8192 3.7 5.4, 32000 5.6 5.5, 64000 7.8 5.5
  const bool scan = (long long)rows * cols <= DEFL_MX4_SCAN_MOST;
  static_assert(DEFL_MX4_SCAN_MOST <= 0x7fffffff, "the kernel counts these values in 32 bits");
  if (fmt == DEFL_NVFP4 && !scan && (!work || !on(work, 4))) return DEFL_ERR_ARG;
  DeviceScope scope(c->device);
  c->err[0] = 0;
  QuantParams p = {};
  p.X = X; p.ld = ld; p.batch_stride = batch_stride; p.b = b; p.rows = rows; p.cols = cols;
  p.tiles_c = (cols + TILE - 1) / TILE;
  if ((long long)p.tiles_c * ((rows + TILE - 1) / TILE) > 0x7fffffffll) return DEFL_ERR_RANK;
  if (by_rows) { p.rc = (uint8_t*)by_rows->codes; p.rs = (uint8_t*)by_rows->scales; p.rscale = fmt == DEFL_NVFP4 ? by_rows->scale : nullptr; }
  if (by_cols) { p.cc = (uint8_t*)by_cols->codes; p.cs = (uint8_t*)by_cols->scales; p.cscale = fmt == DEFL_NVFP4 ? by_cols->scale : nullptr; }
  const bool vec = on(X, 16) && (ld * es) % 16 == 0 && (b == 1 || (batch_stride * es) % 16 == 0);
  if (fmt == DEFL_NVFP4 && !scan) {
    p.nper = partials_of(b);
    p.partial = reinterpret_cast<const float*>(work);
    const cudaError_t e = dtype == DEFL_BF16 ? amax_launch<__nv_bfloat16>(X, ld, batch_stride, rows, cols, b, p.nper, (float*)work, vec, c->stream)
                                             : amax_launch<float>(X, ld, batch_stride, rows, cols, b, p.nper, (float*)work, vec, c->stream);
    ++c->launches;
    if (ctx_fail(c, e, "mx4 largest magnitude")) return DEFL_ERR_CUDA;
  }
  cudaError_t e;
  if (dtype == DEFL_BF16) e = fmt == DEFL_MXFP4 ? quantize_launch<__nv_bfloat16, MXFP4>(p, vec, c->stream) : quantize_launch<__nv_bfloat16, NVFP4>(p, vec, c->stream);
  else e = fmt == DEFL_MXFP4 ? quantize_launch<float, MXFP4>(p, vec, c->stream) : quantize_launch<float, NVFP4>(p, vec, c->stream);
  ++c->launches;
  if (ctx_fail(c, e, "mx4 quantize")) return DEFL_ERR_CUDA;
  return DEFL_OK;
}

int defl_mx4_dequantize(defl_ctx* c, const defl_mx4* a, int b, int rows, int cols, int fmt, void* out, int dtype) {
  if (!c || !a || !out || b <= 0 || rows <= 0 || cols <= 0) return DEFL_ERR_ARG;
  if ((dtype != DEFL_BF16 && dtype != DEFL_F32) || (fmt != DEFL_MXFP4 && fmt != DEFL_NVFP4) || !matrix_ok(a, fmt)) return DEFL_ERR_ARG;
  if (!on(out, (unsigned)dtype_size(dtype))) return DEFL_ERR_ARG;
  if (rows > DEFL_MX4_MAX_SIDE || cols > DEFL_MX4_MAX_SIDE) return DEFL_ERR_RANK;
  const long long grid = ((long long)b * rows + Q_THREADS / 32 - 1) / (Q_THREADS / 32);
  if (grid > 0x7fffffffll) return DEFL_ERR_RANK;
  DeviceScope scope(c->device);
  c->err[0] = 0;
  const Mx4View v = {(const uint8_t*)a->codes, (const uint8_t*)a->scales, a->scale};
  // 0: value by value, 1: 16-byte stores, 2: 32-byte stores
  const int es = (int)dtype_size(dtype), vec = on(out, 32) && (long long)cols * es % 32 == 0 ? 2 : on(out, 16) && cols % 8 == 0 ? 1 : 0;
  const int seg = vec ? 32 / es * SEG : 256;
  const dim3 g((unsigned)grid, (unsigned)((cols + seg - 1) / seg)), t(Q_THREADS);
  cudaError_t e;
  if (dtype == DEFL_BF16) {
    __nv_bfloat16* o = (__nv_bfloat16*)out;
    e = fmt == DEFL_MXFP4 ? launch_kernel(mx4_dequantize_kernel<MXFP4, __nv_bfloat16>, g, t, 0, c->stream, v, b, rows, cols, o, vec)
                          : launch_kernel(mx4_dequantize_kernel<NVFP4, __nv_bfloat16>, g, t, 0, c->stream, v, b, rows, cols, o, vec);
  } else {
    float* o = (float*)out;
    e = fmt == DEFL_MXFP4 ? launch_kernel(mx4_dequantize_kernel<MXFP4, float>, g, t, 0, c->stream, v, b, rows, cols, o, vec)
                          : launch_kernel(mx4_dequantize_kernel<NVFP4, float>, g, t, 0, c->stream, v, b, rows, cols, o, vec);
  }
  ++c->launches;
  if (ctx_fail(c, e, "mx4 dequantize")) return DEFL_ERR_CUDA;
  return DEFL_OK;
}

size_t defl_mx4_gemm_work_bytes(defl_ctx* c, int b, int M, int N, int K, int out_dtype) {
  if (!c || b <= 0 || M <= 0 || N <= 0 || K <= 0 || b > 65535 || M > DEFL_MX4_MAX_SIDE || N > DEFL_MX4_MAX_SIDE || K > DEFL_MX4_MAX_SIDE) return 0;
  return mx4_gemm_split(b, M, N, K, out_dtype, c->num_sms).work_bytes;
}

int defl_mx4_gemm(defl_ctx* c, const defl_mx4* A, const defl_mx4* B, int b, int M, int N, int K, int b_shared, int fmt, float alpha, void* D, int64_t ldd,
                  int64_t batch_stride, int out_dtype, void* work) {
  if (!c || !A || !B || !D || b <= 0 || M <= 0 || N <= 0 || K <= 0 || ldd < N) return DEFL_ERR_ARG;
  if (b > 1 && batch_stride < (int64_t)(M - 1) * ldd + N) return DEFL_ERR_ARG;
  if ((fmt != DEFL_MXFP4 && fmt != DEFL_NVFP4) || (out_dtype != DEFL_BF16 && out_dtype != DEFL_F32)) return DEFL_ERR_ARG;
  if (!matrix_ok(A, fmt) || !matrix_ok(B, fmt) || !on(D, (unsigned)dtype_size(out_dtype))) return DEFL_ERR_ARG;
  if (work && !on(work, 16)) return DEFL_ERR_ARG;
  if (M > DEFL_MX4_MAX_SIDE || N > DEFL_MX4_MAX_SIDE || K > DEFL_MX4_MAX_SIDE || b > 65535) return DEFL_ERR_RANK;
  DeviceScope scope(c->device);
  c->err[0] = 0;
  Mx4Gemm g;
  g.A = {(const uint8_t*)A->codes, (const uint8_t*)A->scales, A->scale};
  g.B = {(const uint8_t*)B->codes, (const uint8_t*)B->scales, B->scale};
  g.b = b; g.M = M; g.N = N; g.K = K; g.fmt = fmt; g.b_shared = b_shared != 0;
  g.D = D; g.ldd = ldd; g.batch_d = batch_stride; g.out_dtype = out_dtype; g.alpha = alpha; g.work = work;
  const unsigned long long wait_ns = (unsigned long long)(c->tc_knobs.wait_ms > 0 ? c->tc_knobs.wait_ms : 2000) * 1000000ull;
  if (ctx_fail(c, mx4_gemm_launch(g, c->stream, c->wait_status + WAIT_MX4, c->num_sms, wait_ns, c->knobs.mx4_hold != 0, &c->launches), "mx4 gemm")) return DEFL_ERR_CUDA;
  return DEFL_OK;
}

}  // extern "C"
