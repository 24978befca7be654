// Products of microscaled 4-bit matrices for sm_100a: D = alpha A B^T.
//
// mx4_tc_kernel, the tensor cores' form: persistent and warp-specialised like the 16-bit engine (gemm_tc.cu): warp 0 copies
// operand tiles and their scales into a ring of shared-memory stages, warps 10..13 move the scales on to tensor memory, warp 1
// issues the products, warps 2..9 read the accumulators out. A stage covers 256 values of K (128 bytes a row, 128-byte swizzle).
// The scales travel as they lie in memory, in tiles of 128 rows x 4 blocks (512 bytes); each of the four warps writes them to its
// own lane quarter (every quarter holds all 128 rows, 32 a column); a product takes 64 values of K and reads its scales there.
//   M > 128   a pair of CTAs per 256 x BN tile (cta_group::2): each stages 128 rows of A, half of the B columns, the scales of its own
//             rows and those of all columns (each multiplies its rows with all of them)
//   M <= 128  one CTA, 128 x BN
// Tensor memory: 512 columns = two accumulators and four sets of scales (24 columns each, nvfp4 48). Two accumulators of 256 columns
// leave no room for that, so they overlap (by 96 and 192 columns); the read-out takes those first and says so, and the next tile's
// products wait for that much only. (Copies run on meanwhile, and products are twice as fast as copies.)
// What bounds it. 8192 x 8192 x 8192: what arrives from L2 at all SMs together, 11 TB/s (5500 to 6000 bytes a cycle at 1.9 GHz), 64 + 6 KB (nvfp4
// + 12) for a 256 x 256 tile and 256 values of K: 206 us in mxfp4, 5.3 PFLOP/s, 226 in nvfp4. 8192 x 6400 x 1600 to bf16, 47 and 52 us, moves
// 530 and 556 MB through L2, 105 of them D: a CTA fetches its 128 rows of A again for each of 25 columns of tiles, half of what it reads. 8192 x
// 1600 x 6400 and 6400 x 1600 x 8192, 47 to 49 and 45 to 47: the last wave (3.03 and 2.36 waves of 256-wide tiles over 74 pairs, taken as four of
// 192 and as three). In nvfp4 the tensor pipe is busy 34, 36 and 37 % of these three, L2's slices 37, 32 and 29 %.
//
// mx4_row_kernel, for up to eight rows of A (by_rows below): the weights are read once at memory speed, each code becomes two bytes by table
// lookup (prmt), four products at a time are integer dot products (dp4a), a block's sum meets its scales in fp32.
#include "ctx.cuh"
#include "mx4.cuh"
#include "tc_ptx.cuh"
#include <cuda_fp8.h>
#include <cudaTypedefs.h>
#include <mutex>

namespace defl {

namespace {

constexpr int KB_ELEMENTS = 256, KB_BYTES = 128;
constexpr int TC_THREADS = 480, TC_EPI_WARPS = 8, SF_WARP = 10;
constexpr int MAX_ST = 8;
constexpr int STG_BYTES = 4096;                    // 32 rows x 128 bytes
constexpr uint32_t SMEM_MOST = 227 * 1024;

// Tensor memory: SF_SETS sets of scales at the end, a stage each: A's four columns a tile, then those of up to two row tiles of B.
constexpr int SF_SETS = 4;
__host__ __device__ constexpr int scale_ring(int fmt) { return fmt == MXFP4 ? 8 : 5; }      // slots in shared memory
__host__ __device__ constexpr uint32_t scale_set(int fmt) { return fmt == MXFP4 ? 24u : 48u; }
__host__ __device__ constexpr uint32_t scale_column(int fmt) { return 512u - SF_SETS * scale_set(fmt); }

struct TcParams4 {
  CUtensorMap tmA, tmB, tmD;
  const uint8_t* sa; const uint8_t* sb; int rt_a, rt_b, kt;      // tiles of scales: row tiles, tiles a row tile
  int M, N, batch, BN, b_shared;
  int tiles_m, tiles_n;
  int total_tiles;
  int kblocks, ksteps_last;                        // stages of K, and products of 64 values in the last of them
  int splits, kper;                                // parts of K that are tiles of their own, stages each; D is then [splits, batch, M, N]
  int stages, sets, overlap;
  uint32_t a_bytes, b_bytes, stage_bytes;
  uint32_t idesc;
  int out_f32, store_tma;
  void* D; long long ldd, batch_d;
  float alpha; const float* scale_a; const float* scale_b;
  int* status; unsigned long long wait_ns;
  int hold;                                        // test hook: no codes are announced or copied
};

// alpha and the matrices' scales in one factor, and `pre`, 1 except where that factor leaves the middle of fp32's range: two matrices of values
// near 1e25 have 2^150 between them, and a sum of zero times that is zero. (A sum that is not zero is between 2^-20 and 2^46 in magnitude, so
// that a factor cut at fp32's largest number still makes it infinite.)
__device__ __forceinline__ float output_factor(float alpha, float scale_a, float scale_b, float& pre) {
  const float both = scale_a * scale_b, f = alpha * both;
  pre = 1.f;
  if (fabsf(both) > 0x1p-100f && fabsf(both) < 0x1p100f && (alpha == 0.f || (fabsf(f) > 0x1p-100f && fabsf(f) < 0x1p100f))) return f;
  const double exact = (double)alpha * (double)scale_a * (double)scale_b, size = fabs(exact);
  if (!(size < 1e300)) return (float)exact;          // a scale or alpha that is not finite
  pre = size > 1.0 ? 0x1p64f : 0x1p-64f;
  const double rest = exact / (double)pre;
  return (float)(rest > 3.4028234663852886e38 ? 3.4028234663852886e38 : rest < -3.4028234663852886e38 ? -3.4028234663852886e38 : rest);
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
      "%28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

// Descriptors are put together from their halves; only the address in the low one changes.
constexpr uint32_t OPERAND_HI = (1024u >> 4) | 1u << 14 | 2u << 29;      // groups of eight rows 1024 bytes apart, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr) { return (saddr >> 4) | 1u << 16; }

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

template <int FMT, int PAIR>
__device__ __forceinline__ void umma4(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define DEFL_MX4_MMA(GROUP, KIND)                                                                                    \
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %7, 0;\n\t"                                    \
               "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"                                                    \
               "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a, b, %4, [%5], [%6], p;\n\t}"                 \
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(OPERAND_HI), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
  if (FMT == MXFP4) {
    if (PAIR) DEFL_MX4_MMA("2", "mxf4.block_scale.scale_vec::2X"); else DEFL_MX4_MMA("1", "mxf4.block_scale.scale_vec::2X");
  } else {
    if (PAIR) DEFL_MX4_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X"); else DEFL_MX4_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X");
  }
#undef DEFL_MX4_MMA
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(tm), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

__device__ __forceinline__ uint32_t ld_word(uint32_t saddr) {
  uint32_t w;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(saddr));
  return w;
}
// element e of a staged row (its 16-byte pieces exchanged by `key`) to the row's place in memory
__device__ __forceinline__ void copy_element(uint8_t* d, uint32_t src, uint32_t key, int e, int es) {
  const uint32_t at = (uint32_t)(e * es), w = ld_word(src + ((at >> 4 ^ key) << 4) + (at & 12u));
  if (es == 4) *reinterpret_cast<uint32_t*>(d + at) = w;
  else *reinterpret_cast<uint16_t*>(d + at) = (uint16_t)(at & 2u ? w >> 16 : w);
}

struct Tile4 { int bz, tm, tn, n_eff, ks, k0, k1; };      // k0 .. k1: the stages of this part of K
template <int PAIR>
__device__ __forceinline__ Tile4 tile_of(const TcParams4& p, int tile) {
  Tile4 t;
  const int per = p.tiles_m * p.tiles_n;
  const int z = tile / per, i = tile - z * per;
  t.ks = p.splits > 1 ? z / p.batch : 0;
  t.bz = z - t.ks * p.batch;
  t.k0 = t.ks * p.kper;
  t.k1 = min(t.k0 + p.kper, p.kblocks);
  t.tn = i / p.tiles_m;                            // tiles of one column of tiles follow one another: they share B
  t.tm = i - t.tn * p.tiles_m;
  const int left = p.N - t.tn * p.BN, q = PAIR ? 31 : 15;
  t.n_eff = min(p.BN, (left + q) & ~q);
  return t;
}

// NSB: 128-row tiles of scales that the B columns of a tile reach into
template <int FMT, int PAIR, int NSB>
__global__ void __launch_bounds__(TC_THREADS, 1) mx4_tc_kernel(const __grid_constant__ TcParams4 p) {
  constexpr int ATOMS = FMT == MXFP4 ? 2 : 4;      // tiles of scales a row tile and stage
  constexpr uint32_t SF_SET = scale_set(FMT);
  constexpr uint32_t SF_COL = scale_column(FMT);
  constexpr int SF_RING = scale_ring(FMT);
  const uint32_t acc1 = (uint32_t)(p.BN - p.overlap);
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[MAX_ST], empty_bar[MAX_ST], land_bar[SF_RING], slot_empty_bar[SF_RING], acc_full_bar[2], acc_empty_bar[2], ovl_bar;
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int tile0 = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, tile_step = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;
  constexpr int TILE_M = PAIR ? 256 : 128;

  if (warp == 2 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.tmA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.tmB) : "memory");
  }
  if (threadIdx.x == 0) {
    abort_flag = 0;
    // (a stage is full when its codes are here and four warps, of each CTA, have its scales in tensor memory)
    for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&full_bar[s]), 1 + (PAIR ? 2 : 1) * 4); mbar_init(smem_u32(&empty_bar[s]), 1); }
    for (int s = 0; s < SF_RING; ++s) { mbar_init(smem_u32(&land_bar[s]), 1); mbar_init(smem_u32(&slot_empty_bar[s]), 4); }
    for (int a = 0; a < 2; ++a) {
      mbar_init(smem_u32(&acc_full_bar[a]), 1);
      mbar_init(smem_u32(&acc_empty_bar[a]), (PAIR ? 2 : 1) * TC_EPI_WARPS);
    }
    mbar_init(smem_u32(&ovl_bar), (PAIR ? 2 : 1) * TC_EPI_WARPS);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) { tmem_alloc_pair(smem_u32(&tmem_base_slot), 512); tmem_relinquish_pair(); }
    else { tmem_alloc(smem_u32(&tmem_base_slot), 512); tmem_relinquish(); }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_slot;
  pdl_launch();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies of the codes: A by lane 0, B by lane 1. Those of a pair
    // count on the leader's barrier, where the products wait for them.
    const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
    const uint32_t full0_sig = PAIR ? map_to_cta(full0, 0) : full0;
    const uint32_t tx = (PAIR ? 2u : 1u) * (p.a_bytes + p.b_bytes);
    const CUtensorMap* tm = lane == 0 ? &p.tmA : &p.tmB;
    const uint32_t off = lane == 0 ? 0u : p.a_bytes;
    uint32_t stage = 0, phase = 0;
    bool live = !p.hold;
    pdl_wait();
    for (int tile = tile0; tile < p.total_tiles && live; tile += tile_step) {
      const Tile4 t = tile_of<PAIR>(p, tile);
      const int n0 = t.tn * p.BN, m0 = t.tm * TILE_M + (int)rank * 128;
      const int bz_b = p.b_shared ? 0 : t.bz;
      const int c1 = lane == 0 ? m0 : n0 + (PAIR ? (int)rank * (t.n_eff >> 1) : 0), c2 = lane == 0 ? t.bz : bz_b;
      for (int kb = t.k0; kb < t.k1; ++kb) {
        int ok = 1;
        if (lane == 0) ok = mbar_wait(empty0 + 8u * stage, phase ^ 1u, &abort_flag, p.status, p.wait_ns) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) { live = false; break; }
        if (lane == 0 && rank == 0) mbar_expect_tx(full0 + 8u * stage, tx);
        if (lane < 2) {
          const uint32_t dst = smem_base + stage * p.stage_bytes + off;
          if (PAIR) tma_load_3d_pair(dst, tm, full0_sig + 8u * stage, kb * KB_BYTES, c1, c2);
          else tma_load_3d(dst, tm, full0 + 8u * stage, kb * KB_BYTES, c1, c2);
        }
        __syncwarp();
        if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    if (lane == 0 && rank == 0) {
      const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
      const uint32_t sf_col = tmem_base + SF_COL, b_off = p.a_bytes >> 4;
      uint32_t stage = 0, phase = 0, set = 0, ready = 0;
      pdl_wait();
      for (int tile = tile0, it = 0; tile < p.total_tiles; tile += tile_step, ++it) {
        const Tile4 t = tile_of<PAIR>(p, tile);
        const uint32_t acc = (uint32_t)it & 1u, use = ((uint32_t)it >> 1) & 1u;
        if (!mbar_wait(smem_u32(&acc_empty_bar[acc]), use ^ 1u, &abort_flag, p.status, p.wait_ns)) break;
        if (p.overlap && it > 0 && !mbar_wait(smem_u32(&ovl_bar), (uint32_t)(it - 1) & 1u, &abort_flag, p.status, p.wait_ns)) break;
        tc_fence_after();
        const uint32_t d = tmem_base + (acc ? acc1 : 0u);
        const uint32_t idesc = p.idesc | ((uint32_t)(t.n_eff >> 3) << 17);
        const uint32_t shift = (uint32_t)((t.tn * p.BN) & 127) >> 5;      // B's first row within its tile of scales, in columns
        int kb = t.k0;
        for (; kb < t.k1; ++kb) {
          if (!ready && !mbar_wait(full0 + 8u * stage, phase, &abort_flag, p.status, p.wait_ns)) break;
          tc_fence_after();
          // a look at the next stage's barrier now: a wait takes 170 cycles also where there is nothing to wait for, and this thread's
          // time is what bounded the kernel (two such waits and the products: 840 cycles a stage)
          ready = stage + 1 == (uint32_t)p.stages ? mbar_test(full0, phase ^ 1u) : mbar_test(full0 + 8u * (stage + 1), phase);
          const uint32_t lo = desc_lo(smem_base + stage * p.stage_bytes), sa = sf_col + set * SF_SET, sb = sa + ATOMS * 4u + shift;
          const int ksteps = kb + 1 < p.kblocks ? 4 : p.ksteps_last;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (kk < ksteps) {
              const int a = FMT == MXFP4 ? kk >> 1 : kk;
              const uint32_t id = FMT == MXFP4 ? (uint32_t)(kk & 1) * 2u : 0u;
              umma4<FMT, PAIR>(d, lo + 2u * kk, lo + b_off + 2u * kk, idesc | id << 4 | id << 29, sa + 4u * a, sb + 4u * (a * NSB), kb > t.k0 || kk > 0 ? 1u : 0u);
            }
          }
          // (one commit a stage, for its codes and its scales: a second one to both CTAs took 250 cycles)
          if (PAIR) umma_commit_pair(empty0 + 8u * stage); else umma_commit(empty0 + 8u * stage);
          if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
          if (++set == (uint32_t)p.sets) set = 0;
        }
        if (kb < t.k1) break;
        if (PAIR) umma_commit_pair(smem_u32(&acc_full_bar[acc])); else umma_commit(smem_u32(&acc_full_bar[acc]));
      }
    }
  } else if (warp >= SF_WARP) {
    // ------------------------------------------------------------------ scales: from memory through a ring of their own to tensor memory,
    // stages ahead of the codes, so that the products wait for codes alone. By register and not with tcgen05.cp: that moves 512
    // bytes in 45 to 120 cycles, six or twelve of them a stage, in the same queue as the products. Plain bulk copies: as boxes of a
    // tensor without swizzle they came at 16 bytes a cycle.
    const uint32_t land0 = smem_u32(&land_bar[0]), slot_empty0 = smem_u32(&slot_empty_bar[0]), empty0 = smem_u32(&empty_bar[0]);
    const uint32_t full0 = PAIR ? map_to_cta(smem_u32(&full_bar[0]), 0) : smem_u32(&full_bar[0]);
    const uint32_t sf_col = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + SF_COL;
    constexpr uint32_t SLOT = (1u + NSB) * ATOMS * 512u;
    const uint32_t ring = smem_base + (uint32_t)p.stages * p.stage_bytes + (uint32_t)TC_EPI_WARPS * STG_BYTES;
    uint32_t slot = 0, phase = 0, set = 0, stage = 0, old = 0, old_phase = 0;
    int step = 0;
    bool live = true;
    pdl_wait();
    if (warp == SF_WARP + 4) {
      // this one asks for them: lane 0 for A's row tile, the next for B's. Row tiles that do not exist are not copied: what their
      // place holds meets rows and columns that are not stored.
      for (int tile = tile0; tile < p.total_tiles && live; tile += tile_step) {
        const Tile4 t = tile_of<PAIR>(p, tile);
        const int rt = lane == 0 ? (t.tm * TILE_M >> 7) + (int)rank : (t.tn * p.BN >> 7) + lane - 1, rts = lane == 0 ? p.rt_a : p.rt_b;
        const bool exists = lane < 1 + NSB && rt < rts;
        const uint32_t count = (uint32_t)__popc(__ballot_sync(0xffffffffu, exists));
        const uint8_t* src = (lane == 0 ? p.sa : p.sb) + ((long long)(lane > 0 && p.b_shared ? 0 : t.bz) * rts + rt) * p.kt * 512 + (long long)t.k0 * (ATOMS * 512);
        for (int kb = t.k0; kb < t.k1; ++kb, src += ATOMS * 512) {
          const uint32_t bytes = (uint32_t)min(ATOMS, p.kt - kb * ATOMS) * 512u;
          int ok = 1;
          if (lane == 0) {
            ok = mbar_wait(slot_empty0 + 8u * slot, phase ^ 1u, &abort_flag, p.status, p.wait_ns) ? 1 : 0;
            if (ok) mbar_expect_tx(land0 + 8u * slot, count * bytes);
          }
          if (!__shfl_sync(0xffffffffu, ok, 0)) { live = false; break; }
          if (exists)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(ring + slot * SLOT + (uint32_t)lane * (ATOMS * 512u)), "l"(src), "r"(bytes), "r"(land0 + 8u * slot) : "memory");
          __syncwarp();
          if (++slot == SF_RING) { slot = 0; phase ^= 1u; }
        }
      }
      live = false;
    }
    for (int tile = tile0; tile < p.total_tiles && live; tile += tile_step) {
      const Tile4 t = tile_of<PAIR>(p, tile);
      for (int kb = t.k0; kb < t.k1; ++kb) {
        // The set is free once the products of the stage that had it before are through: no more sets than stages, so that stage's
        // barrier cannot have gone round again, and this stage's barrier counts the scales of no earlier round.
        uint32_t landed = mbar_test(land0 + 8u * slot, phase), free_set = step < p.sets || mbar_test(empty0 + 8u * old, old_phase);
        bool ok = landed || mbar_wait(land0 + 8u * slot, phase, &abort_flag, p.status, p.wait_ns);
        ok = ok && (free_set || mbar_wait(empty0 + 8u * old, old_phase, &abort_flag, p.status, p.wait_ns));
        if (step >= p.sets && ++old == (uint32_t)p.stages) { old = 0; old_phase ^= 1u; }
        ++step;
        if (!__all_sync(0xffffffffu, ok)) { live = false; break; }
        tc_fence_after();
        uint32_t v[ATOMS * 4 * (1 + NSB)];
        // columns: A's four a tile, then B's, the row tiles of one K position side by side
#pragma unroll
        for (int i = 0; i < ATOMS * (1 + NSB); ++i) {
          const int a = i < ATOMS ? i : (i - ATOMS) / NSB, r = i < ATOMS ? 0 : 1 + (i - ATOMS) % NSB;
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[4 * i]), "=r"(v[4 * i + 1]), "=r"(v[4 * i + 2]), "=r"(v[4 * i + 3])
                       : "r"(ring + slot * SLOT + 16u * lane + (uint32_t)r * (ATOMS * 512u) + 512u * a) : "memory");
        }
        const uint32_t dst = sf_col + set * SF_SET;
#pragma unroll
        for (int i = 0; i < ATOMS * (1 + NSB) / 2; ++i) tmem_st8(dst + 8u * i, v + 8 * i);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_cluster(full0 + 8u * stage); else mbar_arrive(full0 + 8u * stage);
          mbar_arrive(slot_empty0 + 8u * slot);
        }
        __syncwarp();
        if (++slot == SF_RING) { slot = 0; phase ^= 1u; }
        if (++set == (uint32_t)p.sets) set = 0;
        if (++stage == (uint32_t)p.stages) stage = 0;
      }
    }
  } else {
    // ------------------------------------------------------------------ read-out: 32 rows and every other chunk of columns a warp
    const int q = warp & 3, wsel = (warp - 2) >> 2;
    const uint32_t stg = smem_base + (uint32_t)p.stages * p.stage_bytes + (uint32_t)(warp - 2) * STG_BYTES;
    const uint32_t empty_sig = PAIR ? map_to_cta(smem_u32(&acc_empty_bar[0]), 0) : smem_u32(&acc_empty_bar[0]);
    const uint32_t ovl_sig = PAIR ? map_to_cta(smem_u32(&ovl_bar), 0) : smem_u32(&ovl_bar);
    const int cw = p.out_f32 ? 32 : 64;            // columns of 128 bytes
    pdl_wait();
    for (int tile = tile0, it = 0; tile < p.total_tiles; tile += tile_step, ++it) {
      const Tile4 t = tile_of<PAIR>(p, tile);
      const uint32_t acc = (uint32_t)it & 1u, use = ((uint32_t)it >> 1) & 1u;
      float alpha = p.alpha, pre = 1.f;
      if (FMT == NVFP4 && p.splits == 1) alpha = output_factor(alpha, p.scale_a[t.bz], p.scale_b[p.b_shared ? 0 : t.bz], pre);
      const int out_z = t.ks * p.batch + t.bz;
      if (!mbar_wait(smem_u32(&acc_full_bar[acc]), use, &abort_flag, p.status, p.wait_ns)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (acc ? acc1 : 0u);
      const int row0 = t.tm * TILE_M + (int)rank * 128 + q * 32, n0 = t.tn * p.BN;
      const int chunks = (t.n_eff + cw - 1) / cw, ovl_chunks = (p.overlap + cw - 1) / cw, full = p.BN / cw;
      // What has left tensor memory is given back at once, before it is packed and stored: the overlapping columns, which come first (the
      // last ones of the first accumulator, the first ones of the second), then the rest.
      auto tell = [&](bool both, bool accumulator) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (both) { if (PAIR) mbar_arrive_cluster(ovl_sig); else mbar_arrive(ovl_sig); }
          if (accumulator) { if (PAIR) mbar_arrive_cluster(empty_sig + 8u * acc); else mbar_arrive(empty_sig + 8u * acc); }
        }
        __syncwarp();
      };
      bool told = !p.overlap;
      if (wsel >= full || (!told && wsel >= ovl_chunks)) { tell(!told, wsel >= full); told = true; }
      for (int i = wsel; i < full; i += 2) {
        const int c = (p.overlap && acc == 0) ? full - 1 - i : i;
        const bool active = c < chunks && row0 < p.M;
        const int col0 = c * cw;
        uint32_t r[64];
        if (active) {
          tmem_ld32(taddr + col0, r);
          if (!p.out_f32) tmem_ld32(taddr + col0 + 32, r + 32);
          tmem_ld_wait();
        }
        const bool ovl_now = !told && i + 2 >= ovl_chunks, last = i + 2 >= full;
        if (ovl_now || last) tell(ovl_now, last);
        told = told || ovl_now;
        if (!active) continue;
        if (FMT == NVFP4 && pre != 1.f) {
#pragma unroll
          for (int j = 0; j < 64; ++j)
            if (j < 32 || !p.out_f32) r[j] = __float_as_uint(pre * __uint_as_float(r[j]));
        }
        // the last store has read the buffer
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int pc = 0; pc < 8; ++pc) {
          uint32_t w[4];
          if (p.out_f32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(alpha * __uint_as_float(r[4 * pc + j]));
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack16x2(alpha * __uint_as_float(r[8 * pc + 2 * j]), alpha * __uint_as_float(r[8 * pc + 2 * j + 1]), false);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stg + (uint32_t)lane * 128u + ((uint32_t)(pc ^ (lane & 7)) << 4)), "r"(w[0]),
                       "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        }
        if (p.store_tma) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (n0 + col0 < p.N) tma_store_3d(&p.tmD, stg, n0 + col0, row0, out_z);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {
          // Rows that the copy engine cannot address: eight lanes a row, four rows at a time; the whole 16-byte pieces that the row has in
          // memory, put together from the staged row, then the elements before and after them, one a lane. (A store takes some ten
          // cycles of the SM whatever it writes: with 4 bytes a lane 4096 x 4097 took 32 us.)
          __syncwarp();
          const int rows = min(32, p.M - row0), have = min(cw, p.N - n0 - col0), es = p.out_f32 ? 4 : 2, sub = lane & 7;
          const long long step = 4 * p.ldd * es;
          uint8_t* d = reinterpret_cast<uint8_t*>(p.D) + ((long long)out_z * p.batch_d + (long long)(row0 + (lane >> 3)) * p.ldd + n0 + col0) * es;
          for (int r = lane >> 3; r < rows; r += 4, d += step) {
            const uint32_t src = stg + (uint32_t)r * 128u, key = (uint32_t)(r & 7);
            const uint32_t before = (16u - (uint32_t)(reinterpret_cast<uintptr_t>(d) & 15u)) & 15u;      // bytes in front of the first whole piece
            if (have == cw) {
              if (sub < (before ? 7 : 8)) {
                const uint32_t first = (before >> 2) + 4u * sub, odd = (before & 2u) * 8u;
                uint32_t a[5];
#pragma unroll
                for (uint32_t k = 0; k < 5; ++k) a[k] = k < 4 || odd ? ld_word(src + (((first + k) >> 2 ^ key) << 4) + ((first + k) & 3u) * 4u) : 0u;
                *reinterpret_cast<uint4*>(d + before + 16 * sub) = make_uint4(__funnelshift_r(a[0], a[1], odd), __funnelshift_r(a[1], a[2], odd),
                                                                              __funnelshift_r(a[2], a[3], odd), __funnelshift_r(a[3], a[4], odd));
              }
              const int ends = before ? 16 / es : 0, heads = (int)before / es;
              if (sub < ends) copy_element(d, src, key, sub < heads ? sub : cw - ends + sub, es);
            } else {
              for (int e = sub; e < have; e += 8) copy_element(d, src, key, e, es);
            }
          }
          __syncwarp();
        }
      }
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // what is on its way to memory gets there before the CTA ends
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (abort_flag && threadIdx.x == 0) {
    // a wait ran out: copies that may still be in flight get a bounded time to land before the shared memory is released
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) { }
  }
  __syncthreads();
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
  }
}

// ----------------------------------------------------------------------------- up to eight rows
constexpr int ROW_THREADS = 256, ROW_CHUNK = 4096;     // values of K that are staged at a time

__device__ __forceinline__ uint32_t lookup(uint32_t sel) {
  // twice the magnitudes 0 .5 1 1.5 2 3 4 6, one byte for each of four codes; codes with the sign bit give zero (prmt's sign mode)
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(0x03020100u), "r"(0x0C080604u), "r"(sel));
  return r;
}

struct RowParams {
  Mx4View A, B;
  int M, N, K, b_shared;
  void* D; long long ldd, batch_d; int out_f32;
  float alpha;
};

// LPR lanes a row of B: 16 where there are rows enough, else half the CTA. T >= M rows of A. The weights are asked for ahead of
// everything else, a group of pieces (32 codes) a lane, and the next group before one is worked on: a call of one token is a few
// microseconds, of which the first trip to memory is one.
template <int FMT, int T, int LPR>
__global__ void __launch_bounds__(ROW_THREADS) mx4_row_kernel(const RowParams p) {
  constexpr int BLK = FMT == MXFP4 ? 32 : 16, NB = 32 / BLK, GROUP = LPR == 16 ? 4 : 1;
  static_assert(ROW_CHUNK / 32 % (LPR * GROUP) == 0, "a group does not straddle two chunks");
  __shared__ __align__(16) int8_t s_a[T][ROW_CHUNK];
  __shared__ float s_sc[T][ROW_CHUNK / BLK];
  __shared__ float s_part[ROW_THREADS / 32][T];
  const int tid = threadIdx.x, lane = tid & 31;
  const int bz = blockIdx.y;
  const int width = mx4_width(p.K), pieces = width / 32, kt = mx4_scale_tiles(p.K, FMT);
  const long long n = (long long)blockIdx.x * (ROW_THREADS / LPR) + tid / LPR;
  const bool row_ok = n < p.N;
  const int at0 = tid % LPR;
  const int bb = p.b_shared ? 0 : bz;
  const uint4* const w = reinterpret_cast<const uint4*>(p.B.codes + ((long long)bb * p.N + (row_ok ? n : 0)) * (width / 2));
  const int nr = row_ok ? (int)n : 0;
  const uint8_t* const ws = p.B.scales + ((long long)bb * mx4_row_tiles(p.N) + (nr >> 7)) * kt * 512 + (nr & 31) * 16 + ((nr >> 5) & 3) * 4;
  const uint8_t* const ac = p.A.codes + (long long)bz * p.M * (width / 2);
  const uint8_t* const as = p.A.scales + (long long)bz * mx4_row_tiles(p.M) * kt * 512;
  uint4 next[GROUP];
  uint32_t next_sb[GROUP];
  auto fetch = [&](int first) {
#pragma unroll
    for (int k = 0; k < GROUP; ++k) {
      const int i = first + at0 + k * LPR;
      next[k] = make_uint4(0, 0, 0, 0);
      next_sb[k] = 0;
      if (row_ok && i < pieces) {
        next[k] = w[i];
        if (FMT == MXFP4) next_sb[k] = ws[(long long)(i >> 2) * 512 + (i & 3)];
        else next_sb[k] = *reinterpret_cast<const uint16_t*>(ws + (long long)(i >> 1) * 512 + (i & 1) * 2);
      }
    }
  };
  float sum[T];
#pragma unroll
  for (int t = 0; t < T; ++t) sum[t] = 0.f;
  pdl_wait();
  fetch(0);
  for (int k0 = 0; k0 < width; k0 += ROW_CHUNK) {
    const int kn = min(ROW_CHUNK, width - k0);
    if (k0) __syncthreads();
    for (int u = tid; u < T * (kn / 8); u += ROW_THREADS) {
      const int t = T == 1 ? 0 : u / (kn / 8), o = u - t * (kn / 8);
      uint32_t codes = 0;
      if (t < p.M) codes = *reinterpret_cast<const uint32_t*>(ac + (long long)t * (width / 2) + k0 / 2 + 4 * o);
      // signed bytes: the positive ones less the negative ones, byte by byte
      const uint32_t lo = __vsub4(lookup(codes & 0xffffu), lookup((codes & 0xffffu) ^ 0x8888u));
      const uint32_t hi = __vsub4(lookup(codes >> 16), lookup((codes >> 16) ^ 0x8888u));
      *reinterpret_cast<uint2*>(&s_a[t][8 * o]) = make_uint2(lo, hi);
    }
    for (int u = tid; u < T * (kn / BLK); u += ROW_THREADS) {
      const int t = T == 1 ? 0 : u / (kn / BLK), j = u - t * (kn / BLK), blk = k0 / BLK + j;
      float s = 0.f;
      if (t < p.M) s = 0.25f * scale_value<FMT>(as[(long long)(blk >> 2) * 512 + (t & 31) * 16 + (blk & 3)]);
      s_sc[t][j] = s;
    }
    __syncthreads();
    const int first = k0 / 32, last = first + kn / 32;
    for (int i0 = first; i0 < last; i0 += GROUP * LPR) {
      uint4 cur[GROUP];
      uint32_t cur_sb[GROUP];
#pragma unroll
      for (int k = 0; k < GROUP; ++k) { cur[k] = next[k]; cur_sb[k] = next_sb[k]; }
      fetch(i0 + GROUP * LPR);
#pragma unroll
      for (int k = 0; k < GROUP; ++k) {
        const int i = i0 + at0 + k * LPR;
        if (i >= last) break;
        const uint32_t c[4] = {cur[k].x, cur[k].y, cur[k].z, cur[k].w};
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const uint4* a4 = reinterpret_cast<const uint4*>(&s_a[t][(i - first) * 32]);
          const uint4 a0 = a4[0], a1 = a4[1];
          const uint32_t a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
          for (int h = 0; h < NB; ++h) {
            int pos = 0, neg = 0;
#pragma unroll
            for (int j = 0; j < 4 / NB; ++j) {
              const uint32_t x = c[h * (4 / NB) + j];
              const int al = (int)a[2 * (h * (4 / NB) + j)], ah = (int)a[2 * (h * (4 / NB) + j) + 1];
              pos = __dp4a((int)lookup(x & 0xffffu), al, pos);
              neg = __dp4a((int)lookup((x & 0xffffu) ^ 0x8888u), al, neg);
              pos = __dp4a((int)lookup(x >> 16), ah, pos);
              neg = __dp4a((int)lookup((x >> 16) ^ 0x8888u), ah, neg);
            }
            const float sa = s_sc[t][(i - first) * NB + h], sb = scale_value<FMT>(h ? cur_sb[k] >> 8 : cur_sb[k] & 0xffu);
            // The sum meets one scale after the other: their product alone may leave fp32's range. mxfp4, the smaller one first: that product is
            // exact (an integer times at least 2^-129), and the sum times the larger one alone may be past fp32 where the result is not.
            const bool up = FMT == MXFP4 && sb < sa;               // (false beside a NaN, which stays in either place)
            sum[t] += (float)(pos - neg) * (up ? sb : sa) * (up ? sa : sb);
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int o = (LPR < 32 ? LPR : 32) / 2; o > 0; o >>= 1) sum[t] += __shfl_xor_sync(0xffffffffu, sum[t], o);
  if (LPR > 32) {
    if (lane == 0)
#pragma unroll
      for (int t = 0; t < T; ++t) s_part[tid >> 5][t] = sum[t];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < T; ++t) {
      sum[t] = 0.f;
      for (int k = 0; k < LPR / 32; ++k) sum[t] += s_part[tid / LPR * (LPR / 32) + k][t];
    }
  }
  if (row_ok && at0 == 0) {
    float alpha = p.alpha, pre = 1.f;
    if (FMT == NVFP4) alpha = output_factor(alpha, p.A.scale[bz], p.B.scale[bb], pre);
#pragma unroll
    for (int t = 0; t < T; ++t)
      if (t < p.M) {
        sum[t] *= pre;
        const long long at = (long long)bz * p.batch_d + (long long)t * p.ldd + n;
        if (p.out_f32) reinterpret_cast<float*>(p.D)[at] = alpha * sum[t];
        else reinterpret_cast<__nv_bfloat16*>(p.D)[at] = __float2bfloat16_rn(alpha * sum[t]);
      }
  }
}

// ----------------------------------------------------------------------------- host side
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(ptr);
  });
  return fn;
}

// [batch, rows, inner], boxes of box_inner x box_rows, 128 bytes wide and swizzled
bool encode(CUtensorMap* tm, CUtensorMapDataType type, const void* base, long long inner, long long rows, long long batch, long long row_bytes,
            long long batch_bytes, uint32_t box_inner, uint32_t box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch};
  const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)batch_bytes};
  const cuuint32_t box[3] = {box_inner, box_rows, 1}, est[3] = {1, 1, 1};
  return encode_fn()(tm, type, 3, const_cast<void*>(base), dims, strides, box, est, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Few tiles and a long K: K in up to eight parts, at least four stages each, whose sums in fp32 a second launch adds in order.
// (us without and with: 16 x 1600 x 6400 13.4 and 8.3, 128 x 1600 x 6400 13.7 and 9.5, 256 x 256 x 8192 15.8 and 9.2, 100 x 500 x 2048 9.2
// and 7.6, 128 x 1600 x 3200 8.9 and 8.6; parts of two or three stages lose: 16 x 768 x 1600 6.1 and 7.1.)
int choose_splits(long long tiles, int kblocks, int slots) {
  if (tiles * 2 > slots) return 1;
  int n = (int)(slots / tiles);
  if (n > kblocks / 4) n = kblocks / 4;
  if (n > 8) n = 8;
  return n < 2 ? 1 : n;
}

// D = alpha * the sum of the parts (and the matrices' scales), in order. A row of D a block row, four columns a thread.
template <typename O>
__global__ void __launch_bounds__(128) mx4_join_kernel(const float* parts, int splits, int M, int N, int np, long long part, O* D, long long ldd,
                                                       long long batch_d, float alpha, const float* scale_a, const float* scale_b, int b_shared) {
  const int z = blockIdx.y, bz = z / M, r = z - bz * M, c = 4 * ((int)blockIdx.x * 128 + (int)threadIdx.x);
  pdl_wait();
  if (c >= N) return;
  const float* x = parts + (long long)z * np + c;
  float4 sum = *reinterpret_cast<const float4*>(x);
#pragma unroll 4
  for (int k = 1; k < splits; ++k) {
    const float4 y = *reinterpret_cast<const float4*>(x + k * part);
    sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
  }
  float pre = 1.f;
  if (scale_a) alpha = output_factor(alpha, scale_a[bz], scale_b[b_shared ? 0 : bz], pre);
  const float v[4] = {alpha * (pre * sum.x), alpha * (pre * sum.y), alpha * (pre * sum.z), alpha * (pre * sum.w)};
  O* const d = D + bz * batch_d + (long long)r * ldd + c;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < N) d[j] = (O)v[j];
}

// Tile width: the one with the smallest modelled time in cycles. A stage takes the tensor pipe 2 cycles a column, at least what a step
// of the issuing thread takes, at least its operand bytes at the 5500 bytes a cycle that L2 delivers to the chip; the read-out of a
// tile overlaps the next tile's stages, except the last.
int choose_width(const Mx4Gemm& g, bool pair, int num_sms) {
  static const int widths[4] = {256, 192, 128, 64};      // (64 bf16 columns are the read-out's 128 bytes)
  const int slots = pair ? num_sms / 2 : num_sms, tm = (g.M + (pair ? 255 : 127)) / (pair ? 256 : 128);
  const double kb = (g.K + KB_ELEMENTS - 1) / KB_ELEMENTS;
  int best = 0;
  double best_t = 0.0;
  for (int bn : widths) {
    if (bn > 64 && bn / 2 >= g.N) continue;
    const double tiles = (double)g.b * tm * ((g.N + bn - 1) / bn), waves = (double)(long long)((tiles + slots - 1) / slots);
    const double live = (tiles < slots ? tiles : slots) * (pair ? 2 : 1);
    double step = 2.0 * bn;
    if (step < 300.0) step = 300.0;
    const double bytes = (128.0 + (pair ? bn / 2 : bn)) * KB_BYTES + 6.0 * 512.0;      // (and the scales)
    if (step < bytes * live / 5500.0) step = bytes * live / 5500.0;
    const double out = 1000.0 + bn * (g.out_dtype == F32 ? 16.0 : 10.0);
    const double t = (waves - 1.0) * (kb * step > out ? kb * step : out) + kb * step + out;
    if (!best || t < best_t) { best = bn; best_t = t; }
  }
  return best;
}

template <int FMT, int PAIR, int NSB>
cudaError_t tc_start(const TcParams4& p, int grid, size_t smem, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(TC_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = PAIR ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, mx4_tc_kernel<FMT, PAIR, NSB>, p);
}

// Whether up to eight rows go through mx4_row_kernel. Its time grows with the rows it works out (M rounded up to a power of two) times the
// weights, since every weight is looked up once and multiplied with each row; the tensor cores' form takes the same for any M here. us, row
// kernel and tensor cores, mxfp4 with weights from HBM (nvfp4 is within a tenth of it, five to eight rows up to 1.3 times as long):
//   N x K             M = 1        2           3, 4        5 to 8
//   768 x 768         2.0  4.3   2.3  4.3    2.8  4.3    4.2  4.4
//   1600 x 1600       2.8  6.3   3.5  6.3    4.4  6.3    7.1  6.3
//   2048 x 2048       2.9  7.5   3.6  7.4    4.7  7.5    7.8  7.5     2^25 products in eight rows
//   4096 x 2048       3.6  7.7   4.5  7.7    6.2  7.8   10.3  7.9     2^25 in four
//   6400 x 1600       4.3  6.5   5.2  6.5    7.2  6.6   11.8  6.6
//   4096 x 4096       5.0  9.7   6.9  9.7   10.5  9.7   18.3  9.7     2^25 in two
//   12800 x 1600      6.6  7.6   8.8  7.8   12.4  7.6   21.4  7.8
//   16384 x 4096     11.8 13.8  17.7 13.9   30.5 13.8   53.9 14.3     2^26 in one
//   25600 x 1600     10.6  9.6  14.9 10.6   21.4 10.7   36.7 10.2
//   20000 x 256       5.6  4.7   6.9  4.7    8.2  4.7   11.7  4.7     (a CTA for sixteen rows of B: short ones are mostly its start)
bool by_rows(int b, int M, int N, int K) {
  const int t = M <= 2 ? M : M <= 4 ? 4 : 8;
  return M <= 8 && (long long)b * N <= 16384 && (long long)b * N * K * t <= (t == 1 ? 1ll << 26 : 1ll << 25);
}

template <int FMT, int T>
cudaError_t row_start(const RowParams& p, int b, int num_sms, cudaStream_t st) {
  // Sixteen lanes a row of B from four rows an SM on (long rows, which are worth more lanes: six), else half a CTA. us with 16 and with 128 lanes, mxfp4, one row of A and eight:
  //   K 256    N 592   2.0  2.1   3.1  3.1     N 768   2.0  2.2   3.0  3.7     N 1024   2.0  2.4   3.1  4.1
  //   K 1600   N 592   2.4  2.3   6.7  5.4     N 768   2.4  2.4   6.7  5.9     N 1024   2.4  2.5   6.7  7.6
  //   K 6400   N 592   4.9  3.5  20.3 13.6     N 768   4.9  3.7  20.2 15.3     N 1024   4.9  4.2  20.3 19.8     N 1600   4.9  5.6  20.3 28.0
  if (p.N >= num_sms * (p.K <= 1024 ? 4 : 6)) return launch_kernel(mx4_row_kernel<FMT, T, 16>, dim3((unsigned)((p.N + 15) / 16), (unsigned)b), dim3(ROW_THREADS), 0, st, p);
  return launch_kernel(mx4_row_kernel<FMT, T, ROW_THREADS / 2>, dim3((unsigned)((p.N + 1) / 2), (unsigned)b), dim3(ROW_THREADS), 0, st, p);
}
template <int FMT>
cudaError_t row_pick(const RowParams& p, int b, int num_sms, cudaStream_t st) {
  if (p.M == 1) return row_start<FMT, 1>(p, b, num_sms, st);
  if (p.M == 2) return row_start<FMT, 2>(p, b, num_sms, st);
  if (p.M <= 4) return row_start<FMT, 4>(p, b, num_sms, st);
  return row_start<FMT, 8>(p, b, num_sms, st);
}

}  // namespace

namespace {
template <int FMT, int PAIR>
cudaError_t tc_limit() {
  const cudaError_t e = cudaFuncSetAttribute(mx4_tc_kernel<FMT, PAIR, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST - 1024);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(mx4_tc_kernel<FMT, PAIR, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST - 1024);
}
template <int FMT>
cudaError_t tc_pick(const TcParams4& p, bool pair, int nsb, int grid, size_t smem, cudaStream_t st) {
  if (pair) return nsb == 1 ? tc_start<FMT, 1, 1>(p, grid, smem, st) : tc_start<FMT, 1, 2>(p, grid, smem, st);
  return nsb == 1 ? tc_start<FMT, 0, 1>(p, grid, smem, st) : tc_start<FMT, 0, 2>(p, grid, smem, st);
}
}  // namespace

cudaError_t mx4_gemm_prepare() {
  cudaError_t e;
  if ((e = tc_limit<MXFP4, 0>()) != cudaSuccess || (e = tc_limit<MXFP4, 1>()) != cudaSuccess || (e = tc_limit<NVFP4, 0>()) != cudaSuccess) return e;
  return tc_limit<NVFP4, 1>();
}

Mx4Split mx4_gemm_split(int b, int M, int N, int K, int out_dtype, int num_sms) {
  Mx4Split r = {1, 0};
  if (by_rows(b, M, N, K)) return r;
  Mx4Gemm g = {};
  g.b = b; g.M = M; g.N = N; g.K = K; g.out_dtype = out_dtype;
  const bool pair = M > 128;
  const int bn = choose_width(g, pair, num_sms), kblocks = (mx4_width(K) + KB_ELEMENTS - 1) / KB_ELEMENTS;
  const long long tiles = (long long)b * ((M + (pair ? 255 : 127)) / (pair ? 256 : 128)) * ((N + bn - 1) / bn);
  r.splits = choose_splits(tiles, kblocks, pair ? num_sms / 2 : num_sms);
  if (r.splits > 1) {
    // (no part without a stage)
    const int per = (kblocks + r.splits - 1) / r.splits;
    r.splits = (kblocks + per - 1) / per;
    r.work_bytes = (size_t)r.splits * b * M * ((N + 3) & ~3) * sizeof(float);
  }
  return r;
}

cudaError_t mx4_gemm_launch(const Mx4Gemm& g, cudaStream_t st, int* status, int num_sms, unsigned long long wait_ns, bool hold, long long* launches) {
  if (by_rows(g.b, g.M, g.N, g.K)) {
    RowParams r;
    r.A = g.A; r.B = g.B; r.M = g.M; r.N = g.N; r.K = g.K; r.b_shared = g.b_shared;
    r.D = g.D; r.ldd = g.ldd; r.batch_d = g.batch_d; r.out_f32 = g.out_dtype == F32; r.alpha = g.alpha;
    if (launches) ++*launches;
    return g.fmt == MXFP4 ? row_pick<MXFP4>(r, g.b, num_sms, st) : row_pick<NVFP4>(r, g.b, num_sms, st);
  }
  if (!encode_fn()) return cudaErrorNotSupported;
  const bool pair = g.M > 128;
  const int slots = pair ? num_sms / 2 : num_sms;
  TcParams4 p;
  p.M = g.M; p.N = g.N; p.batch = g.b; p.b_shared = g.b_shared;
  p.BN = choose_width(g, pair, num_sms);
  p.tiles_m = (g.M + (pair ? 255 : 127)) / (pair ? 256 : 128);
  p.tiles_n = (g.N + p.BN - 1) / p.BN;
  const long long total = (long long)p.tiles_m * p.tiles_n * g.b;
  if (total > 0x3fffffff) return cudaErrorInvalidValue;
  const int width = mx4_width(g.K), atoms = g.fmt == MXFP4 ? 2 : 4;
  p.kblocks = (width + KB_ELEMENTS - 1) / KB_ELEMENTS;
  const Mx4Split split = mx4_gemm_split(g.b, g.M, g.N, g.K, g.out_dtype, num_sms);
  p.splits = g.work ? split.splits : 1;
  p.kper = (p.kblocks + p.splits - 1) / p.splits;
  p.total_tiles = (int)total * p.splits;
  p.ksteps_last = (width - (p.kblocks - 1) * KB_ELEMENTS + 63) / 64;
  const int nsb = p.BN <= 128 ? 1 : 2;
  p.overlap = 2 * p.BN > (int)scale_column(g.fmt) ? 2 * p.BN - (int)scale_column(g.fmt) : 0;
  const uint32_t b_rows = (uint32_t)(pair ? p.BN / 2 : p.BN);
  p.a_bytes = 128 * KB_BYTES; p.b_bytes = b_rows * KB_BYTES;
  p.stage_bytes = p.a_bytes + p.b_bytes;
  const uint32_t ring = (uint32_t)(scale_ring(g.fmt) * (1 + nsb) * atoms) * 512u, stg = (uint32_t)TC_EPI_WARPS * STG_BYTES, room = SMEM_MOST - 1024 - 1024 - stg - ring;
  p.stages = (int)(room / p.stage_bytes);
  if (p.stages > MAX_ST) p.stages = MAX_ST;
  p.sets = p.stages < SF_SETS ? p.stages : SF_SETS;
  const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + stg + ring;
  // kind::mxf4 / mxf4nvf4: e2m1 operands (1), both K-major; scales e8m0 (1) or e4m3 (0); M / 16 and N / 8 (added per tile)
  p.idesc = 1u << 7 | 1u << 10 | (g.fmt == MXFP4 ? 1u : 0u) << 23 | (pair ? 16u : 8u) << 24;
  p.out_f32 = g.out_dtype == F32;
  const bool join = p.splits > 1;
  const int np = (g.N + 3) & ~3, out_n = join ? np : g.N, out_b = p.splits * g.b;
  p.out_f32 = join || g.out_dtype == F32;
  if (join) { p.D = g.work; p.ldd = np; p.batch_d = (long long)g.M * np; }
  else { p.D = g.D; p.ldd = g.ldd; p.batch_d = g.batch_d; }
  p.alpha = join ? 1.f : g.alpha; p.scale_a = g.A.scale; p.scale_b = g.B.scale;
  p.status = status; p.wait_ns = wait_ns; p.hold = hold;
  const long long es = p.out_f32 ? 4 : 2;
  // (whole rows of 16-byte pieces: the copy engine writes the last piece in full, past a row that ends inside it)
  p.store_tma = (reinterpret_cast<uintptr_t>(p.D) & 15u) == 0 && (out_n * es) % 16 == 0 && (p.ldd * es) % 16 == 0 && (out_b == 1 || (p.batch_d * es) % 16 == 0);
  const int bb = g.b_shared ? 1 : g.b;
  bool ok = encode(&p.tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.A.codes, width / 2, g.M, g.b, width / 2, (long long)g.M * (width / 2), KB_BYTES, 128) &&
            encode(&p.tmB, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.B.codes, width / 2, g.N, bb, width / 2, (long long)g.N * (width / 2), KB_BYTES, b_rows);
  p.sa = g.A.scales; p.sb = g.B.scales; p.rt_a = mx4_row_tiles(g.M); p.rt_b = mx4_row_tiles(g.N); p.kt = mx4_scale_tiles(g.K, g.fmt);
  if (ok && p.store_tma) {
    const long long batch_bytes = out_b > 1 ? p.batch_d * es : p.ldd * es * g.M;
    ok = encode(&p.tmD, p.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p.D, out_n, g.M, out_b, p.ldd * es, batch_bytes,
                p.out_f32 ? 32 : 64, 32);
  }
  if (!ok) return cudaErrorInvalidValue;
  const int runs = p.total_tiles < slots ? p.total_tiles : slots, grid = pair ? 2 * runs : runs;
  if (launches) ++*launches;
  const cudaError_t e = g.fmt == MXFP4 ? tc_pick<MXFP4>(p, pair, nsb, grid, smem, st) : tc_pick<NVFP4>(p, pair, nsb, grid, smem, st);
  if (e != cudaSuccess || !join) return e;
  if (launches) ++*launches;
  const dim3 blocks((unsigned)((np / 4 + 127) / 128), (unsigned)(g.b * g.M));
  const float* const sa = g.fmt == NVFP4 ? g.A.scale : nullptr;
  const long long part = (long long)g.b * g.M * np;
  if (g.out_dtype == F32)
    return launch_kernel(mx4_join_kernel<float>, blocks, dim3(128), 0, st, (const float*)g.work, p.splits, g.M, g.N, np, part, (float*)g.D, g.ldd, g.batch_d,
                         g.alpha, sa, g.B.scale, g.b_shared);
  return launch_kernel(mx4_join_kernel<__nv_bfloat16>, blocks, dim3(128), 0, st, (const float*)g.work, p.splits, g.M, g.N, np, part, (__nv_bfloat16*)g.D, g.ldd,
                       g.batch_d, g.alpha, sa, g.B.scale, g.b_shared);
}

}  // namespace defl
