// Weight gradient of a linear layer whose input was kept as an 8-bit checkpoint:
//   dW[n, k] = sum_m dY[m, n] * X[m, k],   db[n] = sum_m dY[m, n]
// X = the checkpoint's values, or, when the layer's input was a layer norm and the checkpoint holds its normalised
// values xh, X = xh gamma + beta: the affine then leaves the sum,
//   dW[n, k] = gamma[k] * sum_m dY[m, n] xh[m, k] + db[n] * beta[k].
//
// The contraction runs on tcgen05 kind::f16 with bfloat16 operands and FP32 accumulators.  A checkpoint's value has at
// most 7 significant bits, so it is exact in bfloat16; dY is taken as a sum of bfloat16 parts that is exact: one part
// for bfloat16, two for half (8 + 3 bits), three for FP32 (3 x 8 bits; of values below 2^-110 the bits under 2^-133, bfloat16's
// smallest subnormal, are cut off).  Every product is then exact.
//
// The tensor core's accumulator truncates: summing S steps of 16 rows moves a sum of random terms by about
// 2^-24 * 2/3 * S of itself (measured with a library product: 4.7e-7 at 512 rows, 1.9e-5 at 16384).  So the accumulator is
// emptied every WG_CHUNK_STEPS steps (one stage, 12 steps, with three parts) and the chunks are added in FP32 registers, which
// rounds to nearest.  A step truncates by the accumulator's size, however small its own products: a stage takes the lowest parts
// of dY first, while the accumulator is small
// (128 rows of FP32 dY, 500 x 784: 6.3e-8 of the result; chunks of 24 steps with the leading part first had 5.8e-7, a product in
// FP32 has 2.0e-7; 8192 x 2000 x 2000 takes 167 us either way).  With one or two parts, chunks of 16 steps instead of 32 would
// halve the error (bfloat16 512 x 500 x 784 1.0e-7 -> 6.0e-8, the FP32 product 5.7e-8) and cost 3 to 8 % (2048 x 2000 x 2000 29.6 -> 30.8 us,
// half 8192 x 2000 x 784 92.9 -> 100); 32 stay, whose error no longer grows past 512 rows.
//
// Two kernels.  wgrad_prepare_kernel writes the checkpoint's values as bfloat16 into the workspace (and the parts of a dY
// that is not bfloat16 with 16-byte rows), and sums dY's columns on the way.  wgrad_gemm_kernel is a matrix product fed by
// TMA alone.  Expanding the codes inside the product was built first: its warps' chain of barrier waits, shared-memory
// reads, expansion, fence and arrival took 800 to 900 clocks a stage of 64 rows against 512 of the MMAs, however the warps were
// divided, and every tile row expanded the same codes again (4.4 ms against 3.8 to 4.1 at 32768 x 8192 x 8192).
//
// A pair of CTAs (cta_group::2) owns a 256 (n) x bn (k) tile; each stages its 128 rows of n and its half of k.  Both
// operands are read along their contiguous dimension, so both are MN-major: a stage holds 64 contraction rows as blocks
// of 64 columns with the 128-byte swizzle.  Roles of a CTA's 12 warps: warp 0 TMA, warp 1 MMA issue (leader CTA), warps 4-11
// add the chunks, apply the affine, store.  The accumulator is double-buffered in tensor memory (2 x 256 columns), so that
// chunks are added while the next one runs.  Work items are (tile, split of the rows); with one split the epilogue writes
// dW, otherwise partial sums that wgrad_join_kernel adds in order.  Every wait is bounded.
#pragma once
#include "gemm_tc.cuh"
#include "layernorm.cuh"

namespace ffi8 {

constexpr int WG_THREADS = 384;
constexpr int WG_ROWS = 64;                     // contraction rows of a stage
constexpr uint32_t WG_TILE_BYTES = WG_ROWS * 256;   // 64 rows x 128 columns of bfloat16
constexpr int WG_CHUNK_STEPS = 32;              // MMA steps (16 rows of one part) between two emptyings of the accumulator
constexpr uint32_t WG_PATCH_BYTES = 32 * 128;   // 32 rows x 32 columns of FP32: an adding warp's way to whole lines

struct WgradArgs {
  const void* dy;
  long long ld_dy;
  C8View c;
  const float* gamma;
  const float* beta;
  float* dw;             // [N, K]
  float* db;             // nullable [N]
  __nv_bfloat16* x;      // workspace: the checkpoint's values, [rows][ld_x]
  __nv_bfloat16* parts;  // workspace: the parts of dY, [parts][rows][ld_parts]; NULL: dY itself is the operand
  float* db_part;        // workspace: [db_parts][N] sums of dY over groups of rows; NULL: neither db nor beta is given
  float* part;           // workspace, splits > 1: [splits][N][K]
  long long rows, db_rows, ld_x, ld_parts;
  int N, K, accumulate, db_parts;
  int bn;                // tile width along k: a multiple of 64, at most 256
  int tiles_n, tiles_k, splits, stages_per_split, stages;  // stages: of the whole contraction
  uint32_t* status;
};

template <int PARTS>
struct WgGeom {
  static constexpr uint32_t STAGE_BYTES = (PARTS + 1) * WG_TILE_BYTES;   // parts of dY, then X
  static constexpr int STAGES = PARTS == 1 ? 6 : PARTS == 2 ? 4 : 3;
  static constexpr uint32_t SMEM_BYTES = STAGES * STAGE_BYTES + 8 * WG_PATCH_BYTES + 1024 + 512;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
  static constexpr int CHUNK_STAGES = PARTS == 3 ? 1 : WG_CHUNK_STEPS / (PARTS * (WG_ROWS / 16));
};

// D = FP32, A and B = bfloat16, both MN-major, M = 256 over the CTA pair
__device__ __forceinline__ uint32_t wg_idesc(int bn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(bn >> 3) << 17) | ((256u >> 4) << 24);
}
__device__ __forceinline__ void wg_mma(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem_d),
               "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void wg_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void wg_sts16(uint32_t dst, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 wg_lds16(uint32_t src) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
  return v;
}
// Four codes to four bfloat16 values code * 2^E, `scale` = 2^E twice.  In 0x43bb with bb the code's byte, the low seven
// bits are those of 128 + low7; subtracting 128, or 256 where the byte's top bit is set, leaves the code.
__device__ __forceinline__ uint2 wg_expand4(uint32_t c, uint32_t scale) {
  uint32_t r[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t v = __byte_perm(c, 0x43434343u, i ? 0x4342 : 0x4140);
    uint32_t q;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(q) : "r"(v & 0xff7fff7fu), "r"((v & 0x00800080u) | 0xC300C300u));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(q), "r"(scale));
  }
  return make_uint2(r[0], r[1]);
}
__device__ __forceinline__ uint4 wg_expand8(uint32_t c0, uint32_t c1, uint32_t scale) {
  const uint2 a = wg_expand4(c0, scale), b = wg_expand4(c1, scale);
  return make_uint4(a.x, a.y, b.x, b.y);
}
// Eight values as PARTS groups of bfloat16 whose sum is exact: the leading 8 significant bits are cut off, then those of
// the remainder.  An Inf or NaN goes whole into the first part.
template <int PARTS>
__device__ __forceinline__ void wg_split8(const float (&v)[8], uint4 (&out)[PARTS]) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool special = p == 0 && !(fabsf(v[j]) < __uint_as_float(0x7f800000u));
      w[j] = __float_as_uint(r[j]) & 0xffff0000u;
      if (special) w[j] = v[j] == v[j] ? w[j] : 0x7fff0000u;
      if (p + 1 < PARTS) r[j] = special ? 0.0f : __fsub_rn(r[j], __uint_as_float(w[j]));
    }
    out[p] = make_uint4(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632), __byte_perm(w[4], w[5], 0x7632),
                        __byte_perm(w[6], w[7], 0x7632));
  }
}

// Position in the list of stages that a CTA pair works through.
struct WgCursor {
  int item, st, st_end;
  int n0, k0;   // first n / k of the tile
  __device__ __forceinline__ bool start(const WgradArgs& p, int it) {
    item = it;
    if (it >= p.tiles_n * p.tiles_k * p.splits) return false;
    const int tile = it / p.splits, split = it - tile * p.splits;
    int tn, tk;
    tile_coords(tile, p.tiles_n, p.tiles_k, 16, tn, tk);   // 3.61 ms against 3.75 with 8 and 3.85 with 4 at 32768 x 8192 x 8192
    n0 = tn * 256, k0 = tk * p.bn;
    st = split * p.stages_per_split;
    st_end = min(p.stages, st + p.stages_per_split);
    return true;
  }
  __device__ __forceinline__ bool next(const WgradArgs& p, int step) { return ++st < st_end || start(p, item + step); }
};

// The checkpoint's values and dY's parts and column sums.  Blocks below x_blocks expand 256 units of 16 codes each
// (unit i: 16 columns of a row); the others take dy_lanes groups of 8 columns of dY (a power of two, at most 32: a narrow dY
// leaves the other threads to more rows) and db_rows rows.
template <typename T, int PARTS, bool SPLIT, int A>
__global__ void __launch_bounds__(256) wgrad_prepare_kernel(const WgradArgs p, GroupList units, uint32_t x_blocks, uint32_t dy_cols, int dy_lanes) {
  dependents_may_start();
  if (blockIdx.x < x_blocks) {
    constexpr int U = 4;
    const uint32_t i0 = blockIdx.x * (256 * U) + threadIdx.x;
    uint4 c[U];
    uint32_t e[U], row[U], col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      group_at(units, i0 + u * 256, row[u], col[u]);
      col[u] *= 2;   // 16 columns a unit, 8 a group
      if (i0 + u * 256 < units.total && (long long)col[u] < p.ld_x) {
        c[u] = __ldcs(reinterpret_cast<const uint4*>(p.c.q + (long long)row[u] * p.c.ld_q + col[u]));
        e[u] = p.c.e[(long long)row[u] * p.c.ld_e + col[u] / C8_BLOCK];
      } else {
        row[u] = 0xffffffffu;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (row[u] == 0xffffffffu) continue;
      const uint32_t scale = e[u] << 7 | e[u] << 23;   // 2^E twice, as bfloat16
      uint4* dst = reinterpret_cast<uint4*>(p.x + (long long)row[u] * p.ld_x + col[u]);
      dst[0] = wg_expand8(c[u].x, c[u].y, scale);
      dst[1] = wg_expand8(c[u].z, c[u].w, scale);
    }
    return;
  }
  __shared__ float acc[256 * 16];   // row lanes x (8 lanes + 8): 2048 + 2048 / dy_lanes
  const uint32_t b = blockIdx.x - x_blocks, bx = b % dy_cols, by = b / dy_cols;
  const int gx = threadIdx.x & (dy_lanes - 1), ly = threadIdx.x / dy_lanes, row_lanes = 256 / dy_lanes, pitch = dy_lanes * 8 + 8;
  const int col = ((int)bx * dy_lanes + gx) * 8, n = p.N - col;
  const T* dy = static_cast<const T*>(p.dy);
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = 0.0f;
  const long long r0 = by * p.db_rows, r1 = min(r0 + p.db_rows, p.rows);
  for (long long row = r0 + ly; row < r1; row += 4 * row_lanes) {
    Raw8<T> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long m = row + i * row_lanes;
      raw[i] = load8<T, A>(dy + (m < r1 ? m : row) * p.ld_dy + col, m < r1 ? n : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
      unpack8(raw[i], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
      if (SPLIT && n > 0 && row + i * row_lanes < r1) {
        uint4 parts[PARTS];
        wg_split8<PARTS>(v, parts);
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
          *reinterpret_cast<uint4*>(p.parts + ((size_t)q * p.rows + row + i * row_lanes) * p.ld_parts + col) = parts[q];
      }
    }
  }
  if (!p.db_part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[ly * pitch + gx * 8 + j] = s[j];
  __syncthreads();
  for (int h = row_lanes / 2; h >= 8; h >>= 1) {   // many row lanes: halve them first
    for (int i = threadIdx.x; i < h * dy_lanes * 8; i += 256) {
      const int l = i / (dy_lanes * 8), k = i - l * dy_lanes * 8;
      acc[l * pitch + k] += acc[(l + h) * pitch + k];
    }
    __syncthreads();
  }
  const int c = (int)bx * dy_lanes * 8 + threadIdx.x;
  if ((int)threadIdx.x < dy_lanes * 8 && c < p.N) {
    float t = 0.0f;
#pragma unroll
    for (int l = 0; l < 8; ++l) t += acc[l * pitch + threadIdx.x];
    p.db_part[(size_t)by * p.N + c] = t;
  }
}

struct WgRing {  // position in a ring of N slots: slot s, completed rounds' parity ph
  uint32_t s = 0, ph = 0;
  template <int N>
  __device__ __forceinline__ void step() {
    if (++s == N) s = 0, ph ^= 1u;
  }
};

template <int PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WG_THREADS, 1)
    wgrad_gemm_kernel(const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_x, const WgradArgs p) {
  using G = WgGeom<PARTS>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  const uint32_t patches = ring + G::STAGES * G::STAGE_BYTES;
  const uint32_t bar_full = patches + 8 * WG_PATCH_BYTES;   // used in the leader CTA
  const uint32_t bar_empty = bar_full + 8 * G::STAGES;      // one set per CTA
  const uint32_t bar_tfull = bar_empty + 8 * G::STAGES;     // [2] one set per CTA
  const uint32_t bar_tempty = bar_tfull + 16;               // [2] used in the leader CTA
  const uint32_t slot = bar_tempty + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + (slot - raw));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int group = blockIdx.x >> 1, n_groups = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < G::STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);      // the leader's byte count for both CTAs
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_tfull + 8 * s, 1);
      mbar_init(bar_tempty + 8 * s, 16);   // eight adding warps of either CTA
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    wg_fence_async();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_launch_before();
  dependents_may_start();
  const uint32_t lead_full = map_to_cta(bar_full, 0), lead_tempty = map_to_cta(bar_tempty, 0);
  auto raise_abort = [&]() {
    atomicOr(p.status, ST_TIMEOUT);
    *abort_flag = 1;
    st_cluster_u32(map_to_cta(slot + 4, rank ^ 1u), 1u);
  };

  // Registers: 384 threads x 168 at launch; 128 x (40 + 2 x 232) = 128 x 504 after the split.
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0) {
      if (lane == 0) {
        const uint64_t policy = l2_policy_evict_normal();
        const int half = p.bn >> 1;
        const uint32_t tx = 2 * (PARTS * WG_TILE_BYTES + (uint32_t)((half + 63) / 64) * (WG_ROWS * 128));
        WgRing r;
        bool ok = true;
        WgCursor c;
        for (bool more = c.start(p, group); more; more = c.next(p, n_groups)) {
          if (!(ok = mbar_wait<true>(bar_empty + 8 * r.s, r.ph ^ 1u, abort_flag))) break;
          const uint32_t full = lead_full + 8 * r.s, dst = ring + r.s * G::STAGE_BYTES;
          const int n = c.n0 + (int)rank * 128, k = c.k0 + (int)rank * half, m = c.st * WG_ROWS;
          if (rank == 0) mbar_expect_tx(bar_full + 8 * r.s, tx);
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            tma_load_3d<2>(dst + q * WG_TILE_BYTES, &tm_dy, full, n, m, q);
            tma_load_3d<2>(dst + q * WG_TILE_BYTES + WG_ROWS * 128, &tm_dy, full, n + 64, m, q);
          }
          tma_load_2d<2>(dst + PARTS * WG_TILE_BYTES, &tm_x, full, k, m, policy);
          if (half > 64) tma_load_2d<2>(dst + PARTS * WG_TILE_BYTES + WG_ROWS * 128, &tm_x, full, k + 64, m, policy);
          r.step<G::STAGES>();
        }
        if (!ok) raise_abort();
      }
      __syncwarp();
    } else if (warp == 1) {
      if (lane == 0 && rank == 0) {
        const uint32_t idesc = wg_idesc(p.bn), hi = smem_desc_hi(1024, 2u);
        WgRing r, t;
        bool ok = true;
        for (int item = group; item < p.tiles_n * p.tiles_k * p.splits && ok; item += n_groups) {
          const int st0 = (item % p.splits) * p.stages_per_split, st1 = min(p.stages, st0 + p.stages_per_split);
          for (int st = st0; st < st1 && ok;) {
            const int end = min(st1, st + G::CHUNK_STAGES);
            if (!(ok = mbar_wait<true>(bar_tempty + 8 * t.s, t.ph ^ 1u, abort_flag))) break;
            tc_fence_after();
            uint32_t acc = 0u;
            for (; st < end; ++st) {
              if (!(ok = mbar_wait<true>(bar_full + 8 * r.s, r.ph, abort_flag))) break;
              tc_fence_after();
              // a descriptor's start moves by 16 rows of 128 bytes per MMA; blocks of 64 columns lie 64 * 128 bytes apart
              const uint32_t a0 = smem_desc_lo(ring + r.s * G::STAGE_BYTES, WG_ROWS * 128);
              const uint32_t b0 = a0 + ((PARTS * WG_TILE_BYTES) >> 4);
#pragma unroll
              for (int i = PARTS - 1; i >= 0; --i) {
#pragma unroll
                for (int k = 0; k < WG_ROWS / 16; ++k) {
                  wg_mma(tmem_base + t.s * 256, smem_desc_join(a0 + i * (WG_TILE_BYTES >> 4) + k * 128, hi), smem_desc_join(b0 + k * 128, hi), idesc, acc);
                  acc = 1u;
                }
              }
              tc_commit<2>(bar_empty + 8 * r.s);
              r.step<G::STAGES>();
            }
            if (ok) tc_commit<2>(bar_tfull + 8 * t.s);
            t.step<2>();
          }
        }
        if (!ok) raise_abort();
      }
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int quad = warp & 3, side = (warp - 4) >> 2;
    const int chunks = p.bn >> 5, mine = side ? chunks >> 1 : (chunks + 1) >> 1, col_beg = side ? ((chunks + 1) >> 1) * 32 : 0;
    const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)col_beg;
    const uint32_t patch = patches + (uint32_t)(warp - 4) * WG_PATCH_BYTES;
    const int N = p.N, K = p.K;
    const bool whole = p.splits == 1;
    const bool vec = (K & 3) == 0 && (((uintptr_t)p.dw | (uintptr_t)p.gamma | (uintptr_t)p.beta) & 15) == 0;
    const bool add = whole && p.accumulate;
    const float* const gamma = whole ? p.gamma : nullptr;
    const float* const beta = whole ? p.beta : nullptr;
    WgRing t;
    bool ok = true;
    WgCursor c;
    for (int item = group; ok && c.start(p, item); item += n_groups) {
      const int n_warp = c.n0 + (int)rank * 128 + quad * 32;
      float db = 0.0f;
      if (whole && p.db_part && n_warp + lane < N) {
        for (int i = 0; i < p.db_parts; ++i) db += p.db_part[(size_t)i * N + n_warp + lane];
        if (p.db && c.k0 == 0 && side == 0) p.db[n_warp + lane] = p.accumulate ? p.db[n_warp + lane] + db : db;
        if (!beta) db = 0.0f;   // an infinite sum times no beta would be NaN
      }
      float acc[4][32];
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[g][j] = 0.0f;
      for (int st = c.st; st < c.st_end; st += G::CHUNK_STAGES) {
        ok = mbar_wait<true>(bar_tfull + 8 * t.s, t.ph, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (g < mine) {
            int r[32];
            tc_ld32(t_row + t.s * 256 + g * 32, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[g][j] = __fadd_rn(acc[g][j], __int_as_float(r[j]));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(lead_tempty + 8 * t.s);
        t.step<2>();
      }
      if (!ok || n_warp >= N) continue;
      // A lane holds 32 columns of one row; through the patch (16-byte words permuted so that neither side meets a bank
      // twice) eight lanes get the 128 bytes of a row, four rows at a time.
      const int r0 = lane >> 3, ch = lane & 7, k_warp = c.k0 + col_beg + ch * 4;
      float* out = (whole ? p.dw : p.part + (size_t)(item % p.splits) * N * K) + (size_t)(n_warp + r0) * K + k_warp;
      const size_t row_step = (size_t)4 * K;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int k = k_warp + g * 32;
        if (g >= mine || k - ch * 4 >= K) break;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          wg_sts16(patch + lane * 128 + ((j ^ (lane & 7)) << 4),
                   make_uint4(__float_as_uint(acc[g][4 * j]), __float_as_uint(acc[g][4 * j + 1]), __float_as_uint(acc[g][4 * j + 2]),
                              __float_as_uint(acc[g][4 * j + 3])));
        float4 ga = make_float4(1.0f, 1.0f, 1.0f, 1.0f), be = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (vec && k < K) {
          if (gamma) ga = __ldg(reinterpret_cast<const float4*>(gamma + k));
          if (beta) be = __ldg(reinterpret_cast<const float4*>(beta + k));
        }
        float* o = out + g * 32;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i, o += row_step) {
          const int r = i * 4 + r0;
          const uint4 u = wg_lds16(patch + r * 128 + ((ch ^ (r & 7)) << 4));
          float4 v = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
          const float dbr = __shfl_sync(0xffffffffu, db, r);
          if (n_warp + r >= N || k >= K) continue;
          if (vec) {
            v.x = fmaf(dbr, be.x, v.x * ga.x), v.y = fmaf(dbr, be.y, v.y * ga.y), v.z = fmaf(dbr, be.z, v.z * ga.z), v.w = fmaf(dbr, be.w, v.w * ga.w);
            if (add) {
              const float4 old = *reinterpret_cast<const float4*>(o);
              v.x += old.x, v.y += old.y, v.z += old.z, v.w += old.w;
            }
            *reinterpret_cast<float4*>(o) = v;
          } else {
            const float s[4] = {v.x, v.y, v.z, v.w};
#pragma unroll 1
            for (int j = 0; j < 4 && k + j < K; ++j) {
              float x = j == 0 ? s[0] : j == 1 ? s[1] : j == 2 ? s[2] : s[3];
              if (gamma) x *= __ldg(gamma + k + j);
              if (beta) x = fmaf(dbr, __ldg(beta + k + j), x);
              o[j] = add ? o[j] + x : x;
            }
          }
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) raise_abort();
  }

  // ---- teardown: everyone meets, copies in flight are waited for, tensor memory is released ----
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 2000000ull) {
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// dW from the partial sums of the splits, in order (splits = 0: the sum over no rows).
__global__ void __launch_bounds__(256) wgrad_join_kernel(const WgradArgs p, int splits) {
  wait_for_launch_before();
  const int n = blockIdx.x;
  float db = 0.0f;
  if (p.db_part)
    for (int i = 0; i < p.db_parts; ++i) db += p.db_part[(size_t)i * p.N + n];
  if (p.db && blockIdx.y == 0 && threadIdx.x == 0) p.db[n] = p.accumulate ? p.db[n] + db : db;
  const size_t plane = (size_t)p.N * p.K;
  for (int k = blockIdx.y * 256 + threadIdx.x; k < p.K; k += gridDim.y * 256) {
    const size_t at = (size_t)n * p.K + k;
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += p.part[s * plane + at];
    if (p.gamma) v *= __ldg(p.gamma + k);
    if (p.beta) v = fmaf(db, __ldg(p.beta + k), v);
    p.dw[at] = p.accumulate ? p.dw[at] + v : v;
  }
}

// ---- host side ----------------------------------------------------------------------------------
// How a weight gradient is cut.  Cost in clocks of an SM pair: an MMA of 16 rows takes max(bn / 2, 80) clocks (below 160
// columns the operands' loads count), an item 4000 on top (pipeline fill, epilogue), a join 6000, and partial sums go through L2 once
// each way (2000 bytes a clock).  The model was held against all tile widths and splits at ten shapes: its plan is the fastest or
// within 8 % at eight; 8192 x 2000 x 784 half takes 86.7 us where two splits of 256 columns take 79.5, 16384 x 1000 x 1000 bfloat16
// 66.6 where four take 55.9.  The slowest plans took 1.5 to 15 times as long.
// Only the splits depend on the room that the workspace has left for their partial sums: the rest grows with the rows, and one split
// needs none, so what is enough for a batch is enough for every smaller one, and for a device with another number of SMs.
struct WgPlan {
  int bn, tiles_n, tiles_k, splits, stages_per_split, stages, db_parts, dy_lanes;
  long long db_rows, ld_x, ld_parts;
  size_t x_bytes, parts_bytes, db_bytes, part_bytes;   // of the workspace, multiples of 256
};
// Parts of dY's column sums: more make the preparation wider, fewer the epilogue's additions.  With 8, 32, 64, 128 parts: 8192 x 2000 x 784 half
// 144, 97, 89, 88 us; 16384 x 4096 x 1024 bfloat16 157, 138, 146, 149; 2048 x 2000 x 2000 bfloat16 28.7, 25.2, 25.2, 25.3.
constexpr int WG_DB_PARTS = 64;
constexpr size_t WG_PART_CAP = (size_t)256 << 20;   // bytes of partial sums
inline WgPlan wg_plan(long long rows, int N, int K, int parts, bool split_dy, bool sums, int groups, size_t workspace_bytes) {
  WgPlan best{};
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  // dY's share of a block of the preparation: lanes over its columns, and four rows of each of the others at least.  Sums over
  // rows have at most 64 parts (narrow dY: 256), which the product's epilogue adds.
  best.dy_lanes = 32;
  while (best.dy_lanes > 1 && best.dy_lanes * 4 >= N) best.dy_lanes /= 2;
  const long long least = 8 * (256 / best.dy_lanes), most = !sums ? rows : best.dy_lanes < 32 ? 4 * WG_DB_PARTS : WG_DB_PARTS;
  long long gy = (rows + least - 1) / least;
  if (gy > most) gy = most;
  best.db_rows = gy ? (rows + gy - 1) / gy : 1;
  best.db_parts = (int)((rows + best.db_rows - 1) / best.db_rows);
  best.ld_x = ((long long)K + 15) / 16 * 16, best.ld_parts = ((long long)N + 7) / 8 * 8;
  best.x_bytes = up((size_t)rows * best.ld_x * 2);
  best.parts_bytes = split_dy ? up((size_t)parts * rows * best.ld_parts * 2) : 0;
  best.db_bytes = sums ? up((size_t)gy * N * sizeof(float)) : 0;
  const size_t fixed = best.x_bytes + best.parts_bytes + best.db_bytes, left = workspace_bytes > fixed ? workspace_bytes - fixed : 0;
  const size_t room = left < WG_PART_CAP ? left : WG_PART_CAP;
  const int stages = (int)((rows + WG_ROWS - 1) / WG_ROWS);
  const int tiles_n = (N + 255) / 256;
  double best_cost = 0.0;
  best.bn = 64, best.tiles_n = tiles_n, best.tiles_k = (K + 63) / 64, best.splits = 1;   // no rows: nothing is launched
  for (int bn = 256; bn >= 64; bn -= 64) {
    if (bn > 64 && bn - 64 >= K) continue;   // a narrower tile holds the whole width
    const int tiles_k = (K + bn - 1) / bn;
    const long long tiles = (long long)tiles_n * tiles_k;
    const double stage_clk = (double)parts * (WG_ROWS / 16) * (bn / 2 > 80 ? bn / 2 : 80);
    for (int want = 1; want <= 64 && want <= stages; ++want) {
      const int per = (stages + want - 1) / want, splits = (stages + per - 1) / per;
      if (splits != want) continue;
      if (splits > 1 && up((size_t)splits * N * K * sizeof(float)) > room) break;
      const long long items = tiles * splits, waves = (items + groups - 1) / groups;
      double cost = (double)waves * (per * stage_clk + 4000.0);
      if (splits > 1) cost += 6000.0 + (double)splits * N * K * 8.0 / 2000.0;
      if (best_cost == 0.0 || cost < best_cost) {
        best_cost = cost;
        best.bn = bn, best.tiles_k = tiles_k, best.splits = splits, best.stages_per_split = per, best.stages = stages;
      }
    }
  }
  best.part_bytes = best.splits > 1 ? up((size_t)best.splits * N * K * sizeof(float)) : 0;
  return best;
}

// bfloat16 [parts][rows][cols] as boxes of 64 columns x 64 rows (128-byte swizzle), zero outside; parts = 0: a plain 2-D map
inline ff_status wg_make_map(TcState& t, CUtensorMap* tm, const void* base, uint64_t cols, uint64_t rows, uint64_t parts, uint64_t pitch_bytes) {
  ff_status s = tc_init(t);
  if (s != FF_OK) return s;
  cuuint64_t dims[3] = {cols, rows, parts ? parts : 1}, strides[2] = {pitch_bytes, pitch_bytes * rows};
  cuuint32_t box[3] = {64, WG_ROWS, 1}, ones[3] = {1, 1, 1};
  const CUresult r = t.encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, parts ? 3 : 2, const_cast<void*>(base), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    snprintf(t.err, sizeof(t.err), "cuTensorMapEncodeTiled failed (%d): %llu x %llu, pitch %llu", (int)r, (unsigned long long)cols,
             (unsigned long long)rows, (unsigned long long)pitch_bytes);
    return FF_ERR_CUDA;
  }
  return FF_OK;
}

}  // namespace ffi8
