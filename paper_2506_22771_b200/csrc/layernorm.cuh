// Layer norm over the columns of a [rows, cols] tensor, forward and backward.
//   forward    mu = sum x / C, var = sum (x - mu)^2 / C, r = 1 / sqrt(var + eps), xh = (x - mu) r, y = xh gamma + beta
//   backward   g = dy gamma, dx = r (g - sum(g) / C - xh sum(g xh) / C) (+ dadd), dgamma = sum_rows dy xh, dbeta = sum_rows dy
// xh of the backward pass comes from an 8-bit checkpoint that the forward pass wrote, or from x, mu and r again.
// All statistics and sums are FP32; the variance is taken from the centred values (a row stays in registers), so an
// offset of the row costs no digits.  Sums over rows run in a fixed order (per CTA, then over CTAs): no atomics.
//
// HBM is the floor of both directions.  Forward with a checkpoint the instructions bound it (26 a value, 70 % of the issue slots:
// 32768 x 8192 bfloat16 270 us against 206 of HBM); backward, with 27 a value and 59 % of the slots, latencies of arithmetic and shared
// memory and the barrier of each step are not covered by the 16 computing warps of an SM (8192 x 2000 from the checkpoint with a residual
// 33 us against 18).  A team of TEAM threads owns a row, thread t the groups t, t + TEAM, ... of 8 columns.
// Forward, a team has one or two rows and many teams share an SM.  Backward, where a thread keeps sums for its columns over
// many rows, teams walk over the rows: rows of more than 512 columns whose bytes are multiples of 16 arrive in shared memory
// by bulk copies, a ring ahead of the team; others are loaded into registers one row ahead.
#pragma once
#include "ckpt8.cuh"
#include "gemm_tc.cuh"   // mbarrier wrappers with bounded waits

namespace ffi8 {

// A team's barrier; teams of up to a warp need none.  (Barrier 0 is the CTA's.)
template <int TEAM>
__device__ __forceinline__ void team_barrier(int team) {
  if (TEAM > 32) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(TEAM) : "memory");
}
// Sums of NV values (a power of two, at most 32) over the TEAM threads of a row; every one of them gets all.  Within a
// warp the values are folded while they are exchanged (NV / 2 + NV / 4 + ... shuffles instead of 5 NV).  TEAM > 32: `sm` holds
// NV floats for each of the team's warps; the caller gives another buffer to the next call, so that one barrier is enough.
template <int TEAM, int NV>
__device__ __forceinline__ void team_sums(float (&v)[NV], float* sm, int team) {
  if constexpr (TEAM < 32) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int m = TEAM / 2; m > 0; m >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], m);
  } else {
    constexpr int LANES = 32 / NV;   // lanes that end up with the same value
    const int lane = threadIdx.x & 31, mine = lane / LANES, l = lane % LANES;
    float w[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) w[k] = v[k];
#pragma unroll
    for (int s = NV / 2, m = 16; s > 0; s >>= 1, m >>= 1) {
      const bool hi = lane & m;
#pragma unroll
      for (int k = 0; k < s; ++k) {
        const float keep = hi ? w[k + s] : w[k], give = hi ? w[k] : w[k + s];
        w[k] = keep + __shfl_xor_sync(0xffffffffu, give, m);
      }
    }
    float x = w[0];
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
    if constexpr (TEAM > 32) {
      constexpr int W = TEAM / 32;
      const int warp = (threadIdx.x % TEAM) >> 5;
      if (l == 0) sm[mine * W + warp] = x;
      team_barrier<TEAM>(team);
      x = 0.0f;
#pragma unroll
      for (int i = 0; i < W; i += LANES)
        if (i + l < W) x += sm[mine * W + i + l];
#pragma unroll
      for (int m = LANES / 2; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = __shfl_sync(0xffffffffu, x, k * LANES);
  }
}
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float* sm, int team) {
  float a[1] = {v};
  team_sums<TEAM, 1>(a, sm, team);
  return a[0];
}
// Eight FP32 parameters of the group at `col` (`other` where there are none, or outside the row).  vec: p is 32-byte aligned;
// one load of 32 bytes a lane takes half the L1 cycles of two of 16 bytes, and L1 is what the forward pass runs into.
__device__ __forceinline__ void ln_params(const float* p, bool vec, int col, int n, float other, float (&g)[8]) {
  if (p && vec && n >= 8) {
    asm("ld.global.nc.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=f"(g[0]), "=f"(g[1]), "=f"(g[2]), "=f"(g[3]), "=f"(g[4]), "=f"(g[5]), "=f"(g[6]), "=f"(g[7])
        : "l"(p + col));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = (p && j < n) ? __ldg(p + col + j) : other;
  }
}
// The same from shared memory, where ln_stage_params has put them for all rows of the CTA.
__device__ __forceinline__ int ln_padded(int cols) { return (cols + 7) & ~7; }
// The first halves of the groups, then the second ones: lanes read 16 bytes each without meeting a bank twice.
__device__ __forceinline__ void ln_stage_params(const float* p, int cols, float other, float* to) {
  const int half = ln_padded(cols) / 2;
  for (int c = threadIdx.x; c < 2 * half; c += blockDim.x) to[(c & 4 ? half : 0) + (c >> 3) * 4 + (c & 3)] = (p && c < cols) ? __ldg(p + c) : other;
}
__device__ __forceinline__ void ln_staged(const float* from, int half, int group, float (&g)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(from + group * 4), b = *reinterpret_cast<const float4*>(from + half + group * 4);
  g[0] = a.x, g[1] = a.y, g[2] = a.z, g[3] = a.w, g[4] = b.x, g[5] = b.y, g[6] = b.z, g[7] = b.w;
}

// Rows on their way: a team's ring of slots in shared memory, one mbarrier each.  Thread 0 of the team issues the copies.
constexpr int LN_MAX_SLOTS = 8;
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
struct LnRing {
  uint32_t base, bar, slot_bytes;
  int slots, s = 0;
  uint32_t ph = 0;
  bool dead = false;   // a wait ran out: reported once, not waited for again (the barriers of the team stay matched)
  __device__ __forceinline__ uint32_t slot() const { return base + s * slot_bytes; }
  __device__ __forceinline__ uint32_t barrier() const { return bar + 8 * s; }
  __device__ __forceinline__ void wait(uint32_t* status) {
    uint32_t never = 0u;
    if (!dead && !mbar_wait<false>(barrier(), ph, &never)) {
      dead = true;
      atomicOr(status, ST_TIMEOUT);
    }
  }
  __device__ __forceinline__ void step() {
    if (++s == slots) s = 0, ph ^= 1u;
  }
  // Before a thread ends: where a wait ran out, copies may still be on their way into the CTA's shared memory.
  __device__ __forceinline__ void leave() const {
    if (!dead) return;
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 2000000ull) {
    }
  }
};
__device__ __forceinline__ void copy_word(uint32_t dst, const void* src, int bytes) {   // four bytes, zeros past `bytes`
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Room for a row's exponents and the words around them.
__host__ __device__ __forceinline__ uint32_t ln_exponent_bytes(int cols) { return (uint32_t)((cols + C8_BLOCK - 1) / C8_BLOCK + 3 + 3) / 4 * 4; }
template <typename T>
__device__ __forceinline__ Raw8<T> lds8(uint32_t src, int n) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
    r.w[i] = make_uint4(0u, 0u, 0u, 0u);
    if (n > i * (int)(16 / sizeof(T)))   // rows are whole 16-byte words here
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w) : "r"(src + 16 * i));
  }
  return r;
}

// a / n from 1 / n, corrected by its remainder a - q n, which one fused multiply-add gives exactly (the correction of a quotient that Markstein
// described in 1990), and 1 / sqrt(a) with a step of Newton's method, r + r (1 - a r r) / 2: each within an ulp, in a few operations
// that every thread of a row does.
__device__ __forceinline__ float quotient(float a, float n, float inv_n) {
  const float q = a * inv_n;
  return fabsf(q) < __uint_as_float(0x7f800000u) ? fmaf(fmaf(-q, n, a), inv_n, q) : q;   // an infinite sum stays one
}
__device__ __forceinline__ float inverse_root(float a) {
  const float r = rsqrtf(a);
  const float e = fmaf(-a * r, r, 1.0f);
  return a > 0.0f && a < __uint_as_float(0x7f800000u) ? fmaf(0.5f * r, e, r) : r;   // 0, Inf and NaN as they come
}

struct LnFwd {
  const void* x;
  const float* gamma;
  const float* beta;
  void* y;
  float* mean;
  float* rstd;
  long long ld_x, ld_y;
  long long rows;
  int cols;
  float eps;
  bool vec;   // gamma and beta are 32-byte aligned
  C8View c;
  C8Rounding round;
  uint32_t* status;
};

// y = xh g + b and the checkpoint of one group of normalised values (zeros outside the row).  y, q, e: where the row's group
// goes.  Called by all lanes of a warp (c8_encode shuffles).
template <typename T, int A>
__device__ __forceinline__ void ln_emit(const LnFwd& p, const C8Round& rd, const float (&xh)[8], const float (&g)[8], const float (&b)[8], T* y,
                                        int8_t* q, uint8_t* e, long long row, int col, int n) {
  if (p.y && n > 0) {
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = fmaf(xh[j], g[j], b[j]);
    store8<T, A>(y, pack8(o, T()), n);
  }
  if (p.c.q) {
    uint2 codes;
    const uint32_t x = c8_encode(xh, (uint32_t)row, (uint32_t)col, rd, codes);
    if (n > 0) {
      *reinterpret_cast<uint2*>(q) = codes;
      if ((col & (C8_BLOCK - 1)) == 0) {
        *e = (uint8_t)x;
        if (x == 255u) atomicOr(p.status, ST_NONFINITE);
      }
    }
  }
}

// Rows in registers: cols <= TEAM * 8 * V, R rows a team (their sums are reduced together and they share the loads of gamma
// and beta).  No loop over rows: four CTAs of 256 threads an SM hide each other's latencies better than a loop with the next rows
// on their way did (376 us against 288 at 32768 x 8192), in registers or through shared memory.
template <typename T, int TEAM, int V, int R, int A>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256, TEAM > 512 ? 1 : TEAM > 256 ? 2 : 4) ln_forward_kernel(const LnFwd p) {
  constexpr int TEAMS = (TEAM > 256 ? TEAM : 256) / TEAM;
  __shared__ float sm[2][TEAMS][TEAM > 32 ? R * (TEAM / 32) : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const long long row0 = ((long long)blockIdx.x * TEAMS + team) * R;
  if (TEAM >= 32 && row0 >= p.rows) return;   // the whole team
  float v[R][V][8], s[R];
  {
    Raw8<T> raw[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool live = row0 + r < p.rows;
      const T* x = static_cast<const T*>(p.x) + (live ? row0 + r : 0) * p.ld_x + t * 8;
#pragma unroll
      for (int i = 0; i < V; ++i) raw[r][i] = load8<T, A>(x + i * TEAM * 8, live ? p.cols - (i * TEAM + t) * 8 : 0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        unpack8(raw[r][i], v[r][i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[r] += v[r][i][j];
      }
    }
  }
  const float n = (float)p.cols, inv_n = __frcp_rn(n);
  team_sums<TEAM, R>(s, sm[0][team], team);
  float mean[R], rstd[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    mean[r] = quotient(s[r], n, inv_n);
    s[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int m = p.cols - (i * TEAM + t) * 8;
      if (m >= 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[r][i][j] -= mean[r];
          s[r] = fmaf(v[r][i][j], v[r][i][j], s[r]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[r][i][j] = j < m ? v[r][i][j] - mean[r] : 0.0f;
          s[r] = fmaf(v[r][i][j], v[r][i][j], s[r]);
        }
      }
    }
  }
  team_sums<TEAM, R>(s, sm[1][team], team);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    rstd[r] = inverse_root(quotient(s[r], n, inv_n) + p.eps);
    if (t == 0 && row0 + r < p.rows) {
      if (p.mean) p.mean[row0 + r] = mean[r];
      if (p.rstd) p.rstd[row0 + r] = rstd[r];
    }
  }
  const C8Round rd = c8_round(p.round);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int col = (i * TEAM + t) * 8;
    float g[8], b[8];
    ln_params(p.gamma, p.vec, col, p.cols - col, 1.0f, g);
    ln_params(p.beta, p.vec, col, p.cols - col, 0.0f, b);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const long long row = row0 + r;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[r][i][j] *= rstd[r];
      ln_emit<T, A>(p, rd, v[r][i], g, b, static_cast<T*>(p.y) + row * p.ld_y + col, p.c.q + row * p.c.ld_q + col,
                    p.c.e + row * p.c.ld_e + col / C8_BLOCK, row, col, row < p.rows ? p.cols - col : 0);
    }
  }
}

// Any row length: a CTA per row, the row read three times (it stays in L2 between the passes).
constexpr int LN_LONG_THREADS = 512;
template <typename T, int A>
__global__ void __launch_bounds__(LN_LONG_THREADS) ln_forward_long_kernel(const LnFwd p) {
  __shared__ float sm[2][32];
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
  const int span = (p.cols + LN_LONG_THREADS * 8 - 1) / (LN_LONG_THREADS * 8) * (LN_LONG_THREADS * 8);
  float s = 0.0f, v[8];
  for (int col = threadIdx.x * 8; col < span; col += LN_LONG_THREADS * 8) {
    unpack8(load8<T, A>(x + col, p.cols - col), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j];
  }
  const float n = (float)p.cols;
  const float mean = __fdiv_rn(team_sum<LN_LONG_THREADS>(s, sm[0], 0), n);
  float ss = 0.0f;
  for (int col = threadIdx.x * 8; col < span; col += LN_LONG_THREADS * 8) {
    unpack8(load8<T, A>(x + col, p.cols - col), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = col + j < p.cols ? v[j] - mean : 0.0f;
      ss = fmaf(d, d, ss);
    }
  }
  const float var = __fdiv_rn(team_sum<LN_LONG_THREADS>(ss, sm[1], 0), n);
  const float rstd = __frsqrt_rn(var + p.eps);
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
  const C8Round rd = c8_round(p.round);
  for (int col = threadIdx.x * 8; col < span; col += LN_LONG_THREADS * 8) {
    unpack8(load8<T, A>(x + col, p.cols - col), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = col + j < p.cols ? (v[j] - mean) * rstd : 0.0f;
    float g[8], b[8];
    ln_params(p.gamma, p.vec, col, p.cols - col, 1.0f, g);
    ln_params(p.beta, p.vec, col, p.cols - col, 0.0f, b);
    ln_emit<T, A>(p, rd, v, g, b, static_cast<T*>(p.y) + row * p.ld_y + col, p.c.q + row * p.c.ld_q + col, p.c.e + row * p.c.ld_e + col / C8_BLOCK, row, col,
                  p.cols - col);
  }
}

// ---- backward ---------------------------------------------------------------------------------
struct LnBwd {
  const void* dy;
  const void* dadd;   // nullable: added to dx (the gradient that reaches x past the norm)
  const void* x;      // CK = false: x and mean; CK = true: the checkpoint c
  const float* mean;
  const float* rstd;
  const float* gamma;
  void* dx;           // nullable
  long long ld_dy, ld_dadd, ld_x, ld_dx;
  long long rows;
  int cols;
  bool vec;           // gamma is 32-byte aligned
  int slots;          // ring: steps of a team in flight
  uint32_t* status;
  C8View c;
  float* part;        // [CTAs][2][cols] sums of the rows a CTA took: dgamma, dbeta; NULL: neither is wanted
};

// Normalised values of a group.
template <typename T, bool CK, int A>
struct LnSource {
  Raw8<T> raw;
  uint2 codes;
  uint32_t e;
  __device__ __forceinline__ void load(const LnBwd& p, long long row, int col, int n) {
    if (CK) {
      codes = make_uint2(0u, 0u), e = 0u;
      if (n > 0) {
        codes = __ldcs(reinterpret_cast<const uint2*>(p.c.q + row * p.c.ld_q + col));
        e = p.c.e[row * p.c.ld_e + col / C8_BLOCK];
      }
    } else {
      raw = load8<T, A>(static_cast<const T*>(p.x) + row * p.ld_x + col, n);
    }
  }
  __device__ __forceinline__ void values(float (&xh)[8], float mean, float rstd) const {
    if (CK) {
      c8_decode(codes, e, xh);
    } else {
      unpack8(raw, xh);
#pragma unroll
      for (int j = 0; j < 8; ++j) xh[j] = (xh[j] - mean) * rstd;
    }
  }
};

// The sums over rows that a CTA's teams hold, into its part of the workspace: thread t has columns (i * TEAM + t) * 8 ...
// The upper half of the teams hands its sums to the lower half until one is left.  `acc`: ln_acc_floats().
template <int TEAM, int TEAMS, int V>
__host__ __device__ constexpr int ln_acc_floats() {
  return TEAMS > 1 ? TEAMS * TEAM * 8 * V : 1;
}
template <int TEAM, int TEAMS, int V>
__device__ __forceinline__ void ln_leave_sums(const LnBwd& p, float (&dg)[V][8], float (&db)[V][8], int t, int team, float* acc) {
  constexpr int COLS = TEAM * 8 * V;
  auto all = [] { asm volatile("bar.sync 0, %0;" ::"n"(TEAM * TEAMS) : "memory"); };   // the teams' threads
#pragma unroll
  for (int h = TEAMS / 2; h > 0; h >>= 1) {
    float* const a = acc + (team < h ? team : team - h) * 2 * COLS;
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      if (step == 0 ? team >= h && team < 2 * h : team < h) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int at = (i * 8 + j) * TEAM + t;
            if (step == 0)
              a[at] = dg[i][j], a[COLS + at] = db[i][j];
            else
              dg[i][j] += a[at], db[i][j] += a[COLS + at];
          }
      }
      all();
    }
  }
  if (team) return;
  float* part = p.part + (size_t)blockIdx.x * 2 * p.cols;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = (i * TEAM + t) * 8 + j;
      if (col < p.cols) part[col] = dg[i][j], part[p.cols + col] = db[i][j];
    }
}

// Rows through a ring of bulk copies: cols <= TEAM * 8 * V.  A step is R rows of a team, whose sums are reduced together; the
// sums over the rows stay in registers, gamma is in shared memory.  One more warp asks for the rows, as far ahead as the
// slots reach; done by the teams' own first warps, the others waited for them (220 us against 168 at 65536 x 2000).
template <typename T, int TEAM, int V, int R, bool CK>
__global__ void __launch_bounds__((TEAM > 256 ? TEAM : 256) + 32, TEAM > 256 ? 1 : 2) ln_backward_ring_kernel(const LnBwd p) {
  constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM;
  __shared__ float red[2][TEAMS][TEAM > 32 ? 2 * R * (TEAM / 32) : 1];
  __shared__ uint64_t bars[2][TEAMS * LN_MAX_SLOTS];   // full, empty
  __shared__ float acc[ln_acc_floats<TEAM, TEAMS, V>()];
  extern __shared__ __align__(128) uint8_t ln_ring[];
  dependents_may_start();
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM, lane = threadIdx.x & 31;
  float* const sg = reinterpret_cast<float*>(ln_ring);
  // a slot holds R rows of dY, then of codes (or x), then of dAdd, the codes' exponents, rstd and mean
  const uint32_t dy_bytes = (uint32_t)p.cols * sizeof(T), x_bytes = CK ? (uint32_t)(p.cols + 15) / 16 * 16 : dy_bytes;
  const uint32_t x_off = R * dy_bytes, add_off = x_off + R * x_bytes, e_off = add_off + (p.dadd ? R * dy_bytes : 0u);
  const uint32_t e_bytes = CK ? ln_exponent_bytes(p.cols) : 0u, stat_off = e_off + R * e_bytes;
  const uint32_t slot_bytes = (stat_off + R * 8 + 15) / 16 * 16, ring0 = smem_u32(sg + ln_padded(p.cols));
  const long long step = (long long)gridDim.x * (TEAMS * R);
  if (threadIdx.x == 0) {
    for (int i = 0; i < TEAMS * LN_MAX_SLOTS; ++i) {
      mbar_init(smem_u32(&bars[0][i]), 1 + 32);      // the byte count, a warp's words
      mbar_init(smem_u32(&bars[1][i]), TEAM / 32);   // the team's warps
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  ln_stage_params(p.gamma, p.cols, 1.0f, sg);
  __syncthreads();

  if (threadIdx.x >= THREADS) {   // the warp that asks for rows
    const int nb = (p.cols + C8_BLOCK - 1) / C8_BLOCK;
    LnRing empty;
    empty.slots = p.slots, empty.slot_bytes = 0, empty.base = 0, empty.ph = 1u;
    bool going = true;   // no copies into a slot that was not given back: the teams' waits for them run out, too
    for (long long base = (long long)blockIdx.x * (TEAMS * R); base < p.rows && going; base += step) {
      for (int q = 0; q < TEAMS; ++q) {
        const long long row0 = base + q * R;
        if (row0 >= p.rows) break;
        empty.bar = smem_u32(bars[1]) + q * LN_MAX_SLOTS * 8;
        empty.wait(p.status);
        if (!(going = !__any_sync(0xffffffffu, empty.dead))) break;
        const uint32_t slot = ring0 + (q * p.slots + empty.s) * slot_bytes, bar = smem_u32(bars[0]) + (q * LN_MAX_SLOTS + empty.s) * 8;
        const int live = p.rows - row0 < R ? (int)(p.rows - row0) : R;
        if (lane == 0) mbar_expect_tx(bar, live * (dy_bytes + x_bytes + (p.dadd ? dy_bytes : 0u)));
        for (int r = 0; r < live; ++r) {
          const long long row = row0 + r;
          if (lane == 0) {
            bulk_load(slot + r * dy_bytes, static_cast<const T*>(p.dy) + row * p.ld_dy, dy_bytes, bar);
            bulk_load(slot + x_off + r * x_bytes, CK ? static_cast<const void*>(p.c.q + row * p.c.ld_q) : static_cast<const T*>(p.x) + row * p.ld_x,
                      x_bytes, bar);
            if (p.dadd) bulk_load(slot + add_off + r * dy_bytes, static_cast<const T*>(p.dadd) + row * p.ld_dadd, dy_bytes, bar);
            copy_word(slot + stat_off + r * 8, p.rstd + row, 4);
            if (!CK) copy_word(slot + stat_off + r * 8 + 4, p.mean + row, 4);
          }
          if (CK) {   // exponents start at any byte: the words around a row's, the last one only as far as the tensor goes
            const uint8_t* const from = p.c.e + row * p.c.ld_e;
            const int shift = (int)(reinterpret_cast<uintptr_t>(from) & 3), bytes = shift + nb;
            for (int w = lane * 4; w < bytes; w += 128)
              copy_word(slot + e_off + r * e_bytes + w, from - shift + w, row == p.rows - 1 && w + 4 > bytes ? bytes - w : 4);
          }
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
      }
      empty.step();
    }
    empty.leave();
    return;
  }

  LnRing ring;
  ring.slots = p.slots, ring.slot_bytes = slot_bytes, ring.base = ring0 + team * p.slots * slot_bytes;
  ring.bar = smem_u32(bars[0]) + team * LN_MAX_SLOTS * 8;
  const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
  float dg[V][8], db[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = db[i][j] = 0.0f;
  int buf = 0;
  for (long long first = ((long long)blockIdx.x * TEAMS + team) * R; first < p.rows; first += step, buf ^= 1) {
    ring.wait(p.status);
    const uint32_t slot = ring.slot(), done = smem_u32(bars[1]) + (team * LN_MAX_SLOTS + ring.s) * 8;
    float sum[2 * R], d[R][V][8], xh[R][V][8], rs[R];
#pragma unroll
    for (int k = 0; k < 2 * R; ++k) sum[k] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rs[r] = 0.0f;
      if (first + r >= p.rows) continue;
      float mu = 0.0f;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(rs[r]) : "r"(slot + stat_off + r * 8));
      if (!CK) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(mu) : "r"(slot + stat_off + r * 8 + 4));
      const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(p.c.e) + (uintptr_t)((first + r) * p.c.ld_e)) & 3u;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int group = i * TEAM + t, n = p.cols - group * 8;
        if (n <= 0) continue;
        unpack8(lds8<T>(slot + r * dy_bytes + group * 8 * sizeof(T), n), d[r][i]);
        if (CK) {
          uint32_t e;
          uint2 codes;
          asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e) : "r"(slot + e_off + r * e_bytes + shift + group / 4));
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(codes.x), "=r"(codes.y) : "r"(slot + x_off + r * x_bytes + group * 8));
          c8_decode(codes, e, xh[r][i]);
        } else {
          unpack8(lds8<T>(slot + x_off + r * x_bytes + group * 8 * sizeof(T), n), xh[r][i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) xh[r][i][j] = (xh[r][i][j] - mu) * rs[r];
        }
        if (n < 8) {   // padding of the codes; (0 - mean) rstd
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j >= n) xh[r][i][j] = 0.0f;
        }
        float g[8];
        ln_staged(sg, ln_padded(p.cols) / 2, group, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float gy = d[r][i][j] * g[j];
          sum[2 * r] += gy;
          sum[2 * r + 1] = fmaf(gy, xh[r][i][j], sum[2 * r + 1]);
          dg[i][j] = fmaf(d[r][i][j], xh[r][i][j], dg[i][j]);
          db[i][j] += d[r][i][j];
          d[r][i][j] = gy;
        }
      }
    }
    if (p.dx) {
      team_sums<TEAM, 2 * R>(sum, red[buf][team], team);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const long long row = first + r;
        if (row >= p.rows) continue;
        const float c1 = -sum[2 * r] * inv_n * rs[r], c2 = -sum[2 * r + 1] * inv_n * rs[r];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int group = i * TEAM + t, n = p.cols - group * 8;
          if (n <= 0) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) d[r][i][j] = fmaf(xh[r][i][j], c2, fmaf(d[r][i][j], rs[r], c1));
          if (p.dadd) {
            float b[8];
            unpack8(lds8<T>(slot + add_off + r * dy_bytes + group * 8 * sizeof(T), n), b);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[r][i][j] += b[j];
          }
          store8<T, 16>(static_cast<T*>(p.dx) + row * p.ld_dx + group * 8, pack8(d[r][i], T()), n);
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(done);
    ring.step();
  }
  ring.leave();
  if (p.part) ln_leave_sums<TEAM, TEAMS, V>(p, dg, db, t, team, acc);
}

// Rows that bulk copies cannot address (or short ones), in registers: cols <= TEAM * 8 * V.  A team walks over its rows with the
// stride of the grid, the next row on its way while it computes this one.  gamma and the sums over its rows of dy xh and
// dy for a thread's columns stay in registers.
template <typename T, int TEAM, int V, bool CK, int A>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256, TEAM <= 256 ? 2 : 1) ln_backward_kernel(const LnBwd p) {
  constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM, PER_WARP = TEAM < 32 ? 32 / TEAM : 1;
  __shared__ float red[2][TEAMS][TEAM > 32 ? 2 * (TEAM / 32) : 1];
  __shared__ float acc[ln_acc_floats<TEAM, TEAMS, V>()];
  dependents_may_start();
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM, sub = team % PER_WARP;
  const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
  float dg[V][8], db[V][8], g[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    ln_params(p.gamma, p.vec, (i * TEAM + t) * 8, p.cols - (i * TEAM + t) * 8, 1.0f, g[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = db[i][j] = 0.0f;
  }
  Raw8<T> dy[V], add[V];
  LnSource<T, CK, A> src[V];
  float mean, rstd;
  auto fetch = [&](long long row) {
    const bool live = row < p.rows;
    if (!live) row = 0;
    mean = (!CK && live) ? p.mean[row] : 0.0f;
    rstd = live ? p.rstd[row] : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int col = (i * TEAM + t) * 8, n = live ? p.cols - col : 0;
      dy[i] = load8<T, A>(static_cast<const T*>(p.dy) + row * p.ld_dy + t * 8 + i * TEAM * 8, n);
      src[i].load(p, row, col, n);
      if (p.dadd) add[i] = load8<T, A>(static_cast<const T*>(p.dadd) + row * p.ld_dadd + t * 8 + i * TEAM * 8, n);
    }
  };
  const long long step = (long long)gridDim.x * TEAMS;
  long long first = (long long)blockIdx.x * TEAMS + team - sub;   // first row of the warp's teams: its loop is the warp's
  int buf = 0;
  fetch(first + sub);
  for (; first < p.rows; first += step, buf ^= 1) {
    const long long row = first + sub;
    const bool live = row < p.rows;
    float d[V][8], xh[V][8], sum[2] = {0.0f, 0.0f};
    const float rs = rstd;
    Raw8<T> a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int n = live ? p.cols - (i * TEAM + t) * 8 : 0;
      unpack8(dy[i], d[i]);
      src[i].values(xh[i], mean, rstd);
      a[i] = add[i];
      if (n < 8) {   // padding of the codes; (0 - mean) rstd
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j >= n) xh[i][j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {   // dy is zero outside the row
        const float gy = d[i][j] * g[i][j];
        sum[0] += gy;
        sum[1] = fmaf(gy, xh[i][j], sum[1]);
        dg[i][j] = fmaf(d[i][j], xh[i][j], dg[i][j]);
        db[i][j] += d[i][j];
        d[i][j] = gy;
      }
    }
    fetch(row + step);
    if (!p.dx) continue;
    team_sums<TEAM, 2>(sum, red[buf][team], team);
    if (!live) continue;
    const float c1 = -sum[0] * inv_n * rs, c2 = -sum[1] * inv_n * rs;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int n = p.cols - (i * TEAM + t) * 8;
      if (n <= 0) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[i][j] = fmaf(xh[i][j], c2, fmaf(d[i][j], rs, c1));
      if (p.dadd) {
        float b[8];
        unpack8(a[i], b);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[i][j] += b[j];
      }
      store8<T, A>(static_cast<T*>(p.dx) + row * p.ld_dx + t * 8 + i * TEAM * 8, pack8(d[i], T()), n);
    }
  }
  if (p.part) ln_leave_sums<TEAM, TEAMS, V>(p, dg, db, t, team, acc);
}

// Any row length: a CTA per row reads it twice; the sums over rows are ln_column_sums_kernel's, which runs before this one.
template <typename T, bool CK, int A>
__global__ void __launch_bounds__(LN_LONG_THREADS) ln_backward_long_kernel(const LnBwd p) {
  __shared__ float sm[2][32];
  dependents_may_start();
  const long long row = blockIdx.x;
  const float mean = CK ? 0.0f : p.mean[row], rstd = p.rstd[row];
  const T* dy = static_cast<const T*>(p.dy) + row * p.ld_dy;
  float s1 = 0.0f, s2 = 0.0f, d[8], xh[8], g[8];
  LnSource<T, CK, A> src;
  for (int col = threadIdx.x * 8; col < p.cols; col += LN_LONG_THREADS * 8) {
    const int n = p.cols - col;
    unpack8(load8<T, A>(dy + col, n), d);
    src.load(p, row, col, n);
    src.values(xh, mean, rstd);
    ln_params(p.gamma, p.vec, col, n, 1.0f, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gy = d[j] * g[j];
      s1 += gy;
      s2 = fmaf(gy, j < n ? xh[j] : 0.0f, s2);
    }
  }
  const float inv_n = __fdiv_rn(1.0f, (float)p.cols);
  const float c1 = team_sum<LN_LONG_THREADS>(s1, sm[0], 0) * inv_n, c2 = team_sum<LN_LONG_THREADS>(s2, sm[1], 0) * inv_n;
  for (int col = threadIdx.x * 8; col < p.cols; col += LN_LONG_THREADS * 8) {
    const int n = p.cols - col;
    unpack8(load8<T, A>(dy + col, n), d);
    src.load(p, row, col, n);
    src.values(xh, mean, rstd);
    ln_params(p.gamma, p.vec, col, n, 1.0f, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = rstd * fmaf(-xh[j], c2, fmaf(d[j], g[j], -c1));
    if (p.dadd) {
      float a[8];
      unpack8(load8<T, A>(static_cast<const T*>(p.dadd) + row * p.ld_dadd + col, n), a);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] += a[j];
    }
    store8<T, A>(static_cast<T*>(p.dx) + row * p.ld_dx + col, pack8(d, T()), n);
  }
}

// dgamma / dbeta sums of rows [blockIdx.y * rows_per, ...) for 32 groups of columns; 8 row lanes per group.
template <typename T, bool CK, int A>
__global__ void __launch_bounds__(256) ln_column_sums_kernel(const LnBwd p, long long rows_per) {
  __shared__ float acc[8][2][32 * 8];
  dependents_may_start();
  const int gx = threadIdx.x & 31, lanes = threadIdx.x >> 5;
  const int col = (blockIdx.x * 32 + gx) * 8, n = p.cols - col;
  float dg[8], db[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) dg[j] = db[j] = 0.0f;
  const long long r0 = blockIdx.y * rows_per, r1 = min(r0 + rows_per, p.rows);
  for (long long row = r0 + lanes; row < r1; row += 8) {
    float d[8], xh[8];
    LnSource<T, CK, A> src;
    unpack8(load8<T, A>(static_cast<const T*>(p.dy) + row * p.ld_dy + col, n), d);
    src.load(p, row, col, n);
    src.values(xh, CK ? 0.0f : p.mean[row], p.rstd[row]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dg[j] = fmaf(d[j], j < n ? xh[j] : 0.0f, dg[j]);
      db[j] += d[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[lanes][0][gx * 8 + j] = dg[j], acc[lanes][1][gx * 8 + j] = db[j];
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c < p.cols) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float s = 0.0f;
#pragma unroll
      for (int l = 0; l < 8; ++l) s += acc[l][k][threadIdx.x];
      p.part[((size_t)blockIdx.y * 2 + k) * p.cols + c] = s;
    }
  }
}

// out[k][c] (+)= sum over parts of part[.][k][c], k = 0: dgamma, 1: dbeta.  32 columns per CTA, 16 lanes over the parts.
__global__ void __launch_bounds__(512) ln_finish_kernel(const float* __restrict__ part, int parts, int cols, float* __restrict__ dgamma,
                                                        float* __restrict__ dbeta, int accumulate) {
  __shared__ float sm[16][33];
  wait_for_launch_before();
  const int cx = threadIdx.x & 31, ly = threadIdx.x >> 5;
  const int flat = blockIdx.x * 32 + cx;   // over [2][cols]
  float s = 0.0f;
  if (flat < 2 * cols) {
#pragma unroll 8
    for (int b = ly; b < parts; b += 16) s += part[(size_t)b * 2 * cols + flat];
  }
  sm[ly][cx] = s;
  __syncthreads();
  if (ly == 0 && flat < 2 * cols) {
    s = 0.0f;
#pragma unroll
    for (int l = 0; l < 16; ++l) s += sm[l][cx];
    float* out = flat < cols ? dgamma : dbeta;
    if (out) {
      out += flat < cols ? flat : flat - cols;
      *out = accumulate ? *out + s : s;
    }
  }
}

}  // namespace ffi8
