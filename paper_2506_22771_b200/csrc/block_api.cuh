// Host side of the operators of a locally back-propagated block (declared in include/ffint8.h): layer norm, 8-bit
// activation checkpoints, activations and the weight gradient that read them.  Included by ffint8_api.cu, whose context,
// error and launch helpers it uses.
#pragma once
#include "ckpt8.cuh"
#include "ckpt_wgrad.cuh"
#include "layernorm.cuh"

namespace {

inline bool known_dtype(int d) { return d == FF_F32 || d == FF_BF16 || d == FF_F16; }
inline size_t dtype_bytes(int d) { return d == FF_F32 ? 4 : 2; }
template <class F>
ff_status for_dtype(int d, F f) {  // f(T()) for the tensor's type
  if (d == FF_F32) return f(float());
  if (d == FF_BF16) return f(__nv_bfloat16());
  return f(__half());
}
template <class F>
ff_status for_flag(bool b, F f) {
  return b ? f(std::true_type()) : f(std::false_type());
}

// A launch that may start before the launch before it on the stream has ended; its kernel calls wait_for_launch_before().
template <class K, class... Args>
ff_status launch_after(ff_ctx* ctx, K kern, dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at, cfg.numAttrs = 1;
  FF_CUDA(ctx, cudaLaunchKernelEx(&cfg, kern, args...));
  FF_LAUNCH_CHECK(ctx);
  return FF_OK;
}

// What an earlier launch of a kernel found out about its residency (0: nothing yet).
inline int known_resident(const ff_ctx* ctx, const void* kern, size_t smem) {
  for (const auto& r : ctx->resident)
    if (r.kern == kern && r.smem == smem) return r.n;
  return 0;
}
inline void keep_resident(ff_ctx* ctx, const void* kern, size_t smem, int n) {
  auto& r = ctx->resident[ctx->resident_next];
  ctx->resident_next = (ctx->resident_next + 1) % (int)(sizeof(ctx->resident) / sizeof(ctx->resident[0]));
  r.kern = kern, r.smem = smem, r.n = n;
}

constexpr long long BLOCK_MAX_ROWS = (1LL << 31) - 1;

// Sizes that every operator here shares.  An element offset may pass 32 bits; the number of 8-value groups may not.
ff_status check_extent(ff_ctx* ctx, int64_t rows, int64_t cols, int dtype, int round) {
  if (!known_dtype(dtype)) return fail(ctx, FF_ERR_ARG, "unknown dtype");
  if (round & ~(FF_ROUND_STOCHASTIC | FF_ROUND_KEEP_SIGN)) return fail(ctx, FF_ERR_ARG, "unknown rounding mode");
  if (rows < 0) return fail(ctx, FF_ERR_ARG, "rows must not be negative");
  if (cols <= 0) return fail(ctx, FF_ERR_ARG, "cols must be positive");
  if (rows > BLOCK_MAX_ROWS || cols > (1LL << 24)) return fail(ctx, FF_ERR_RANGE, "more than 2^31 - 1 rows or 2^24 columns");
  const long long groups = (cols + C8_BLOCK - 1) / C8_BLOCK * 4;
  if (rows && rows > ((1LL << 31) - 1 - (1LL << 16)) / groups) return fail(ctx, FF_ERR_RANGE, "tensor has too many values");
  if ((round & FF_ROUND_STOCHASTIC) && rows * cols >= (1LL << 32))
    return fail(ctx, FF_ERR_RANGE, "stochastic rounding counts 2^32 values");
  return FF_OK;
}
// A [rows, cols] tensor of the operator's type (`what` names it in the message).
ff_status check_tensor(ff_ctx* ctx, const void* p, int64_t ld, int64_t cols, int dtype, const char* what) {
  if (!p) return fail(ctx, FF_ERR_ARG, "%s is NULL", what);
  if (ld < cols) return fail(ctx, FF_ERR_ARG, "row pitch of %s is smaller than cols", what);
  if (reinterpret_cast<uintptr_t>(p) % dtype_bytes(dtype)) return fail(ctx, FF_ERR_ALIGN, "%s is not aligned to its type", what);
  return FF_OK;
}
ff_status check_floats(ff_ctx* ctx, const void* p, const char* what) {
  if (reinterpret_cast<uintptr_t>(p) & 3) return fail(ctx, FF_ERR_ALIGN, "%s is not aligned to its type", what);
  return FF_OK;
}
ff_status check_ckpt(ff_ctx* ctx, const ff_ckpt8& c, int64_t cols) {
  if (!c.q || !c.e) return fail(ctx, FF_ERR_ARG, "a checkpoint needs q and e");
  if (c.ld_q < cols || c.ld_q % 16) return fail(ctx, FF_ERR_ARG, "ld_q must be >= cols and a multiple of 16");
  if (c.ld_e < (cols + C8_BLOCK - 1) / C8_BLOCK) return fail(ctx, FF_ERR_ARG, "ld_e must be >= the number of blocks of a row");
  if (!aligned16(c.q)) return fail(ctx, FF_ERR_ALIGN, "a checkpoint's q is not 16-byte aligned");
  return FF_OK;
}
// Alignment of a tensor's rows in bytes, at most 16: the widest access to its groups of 8 (see load8).  NULL: no tensor.
inline unsigned row_alignment(const void* p, int64_t ld, int dtype) {
  if (!p) return 16;
  const uintptr_t v = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * dtype_bytes(dtype));
  return v & 15 ? v & 7 ? (unsigned)dtype_bytes(dtype) : 8 : 16;
}
template <typename T, class F>
ff_status for_alignment(unsigned a, F f) {
  if (a >= 16) return f(std::integral_constant<int, 16>());
  if (a == 8) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, (int)sizeof(T)>());
}
inline unsigned least(unsigned a, unsigned b) { return a < b ? a : b; }

inline C8View view(const ff_ckpt8& c) { return C8View{c.q, c.e, c.ld_q, c.ld_e}; }
inline C8Rounding rounding(int round, uint64_t seed, int role, int index, uint64_t step, int64_t cols) {
  return C8Rounding{round & FF_ROUND_STOCHASTIC, round & FF_ROUND_KEEP_SIGN, make_key_spec(seed, role, index, nullptr).s1, step, (uint32_t)cols};
}
inline int group_blocks(const GroupList& g) { return (int)((g.total + C8_THREADS * C8_UNROLL - 1) / (C8_THREADS * C8_UNROLL)); }

// ---- layer norm -----------------------------------------------------------------------------
constexpr int LN_MAX_COLS = 8192;       // longest row that a team keeps in registers
// Most CTAs of a backward pass that sums over rows, four an SM of 148.  What it limits is the workspace, not the kernels: one or two CTAs an
// SM are resident (8192 x 2000 bfloat16 with at most 148 parts 37.9 us, with 296 to 1184 30.5; 60000 x 500 half 102 and 68).
constexpr int LN_MAX_PARTS = 592;
inline size_t ln_part_bytes(int cols, int64_t rows) {   // a CTA takes at least one row
  return (size_t)(rows < LN_MAX_PARTS ? rows : LN_MAX_PARTS) * 2 * cols * sizeof(float);
}

ff_status check_ln(ff_ctx* ctx, const ff_layernorm_desc* d, const ff_layernorm_bufs* b, int64_t rows) {
  if (!d || !b) return fail(ctx, FF_ERR_ARG, "layer norm descriptor or buffer struct is NULL");
  ff_status s = check_extent(ctx, rows, d->cols, d->dtype, d->round);
  if (s != FF_OK) return s;
  if (!(d->eps >= 0.0f)) return fail(ctx, FF_ERR_ARG, "eps must be >= 0");
  const struct {
    const void* p;
    const char* name;
  } f[] = {{b->gamma, "gamma"}, {b->beta, "beta"}, {b->mean, "mean"}, {b->rstd, "rstd"}, {b->dgamma, "dgamma"}, {b->dbeta, "dbeta"}};
  for (const auto& x : f)
    if ((s = check_floats(ctx, x.p, x.name)) != FF_OK) return s;
  return FF_OK;
}

// CTAs of a row loop that stay resident together, with smem bytes of dynamic shared memory each.
template <class K>
ff_status resident_ctas(ff_ctx* ctx, K kern, int threads, size_t smem, int* n) {
  if ((*n = known_resident(ctx, reinterpret_cast<const void*>(kern), smem)) > 0) return FF_OK;
  int per_sm = 0;
  if (smem > 0) {   // the limit belongs to the kernel, whose other launches may need more: all that a CTA can have
    cudaFuncAttributes fa;
    FF_CUDA(ctx, cudaFuncGetAttributes(&fa, kern));
    FF_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)fa.sharedSizeBytes));
  }
  FF_CUDA(ctx, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, smem));
  *n = (per_sm > 0 ? per_sm : 1) * ctx->sm_count;
  keep_resident(ctx, reinterpret_cast<const void*>(kern), smem, *n);
  return FF_OK;
}
// Rows in flight: as many slots as fit the share of shared memory that a CTA may take, two to eight.
inline int ln_slots(size_t slot_bytes, size_t share) {
  const size_t n = share / slot_bytes;
  return n > LN_MAX_SLOTS ? LN_MAX_SLOTS : (int)n;
}
template <typename T, int TEAM, int V, int R, int A>
ff_status ln_forward_launch(ff_ctx* ctx, const LnFwd& p, cudaStream_t st) {
  constexpr int threads = TEAM > 256 ? TEAM : 256, per = threads / TEAM * R;
  ln_forward_kernel<T, TEAM, V, R, A><<<(unsigned)((p.rows + per - 1) / per), threads, 0, st>>>(p);
  FF_LAUNCH_CHECK(ctx);
  return FF_OK;
}
template <typename T, int A>
ff_status ln_forward_dispatch(ff_ctx* ctx, const LnFwd& p, cudaStream_t st) {
  if (p.cols <= 64) return ln_forward_launch<T, 8, 1, 1, A>(ctx, p, st);
  if (p.cols <= 128) return ln_forward_launch<T, 16, 1, 1, A>(ctx, p, st);
  if (p.cols <= 256) return ln_forward_launch<T, 32, 1, 1, A>(ctx, p, st);
  // Few rows: a group a thread, for the shortest way through a row, as long as the threads that fit the device (1024 an SM) hold
  // the tensor, or nearly.  Against two groups a thread and two rows a team, bfloat16: 148 x 784 2.7 us against 4.4, 1184 x 784 3.7 against
  // 4.5, 2368 x 784 5.9 against 5.1; 592 x 2000 3.7 against 4.5, 1184 x 2000 5.7 against 5.2; 148 x 8192 3.6 against 4.8, 296 x 8192
  // 6.0 against 5.0, 592 x 8192 10.8 against 6.9.
  if (3 * p.rows * p.cols <= 4LL * (1024 * C8_GROUP) * ctx->sm_count) {
    if (p.cols <= 512) return ln_forward_launch<T, 64, 1, 1, A>(ctx, p, st);
    if (p.cols <= 1024) return ln_forward_launch<T, 128, 1, 1, A>(ctx, p, st);
    if (p.cols <= 2048) return ln_forward_launch<T, 256, 1, 1, A>(ctx, p, st);
    if (p.cols <= 4096) return ln_forward_launch<T, 512, 1, 1, A>(ctx, p, st);
    if (p.cols <= LN_MAX_COLS) return ln_forward_launch<T, 1024, 1, 1, A>(ctx, p, st);
  }
  if (p.cols <= 512) return ln_forward_launch<T, 32, 2, 2, A>(ctx, p, st);
  if (p.cols <= 1024) return ln_forward_launch<T, 64, 2, 2, A>(ctx, p, st);
  if (p.cols <= 2048) return ln_forward_launch<T, 128, 2, 2, A>(ctx, p, st);
  if (p.cols <= 4096) return ln_forward_launch<T, 256, 2, 2, A>(ctx, p, st);
  if (p.cols <= LN_MAX_COLS) return ln_forward_launch<T, 512, 2, 2, A>(ctx, p, st);
  ln_forward_long_kernel<T, A><<<(unsigned)p.rows, LN_LONG_THREADS, 0, st>>>(p);
  FF_LAUNCH_CHECK(ctx);
  return FF_OK;
}

// CTAs of a backward pass: they stay resident and share the rows; `parts` of them leave sums to add up.
template <class K>
ff_status ln_backward_launch(ff_ctx* ctx, K kern, const LnBwd& p, int threads, int rows_per_step, size_t smem, int* parts, cudaStream_t st) {
  int most = 0;
  const ff_status s = resident_ctas(ctx, kern, threads, smem, &most);
  if (s != FF_OK) return s;
  const long long want = (p.rows + rows_per_step - 1) / rows_per_step;
  long long grid = want < most ? want : most;
  if (grid > LN_MAX_PARTS) grid = LN_MAX_PARTS;
  *parts = (int)grid;
  kern<<<(unsigned)grid, threads, smem, st>>>(p);
  FF_LAUNCH_CHECK(ctx);
  return FF_OK;
}
template <typename T, bool CK, int TEAM, int V>
ff_status ln_backward_ring(ff_ctx* ctx, const LnBwd& p, int* parts, cudaStream_t st) {
  constexpr int threads = TEAM > 256 ? TEAM : 256, teams = threads / TEAM;
  const size_t row = (size_t)p.cols * sizeof(T), x = CK ? (size_t)(p.cols + 15) / 16 * 16 : row, params = ((size_t)p.cols + 7) / 8 * 32;
  auto slot = [&](int rows) {   // of one team, as the kernel lays it out
    return (rows * (row * (p.dadd ? 2 : 1) + x + (CK ? ln_exponent_bytes(p.cols) : 0) + 8) + 15) / 16 * 16;
  };
  // shared memory of one or two CTAs an SM, less what the kernel has for itself
  const size_t share = (size_t)(TEAM > 256 ? 220 : 110) * 1024 - 2048 - params - (teams > 1 ? ln_acc_floats<TEAM, teams, V>() * sizeof(float) : 0);
  LnBwd q = p;
  // two rows a step where three steps fit the ring: half as many barriers (with two groups a thread there are no registers for it).
  // From the checkpoint, two rows against one: 32768 x 4096 bfloat16 160 us against 186, 16384 x 2048 FP32 58 against 65, 32768 x 1000 FP32 68 against 65.
  if constexpr (V == 1)
    if ((q.slots = ln_slots(teams * slot(2), share)) >= 3)
      return ln_backward_launch(ctx, ln_backward_ring_kernel<T, TEAM, V, 2, CK>, q, threads + 32, 2 * teams, params + q.slots * teams * slot(2), parts, st);
  if ((q.slots = ln_slots(teams * slot(1), share)) < 2) q.slots = 2;
  return ln_backward_launch(ctx, ln_backward_ring_kernel<T, TEAM, V, 1, CK>, q, threads + 32, teams, params + q.slots * teams * slot(1), parts, st);
}
template <typename T, bool CK, int A>
ff_status ln_backward_dispatch(ff_ctx* ctx, const LnBwd& p, int* parts, cudaStream_t st) {
  // The ring against rows in registers, from the checkpoint, bfloat16: 65536 x 520 119 us against 119 (from x 97 against 121), 32768 x 1000 66 against
  // 78, 65536 x 2000 163 against 296, 32768 x 8192 296 against 350; with one row a CTA (300 x 8192) 20 against 19.
  if constexpr (A == 16) {
    if (p.cols > 512 && p.cols <= LN_MAX_COLS && p.cols * sizeof(T) % 16 == 0 && (!CK || (reinterpret_cast<uintptr_t>(p.c.e) & 3) == 0)) {
      if (p.cols <= 1024) return ln_backward_ring<T, CK, 128, 1>(ctx, p, parts, st);
      if (p.cols <= 2048) return ln_backward_ring<T, CK, 256, 1>(ctx, p, parts, st);
      if (p.cols <= 4096) return ln_backward_ring<T, CK, 512, 1>(ctx, p, parts, st);
      return ln_backward_ring<T, CK, 512, 2>(ctx, p, parts, st);
    }
  }
  if (p.cols <= 64) return ln_backward_launch(ctx, ln_backward_kernel<T, 8, 1, CK, A>, p, 256, 32, 0, parts, st);
  if (p.cols <= 256) return ln_backward_launch(ctx, ln_backward_kernel<T, 32, 1, CK, A>, p, 256, 8, 0, parts, st);
  if (p.cols <= 512) return ln_backward_launch(ctx, ln_backward_kernel<T, 32, 2, CK, A>, p, 256, 8, 0, parts, st);
  if (p.cols <= 1024) return ln_backward_launch(ctx, ln_backward_kernel<T, 128, 1, CK, A>, p, 256, 2, 0, parts, st);
  if (p.cols <= 2048) return ln_backward_launch(ctx, ln_backward_kernel<T, 256, 1, CK, A>, p, 256, 1, 0, parts, st);
  if (p.cols <= 4096) return ln_backward_launch(ctx, ln_backward_kernel<T, 512, 1, CK, A>, p, 512, 1, 0, parts, st);
  if (p.cols <= LN_MAX_COLS) return ln_backward_launch(ctx, ln_backward_kernel<T, 512, 2, CK, A>, p, 512, 1, 0, parts, st);
  // the sums first: they read dY, which dX may overwrite
  if (p.part) {
    const int gx = (p.cols + 255) / 256;
    long long gy = (8LL * ctx->sm_count + gx - 1) / gx;
    if (gy > (p.rows + 63) / 64) gy = (p.rows + 63) / 64;
    if (gy > LN_MAX_PARTS) gy = LN_MAX_PARTS;
    const long long rows_per = (p.rows + gy - 1) / gy;
    gy = (p.rows + rows_per - 1) / rows_per;
    *parts = (int)gy;
    ln_column_sums_kernel<T, CK, A><<<dim3(gx, (unsigned)gy), 256, 0, st>>>(p, rows_per);
    FF_LAUNCH_CHECK(ctx);
  }
  if (p.dx) {
    ln_backward_long_kernel<T, CK, A><<<(unsigned)p.rows, LN_LONG_THREADS, 0, st>>>(p);
    FF_LAUNCH_CHECK(ctx);
  }
  return FF_OK;
}

// ---- weight gradient ------------------------------------------------------------------------
inline int wgrad_parts(int dtype) { return dtype == FF_F32 ? 3 : dtype == FF_F16 ? 2 : 1; }
template <int PARTS>
ff_status wgrad_gemm(ff_ctx* ctx, const WgradArgs& p, cudaStream_t st) {
  using G = WgGeom<PARTS>;
  auto kern = wgrad_gemm_kernel<PARTS>;
  CUtensorMap dy, x;
  ff_status s = p.parts ? wg_make_map(ctx->tc, &dy, p.parts, p.N, p.rows, PARTS, p.ld_parts * 2)
                        : wg_make_map(ctx->tc, &dy, p.dy, p.N, p.rows, 1, p.ld_dy * 2);
  if (s == FF_OK) s = wg_make_map(ctx->tc, &x, p.x, p.K, p.rows, 0, p.ld_x * 2);
  if (s != FF_OK) return fail(ctx, s, "%s", ctx->tc.err);
  int groups = known_resident(ctx, reinterpret_cast<const void*>(kern), G::SMEM_BYTES);   // CTA pairs that fit on the device
  if (groups == 0) {
    FF_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)G::SMEM_BYTES));
    groups = ctx->sm_count / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * groups), cfg.blockDim = dim3(WG_THREADS), cfg.dynamicSmemBytes = G::SMEM_BYTES;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) == cudaSuccess && n > 0 && n < groups) groups = n;
    (void)cudaGetLastError();
    keep_resident(ctx, reinterpret_cast<const void*>(kern), G::SMEM_BYTES, groups);
  }
  const int items = p.tiles_n * p.tiles_k * p.splits;
  return launch_after(ctx, kern, dim3(2 * (items < groups ? items : groups)), WG_THREADS, G::SMEM_BYTES, st, dy, x, p);
}

// ---- activations ----------------------------------------------------------------------------
template <class F>
ff_status for_act(int kind, F f) {
  if (kind == FF_ACT_RELU) return f(std::integral_constant<int, ACT_RELU>());
  if (kind == FF_ACT_GELU) return f(std::integral_constant<int, ACT_GELU>());
  return f(std::integral_constant<int, ACT_SILU>());
}
ff_status check_act(ff_ctx* ctx, const ff_activation_desc* d, const ff_activation_bufs* b, int64_t rows) {
  if (!d || !b) return fail(ctx, FF_ERR_ARG, "activation descriptor or buffer struct is NULL");
  if (d->kind != FF_ACT_RELU && d->kind != FF_ACT_GELU && d->kind != FF_ACT_SILU) return fail(ctx, FF_ERR_ARG, "unknown activation");
  return check_extent(ctx, rows, d->cols, d->dtype, d->round);
}

}  // namespace

extern "C" {

ff_status ff_layernorm_workspace_bytes(const ff_layernorm_desc* d, int64_t rows, size_t* out_bytes) {
  if (!d || !out_bytes || d->cols <= 0 || rows < 0) return FF_ERR_ARG;
  *out_bytes = WS_BYTES + up256(ln_part_bytes(d->cols, rows));
  return FF_OK;
}

ff_status ff_layernorm_forward(ff_ctx* ctx, const ff_layernorm_desc* d, const ff_layernorm_bufs* b, int64_t rows, uint64_t step,
                               void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if ((s = check_ln(ctx, d, b, rows)) != FF_OK) return s;
  const bool ck = b->C.q || b->C.e;
  if (rows) {
    if ((s = check_tensor(ctx, b->X, b->ld_x, d->cols, d->dtype, "X")) != FF_OK) return s;
    if (b->Y && (s = check_tensor(ctx, b->Y, b->ld_y, d->cols, d->dtype, "Y")) != FF_OK) return s;
    if (ck && (s = check_ckpt(ctx, b->C, d->cols)) != FF_OK) return s;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if ((s = ensure_status(ctx, st)) != FF_OK) return s;
  if (!rows) return FF_OK;
  LnFwd p;
  p.x = b->X, p.gamma = b->gamma, p.beta = b->beta, p.y = b->Y, p.mean = b->mean, p.rstd = b->rstd;
  p.ld_x = b->ld_x, p.ld_y = b->ld_y, p.rows = rows, p.cols = d->cols, p.eps = d->eps;
  p.c = view(b->C), p.round = rounding(d->round, d->seed, ROLE_CKPT, d->index, step, d->cols), p.status = status_ptr(ctx);
  p.vec = ((reinterpret_cast<uintptr_t>(b->gamma) | reinterpret_cast<uintptr_t>(b->beta)) & 31) == 0;
  const unsigned al = least(row_alignment(b->X, b->ld_x, d->dtype), row_alignment(b->Y, b->ld_y, d->dtype));
  ProfScope prof(ctx, FF_K_LAYERNORM_FWD, st);
  return for_dtype(d->dtype, [&](auto t) {
    using T = decltype(t);
    return for_alignment<T>(al, [&](auto a) { return ln_forward_dispatch<T, decltype(a)::value>(ctx, p, st); });
  });
}

ff_status ff_layernorm_backward(ff_ctx* ctx, const ff_layernorm_desc* d, const ff_layernorm_bufs* b, int64_t rows, void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if ((s = check_ln(ctx, d, b, rows)) != FF_OK) return s;
  const bool ck = b->C.q || b->C.e;
  const bool sums = b->dgamma || b->dbeta;
  if (!b->dX && !sums) return fail(ctx, FF_ERR_ARG, "nothing to compute: dX, dgamma and dbeta are all NULL");
  if (rows) {
    if ((s = check_tensor(ctx, b->dY, b->ld_dy, d->cols, d->dtype, "dY")) != FF_OK) return s;
    if (b->dX && (s = check_tensor(ctx, b->dX, b->ld_dx, d->cols, d->dtype, "dX")) != FF_OK) return s;
    if (b->dAdd && (s = check_tensor(ctx, b->dAdd, b->ld_dadd, d->cols, d->dtype, "dAdd")) != FF_OK) return s;
    if (!b->rstd) return fail(ctx, FF_ERR_ARG, "%s is NULL", "rstd");
    if (ck) {
      if ((s = check_ckpt(ctx, b->C, d->cols)) != FF_OK) return s;
    } else {
      if ((s = check_tensor(ctx, b->X, b->ld_x, d->cols, d->dtype, "X")) != FF_OK) return s;
      if (!b->mean) return fail(ctx, FF_ERR_ARG, "%s is NULL", "mean");
    }
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (sums && ctx->workspace_bytes < WS_BYTES + ln_part_bytes(d->cols, rows))
    return fail(ctx, FF_ERR_WORKSPACE, "workspace too small for the sums over rows (ff_layernorm_workspace_bytes)");
  if ((s = ensure_status(ctx, st)) != FF_OK) return s;
  LnBwd p;
  p.dy = b->dY, p.dadd = b->dAdd, p.x = b->X, p.mean = b->mean, p.rstd = b->rstd, p.gamma = b->gamma, p.dx = b->dX;
  p.ld_dy = b->ld_dy, p.ld_dadd = b->ld_dadd, p.ld_x = b->ld_x, p.ld_dx = b->ld_dx, p.rows = rows, p.cols = d->cols;
  p.c = view(b->C), p.slots = 0, p.status = status_ptr(ctx);
  p.part = sums ? reinterpret_cast<float*>(static_cast<char*>(ctx->workspace) + WS_BYTES) : nullptr;
  int parts = 0;
  ProfScope prof(ctx, FF_K_LAYERNORM_BWD, st);
  if (rows) {
    p.vec = (reinterpret_cast<uintptr_t>(b->gamma) & 31) == 0;
    const unsigned al = least(least(row_alignment(b->dY, b->ld_dy, d->dtype), row_alignment(b->dX, b->ld_dx, d->dtype)),
                              least(row_alignment(b->dAdd, b->ld_dadd, d->dtype), ck ? 16 : row_alignment(b->X, b->ld_x, d->dtype)));
    s = for_dtype(d->dtype, [&](auto t) {
      using T = decltype(t);
      return for_alignment<T>(al, [&](auto a) {
        return for_flag(ck, [&](auto c) { return ln_backward_dispatch<T, decltype(c)::value, decltype(a)::value>(ctx, p, &parts, st); });
      });
    });
    if (s != FF_OK) return s;
  }
  if (sums) {
    s = launch_after(ctx, ln_finish_kernel, dim3((2 * d->cols + 31) / 32), 512, 0, st, static_cast<const float*>(p.part), parts, (int)d->cols, b->dgamma,
                     b->dbeta, (int)d->accumulate);
    if (s != FF_OK) return s;
  }
  return FF_OK;
}

ff_status ff_ckpt8_save(ff_ctx* ctx, const void* X, int64_t ld_x, int32_t dtype, int64_t rows, int32_t cols, const ff_ckpt8* c,
                        int32_t round, uint64_t seed, int32_t index, uint64_t step, void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if (!c) return fail(ctx, FF_ERR_ARG, "checkpoint struct is NULL");
  if ((s = check_extent(ctx, rows, cols, dtype, round)) != FF_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (rows) {
    if ((s = check_tensor(ctx, X, ld_x, cols, dtype, "X")) != FF_OK) return s;
    if ((s = check_ckpt(ctx, *c, cols)) != FF_OK) return s;
  }
  if ((s = ensure_status(ctx, st)) != FF_OK) return s;
  if (!rows) return FF_OK;
  const GroupList gl = make_group_list(rows, cols);
  ProfScope prof(ctx, FF_K_CKPT8, st);
  return for_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    return for_alignment<T>(row_alignment(X, ld_x, dtype), [&](auto f) -> ff_status {
      ckpt8_save_kernel<T, decltype(f)::value><<<group_blocks(gl), C8_THREADS, 0, st>>>(
          static_cast<const T*>(X), ld_x, cols, gl, view(*c), rounding(round, seed, ROLE_CKPT, index, step, cols), status_ptr(ctx));
      FF_LAUNCH_CHECK(ctx);
      return FF_OK;
    });
  });
}

ff_status ff_ckpt8_restore(ff_ctx* ctx, const ff_ckpt8* c, int64_t rows, int32_t cols, void* Y, int64_t ld_y, int32_t dtype,
                           void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if (!c) return fail(ctx, FF_ERR_ARG, "checkpoint struct is NULL");
  if ((s = check_extent(ctx, rows, cols, dtype, FF_ROUND_NEAREST_EVEN)) != FF_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!rows) return FF_OK;
  if ((s = check_tensor(ctx, Y, ld_y, cols, dtype, "Y")) != FF_OK) return s;
  if ((s = check_ckpt(ctx, *c, cols)) != FF_OK) return s;
  const GroupList gl = make_group_list(rows, cols);
  ProfScope prof(ctx, FF_K_CKPT8, st);
  return for_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    return for_alignment<T>(row_alignment(Y, ld_y, dtype), [&](auto f) -> ff_status {
      ckpt8_restore_kernel<T, decltype(f)::value><<<group_blocks(gl), C8_THREADS, 0, st>>>(view(*c), cols, gl, static_cast<T*>(Y), ld_y);
      FF_LAUNCH_CHECK(ctx);
      return FF_OK;
    });
  });
}

ff_status ff_activation_forward(ff_ctx* ctx, const ff_activation_desc* d, const ff_activation_bufs* b, int64_t rows, uint64_t step,
                                void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if ((s = check_act(ctx, d, b, rows)) != FF_OK) return s;
  const bool kh = b->CH.q || b->CH.e, kz = b->CZ.q || b->CZ.e;
  if (!b->Z && !kh && !kz) return fail(ctx, FF_ERR_ARG, "nothing to compute: Z and both checkpoints are NULL");
  if (rows) {
    if ((s = check_tensor(ctx, b->H, b->ld_h, d->cols, d->dtype, "H")) != FF_OK) return s;
    if (b->Z && (s = check_tensor(ctx, b->Z, b->ld_z, d->cols, d->dtype, "Z")) != FF_OK) return s;
    if (kh && (s = check_ckpt(ctx, b->CH, d->cols)) != FF_OK) return s;
    if (kz && (s = check_ckpt(ctx, b->CZ, d->cols)) != FF_OK) return s;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if ((s = ensure_status(ctx, st)) != FF_OK) return s;
  if (!rows) return FF_OK;
  const GroupList gl = make_group_list(rows, d->cols);
  const unsigned al = least(row_alignment(b->H, b->ld_h, d->dtype), row_alignment(b->Z, b->ld_z, d->dtype));
  ProfScope prof(ctx, FF_K_ACTIVATION, st);
  return for_dtype(d->dtype, [&](auto t) {
    using T = decltype(t);
    return for_act(d->kind, [&](auto k) {
      return for_alignment<T>(al, [&](auto f) -> ff_status {
        act_forward_kernel<T, decltype(k)::value, decltype(f)::value><<<group_blocks(gl), C8_THREADS, 0, st>>>(
            static_cast<const T*>(b->H), b->ld_h, static_cast<T*>(b->Z), b->ld_z, d->cols, gl, view(b->CH), view(b->CZ),
            rounding(d->round, d->seed, ROLE_CKPT, d->index, step, d->cols),
            rounding(d->round & ~FF_ROUND_KEEP_SIGN, d->seed, ROLE_CKPT_OUT, d->index, step, d->cols), status_ptr(ctx));
        FF_LAUNCH_CHECK(ctx);
        return FF_OK;
      });
    });
  });
}

ff_status ff_activation_backward(ff_ctx* ctx, const ff_activation_desc* d, const ff_activation_bufs* b, int64_t rows, void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if ((s = check_act(ctx, d, b, rows)) != FF_OK) return s;
  if (!rows) return FF_OK;
  if ((s = check_tensor(ctx, b->dZ, b->ld_dz, d->cols, d->dtype, "dZ")) != FF_OK) return s;
  if ((s = check_tensor(ctx, b->dH, b->ld_dh, d->cols, d->dtype, "dH")) != FF_OK) return s;
  if ((s = check_ckpt(ctx, b->CH, d->cols)) != FF_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const GroupList gl = make_group_list(rows, d->cols);
  const unsigned al = least(row_alignment(b->dZ, b->ld_dz, d->dtype), row_alignment(b->dH, b->ld_dh, d->dtype));
  ProfScope prof(ctx, FF_K_ACTIVATION, st);
  return for_dtype(d->dtype, [&](auto t) {
    using T = decltype(t);
    return for_act(d->kind, [&](auto k) {
      return for_alignment<T>(al, [&](auto f) -> ff_status {
        const int all = group_blocks(gl), most = 8 * ctx->sm_count;   // resident CTAs: each computes its table once
        act_backward_kernel<T, decltype(k)::value, decltype(f)::value><<<all < most ? all : most, C8_THREADS, 0, st>>>(
            static_cast<const T*>(b->dZ), b->ld_dz, view(b->CH), static_cast<T*>(b->dH), b->ld_dh, d->cols, gl);
        FF_LAUNCH_CHECK(ctx);
        return FF_OK;
      });
    });
  });
}

ff_status ff_ckpt8_wgrad_workspace_bytes(const ff_ckpt8_wgrad_desc* d, int64_t rows, size_t* out_bytes) {
  if (!d || !out_bytes || d->N <= 0 || d->K <= 0 || !known_dtype(d->dtype) || rows < 0 || rows > BLOCK_MAX_ROWS) return FF_ERR_ARG;
  // the splits that the CTA pairs of a 148-SM device want; a bfloat16 dY may turn out to need a copy with aligned rows
  const WgPlan pl = wg_plan(rows, d->N, d->K, wgrad_parts(d->dtype), true, true, 74, SIZE_MAX);
  *out_bytes = WS_BYTES + pl.x_bytes + pl.parts_bytes + pl.db_bytes + pl.part_bytes;
  return FF_OK;
}

ff_status ff_ckpt8_wgrad(ff_ctx* ctx, const ff_ckpt8_wgrad_desc* d, const ff_ckpt8_wgrad_bufs* b, int64_t rows, void* cuda_stream) {
  ff_status s = check_ctx(ctx);
  if (s != FF_OK) return s;
  if (!d || !b) return fail(ctx, FF_ERR_ARG, "weight gradient descriptor or buffer struct is NULL");
  if ((s = check_extent(ctx, rows, d->K, d->dtype, FF_ROUND_NEAREST_EVEN)) != FF_OK) return s;
  if ((s = check_extent(ctx, rows, d->N, d->dtype, FF_ROUND_NEAREST_EVEN)) != FF_OK) return s;
  if ((long long)d->N * d->K > (1LL << 40)) return fail(ctx, FF_ERR_RANGE, "dW has more than 2^40 values");
  if (!b->dW) return fail(ctx, FF_ERR_ARG, "%s is NULL", "dW");
  const struct {
    const void* p;
    const char* name;
  } f[] = {{b->gamma, "gamma"}, {b->beta, "beta"}, {b->dW, "dW"}, {b->dbias, "dbias"}};
  for (const auto& x : f)
    if ((s = check_floats(ctx, x.p, x.name)) != FF_OK) return s;
  if (rows) {
    if ((s = check_tensor(ctx, b->dY, b->ld_dy, d->N, d->dtype, "dY")) != FF_OK) return s;
    if ((s = check_ckpt(ctx, b->C, d->K)) != FF_OK) return s;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned al = row_alignment(b->dY, b->ld_dy, d->dtype);
  const bool split = !(d->dtype == FF_BF16 && al == 16);   // dY itself cannot be the operand
  const bool sums = rows && (b->dbias || b->beta);
  const WgPlan pl = wg_plan(rows, d->N, d->K, wgrad_parts(d->dtype), split, sums, ctx->sm_count / 2,
                            ctx->workspace_bytes - WS_BYTES);   // ff_set_workspace takes no less than WS_BYTES
  const size_t need = WS_BYTES + pl.x_bytes + pl.parts_bytes + pl.db_bytes + pl.part_bytes;
  if (ctx->workspace_bytes < need) return fail(ctx, FF_ERR_WORKSPACE, "workspace too small (ff_ckpt8_wgrad_workspace_bytes): needs %s%lld", "", (long long)need);
  if ((s = ensure_status(ctx, st)) != FF_OK) return s;
  WgradArgs p;
  char* ws = static_cast<char*>(ctx->workspace) + WS_BYTES;
  p.dy = b->dY, p.ld_dy = b->ld_dy, p.c = view(b->C), p.gamma = b->gamma, p.beta = b->beta, p.dw = b->dW, p.db = b->dbias;
  p.x = reinterpret_cast<__nv_bfloat16*>(ws);
  p.parts = split ? reinterpret_cast<__nv_bfloat16*>(ws + pl.x_bytes) : nullptr;
  p.db_part = sums ? reinterpret_cast<float*>(ws + pl.x_bytes + pl.parts_bytes) : nullptr;
  p.part = reinterpret_cast<float*>(ws + pl.x_bytes + pl.parts_bytes + pl.db_bytes);
  p.rows = rows, p.db_rows = pl.db_rows, p.ld_x = pl.ld_x, p.ld_parts = pl.ld_parts;
  p.N = d->N, p.K = d->K, p.accumulate = d->accumulate, p.db_parts = pl.db_parts;
  p.bn = pl.bn, p.tiles_n = pl.tiles_n, p.tiles_k = pl.tiles_k, p.splits = pl.splits, p.stages_per_split = pl.stages_per_split;
  p.stages = pl.stages, p.status = status_ptr(ctx);
  ProfScope prof(ctx, FF_K_CKPT8_WGRAD, st);
  if (rows) {
    // 16 codes a unit: the list of a tensor with half as many columns, in blocks of four units
    const GroupList units = make_group_list(rows, (int)((pl.ld_x + 1) / 2));
    const uint32_t x_blocks = (units.total + 1023) / 1024, dy_cols = (uint32_t)((d->N + pl.dy_lanes * 8 - 1) / (pl.dy_lanes * 8));
    const uint32_t blocks = x_blocks + (split || sums ? dy_cols * (uint32_t)pl.db_parts : 0u);
    s = for_dtype(d->dtype, [&](auto t) {
      using T = decltype(t);
      constexpr int PARTS = sizeof(T) == 4 ? 3 : std::is_same<T, __half>::value ? 2 : 1;
      return for_flag(split, [&](auto sp) {
        return for_alignment<T>(al, [&](auto fl) -> ff_status {
          wgrad_prepare_kernel<T, PARTS, decltype(sp)::value, decltype(fl)::value><<<blocks, 256, 0, st>>>(p, units, x_blocks, dy_cols, pl.dy_lanes);
          FF_LAUNCH_CHECK(ctx);
          return FF_OK;
        });
      });
    });
    if (s != FF_OK) return s;
    s = d->dtype == FF_BF16 ? wgrad_gemm<1>(ctx, p, st) : d->dtype == FF_F16 ? wgrad_gemm<2>(ctx, p, st) : wgrad_gemm<3>(ctx, p, st);
    if (s != FF_OK) return s;
  }
  if (!rows || pl.splits > 1) {
    const int ky = (d->K + 1023) / 1024;
    s = launch_after(ctx, wgrad_join_kernel, dim3(d->N, ky < 65535 ? ky : 65535), 256, 0, st, p, rows ? pl.splits : 0);
    if (s != FF_OK) return s;
  }
  return FF_OK;
}

}  // extern "C"
