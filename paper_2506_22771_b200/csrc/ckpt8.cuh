// 8-bit activation checkpoints and the element-wise operators that write and read them.
//
// A checkpoint holds a [rows, cols] tensor as INT8 codes with one power of two per block of 32 consecutive columns
// of a row: E is the least integer with max|x| <= 127 * 2^E, the code is x * 2^-E rounded (nearest even, or
// floor(t + u) with the library's rounding hash), the stored byte is E + 127.  With a power of two the quantiser's
// product is exact, so a code has one correct value, and code * 2^E has at most 7 significant bits: the
// restored value is exact in bfloat16 and in FP32, and a matrix instruction takes it without another rounding.
// At E = 122 codes stop at 63 (64 * 2^122 would be past FP32).  Where signs are kept, code 0 is for zeros alone.
// A block whose maximum lies below 2^-100 is zero (the range rule of the library's INT8 quantiser).  A block with an
// Inf or a NaN gets byte 255: its codes are zero, it restores to NaN (0 * Inf) and raises ST_NONFINITE.
//
// A thread owns a group of 8 consecutive columns, four neighbouring lanes a block, and issues the loads of several groups before
// it computes.  Save, restore and the activations' backward pass are bound by HBM (3 to 9 bytes per value, 5.9 to 6.5 TB/s on rows
// of whole 16-byte words), the activations' forward pass with two checkpoints by its instructions (8192 x 2000 bfloat16 28 us
// against 15 of HBM), every form with stochastic rounding by the hash (save 9.5 us nearest, 21 stochastic; two checkpoints of GELU 28 and 52).
// Rows aligned only to their type go value by value and are bound by these accesses (save 13 us, restore 53 against 7.4).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace ffi8 {

constexpr int ROLE_CKPT = 3;      // rounding key of a saved input (or of a layer norm's normalised value)
constexpr int ROLE_CKPT_OUT = 4;  // rounding key of a saved activation output
constexpr int C8_BLOCK = 32, C8_GROUP = 8;

// Two launches of one call: the second one is launched with the programmatic attribute (launch_after), may start while the
// first one's last blocks run, and waits here before it reads what the first one wrote.
__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- groups of 8 values ----------------------------------------------------------------------
template <typename T>
struct Raw8 {  // as in memory
  uint4 w[sizeof(T) * 8 / 16];
};
// A: alignment in bytes that the tensor's rows are known to have (16, 8, or only that of the type): a whole group moves in
// words of that size, a group that the row's end cuts value by value.  n = values of the group inside the row (<= 0: none).
template <typename T, int A>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = make_uint4(0u, 0u, 0u, 0u);
  if (A > (int)sizeof(T) && n >= 8) {
    if (A == 16) {
#pragma unroll
      for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint2*>(r.w)[i] = __ldcs(reinterpret_cast<const uint2*>(p) + i);
    }
  } else {
    uint32_t* u = reinterpret_cast<uint32_t*>(r.w);
    if (sizeof(T) == 4) {
      const uint32_t* s = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) u[j] = s[j];
    } else {
      const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) u[j >> 1] |= (uint32_t)s[j] << (16 * (j & 1));
    }
  }
  return r;
}
template <typename T, int A>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r, int n) {
  if (A > (int)sizeof(T) && n >= 8) {
    if (A == 16) {
#pragma unroll
      for (int i = 0; i < (int)(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = r.w[i];
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint2*>(p)[i] = reinterpret_cast<const uint2*>(r.w)[i];
    }
  } else {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(r.w);
    if (sizeof(T) == 4) {
      uint32_t* d = reinterpret_cast<uint32_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) d[j] = u[j];
    } else {
      uint16_t* d = reinterpret_cast<uint16_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) d[j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
    }
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[4 * i] = __uint_as_float(r.w[i].x), v[4 * i + 1] = __uint_as_float(r.w[i].y);
    v[4 * i + 2] = __uint_as_float(r.w[i].z), v[4 * i + 3] = __uint_as_float(r.w[i].w);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
  const uint32_t u[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__half>& r, float (&v)[8]) {
  const uint32_t u[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}
// rounded to the tensor's type, once
__device__ __forceinline__ Raw8<float> pack8(const float (&v)[8], float) {
  Raw8<float> r;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    r.w[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
  return r;
}
__device__ __forceinline__ Raw8<__nv_bfloat16> pack8(const float (&v)[8], __nv_bfloat16) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  Raw8<__nv_bfloat16> r;
  r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
  return r;
}
__device__ __forceinline__ Raw8<__half> pack8(const float (&v)[8], __half) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  Raw8<__half> r;
  r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
  return r;
}

// ---- the codec -------------------------------------------------------------------------------
// Largest magnitude of three; a NaN stays.
__device__ __forceinline__ float max_abs_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float c8_scale(uint32_t e) { return __uint_as_float(e << 23); }

struct C8Round {  // how codes are rounded
  int stochastic, keep_sign;
  RoundKey key;
  uint32_t cols;  // the rounding counter is the dense element index row * cols + column
};
// Codes of a group, whose values outside the row are zeros; the four lanes of its block have called this together
// (shuffles inside).  Returns the block's stored byte.
__device__ __forceinline__ uint32_t c8_encode(const float (&v)[8], uint32_t row, uint32_t col, const C8Round& rd, uint2& codes) {
  float most = max_abs_nan(v[0], v[1], v[2]);
  most = max_abs_nan(most, v[3], v[4]);
  most = max_abs_nan(most, v[5], max_abs_nan(v[6], v[7], v[7]));
  const float other = __shfl_xor_sync(0xffffffffu, most, 1);
  most = max_abs_nan(most, other, other);
  const float far = __shfl_xor_sync(0xffffffffu, most, 2);
  most = max_abs_nan(most, far, far);
  const uint32_t bits = __float_as_uint(most);   // >= 0, or NaN
  uint32_t e = ((bits + 0x1FFFFu) >> 23) - 6u;   // 127 = 1.984375 * 2^6: a mantissa above 0x7E0000 carries into the next binade
  const float inv = __uint_as_float((254u - e) << 23);
  const bool plain = bits - 0x0D800000u < 0x7f800000u - 0x0D800000u && e != 249u;   // 2^-100 <= most < Inf
  int q[8];
  if (!rd.stochastic) {
    // x * 2^-E is exact and at most 127, so adding 1.5 * 2^23 in the same operation leaves it rounded to nearest even
    // in the low byte (the sum's last place is 1)
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = (int)__float_as_uint(fmaf(v[j], inv, 12582912.0f));
  } else {
    const uint32_t i0 = row * rd.cols + col;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = quant_one<ROUND_STOCHASTIC>(v[j], inv, i0 + j, rd.key);
  }
  if (rd.keep_sign) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if ((q[j] & 255) == 0 && v[j] != 0.0f) q[j] = v[j] > 0.0f ? 1 : -1;
  }
  if (!plain) {   // zero or non-finite block; at E = 122 the code 64 would restore to 2^128
    e = most < TINY_RANGE ? 0u : bits >= 0x7f800000u ? 255u : 249u;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = e == 249u ? max(-63, min(63, (int)(int8_t)q[j])) : 0;
  }
  codes = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
  return e;
}
__device__ __forceinline__ void c8_decode(uint2 codes, uint32_t e, float (&v)[8]) {
  // byte ^ 0x80 placed in the mantissa of 2^23 is 2^23 + 128 + q; times 2^E less (2^23 + 128) 2^E in one operation is exact
  const uint32_t a = codes.x ^ 0x80808080u, b = codes.y ^ 0x80808080u;
  const float scale = c8_scale(e);
  if (e < 230u) {
    const float bias = -8388736.0f * scale;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = fmaf(__uint_as_float(__byte_perm(a, 0x4B000000u, 0x7540 + j)), scale, bias);
      v[4 + j] = fmaf(__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7540 + j)), scale, bias);
    }
  } else {   // (2^23 + 128) 2^E is past FP32, or the block restores to NaN (0 * Inf)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = __fmul_rn(__fsub_rn(__uint_as_float(__byte_perm(a, 0x4B000000u, 0x7540 + j)), 8388736.0f), scale);
      v[4 + j] = __fmul_rn(__fsub_rn(__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7540 + j)), 8388736.0f), scale);
    }
  }
}

// A checkpoint's arrays; every row starts on a 16-byte boundary (ld_q), so a group is one 8-byte word even where the
// row ends inside it (the bytes up to the next multiple of 8 are written as zeros).
struct C8View {
  int8_t* q;
  uint8_t* e;
  long long ld_q, ld_e;
};
__device__ __forceinline__ void c8_store(const C8View& c, long long row, int col, uint2 codes, uint32_t e, uint32_t* status) {
  *reinterpret_cast<uint2*>(c.q + row * c.ld_q + col) = codes;
  if ((col & (C8_BLOCK - 1)) == 0) {
    c.e[row * c.ld_e + col / C8_BLOCK] = (uint8_t)e;
    if (e == 255u) atomicOr(status, ST_NONFINITE);
  }
}

// rows x groups of 8 columns as one list: item i is group i % per_row of row i / per_row, per_row a multiple of 4 (whole
// blocks).  The quotient is a multiplication: m = ceil(2^(32+s) / per_row) with 2^s >= per_row > 2^(s-1) is exact for i < 2^31.
struct GroupList {
  uint32_t total, per_row, m, s;
};
__host__ inline GroupList make_group_list(long long rows, int cols) {
  GroupList g;
  g.per_row = (uint32_t)((cols + C8_BLOCK - 1) / C8_BLOCK * 4);
  g.total = (uint32_t)(rows * g.per_row);
  g.s = 0;
  while ((1ull << g.s) < g.per_row) ++g.s;
  // 2^(32+s)/per_row lies in [2^32, 2^33): its excess over 2^32 is kept
  g.m = (uint32_t)((((1ull << g.s) - g.per_row) << 32) / g.per_row + 1);
  return g;
}
__device__ __forceinline__ void group_at(const GroupList& g, uint32_t i, uint32_t& row, uint32_t& col) {
  const uint32_t t = __umulhi(i, g.m);
  row = (t + ((i - t) >> 1)) >> (g.s - 1);   // s >= 2: per_row is at least 4
  col = (i - row * g.per_row) * C8_GROUP;
}

constexpr int C8_THREADS = 256, C8_UNROLL = 4;

struct C8Rounding {  // kernel argument: resolved to a C8Round on the device
  int stochastic, keep_sign;
  unsigned long long s1, step;
  uint32_t cols;
};
__device__ __forceinline__ C8Round c8_round(const C8Rounding& a) {
  C8Round r;
  r.stochastic = a.stochastic, r.keep_sign = a.keep_sign;
  r.cols = a.cols;
  const uint64_t s2 = a.stochastic ? splitmix64(a.s1 ^ a.step) : 0ull;
  r.key.k0 = (uint32_t)s2, r.key.k1 = (uint32_t)(s2 >> 32);
  return r;
}

// Reads one value and writes 33/32 of a byte for it.
template <typename T, int A>
__global__ void __launch_bounds__(C8_THREADS) ckpt8_save_kernel(const T* __restrict__ x, long long ld_x, int cols, GroupList gl,
                                                                C8View c, C8Rounding ra, uint32_t* __restrict__ status) {
  const C8Round rd = c8_round(ra);
  const uint32_t i0 = blockIdx.x * (C8_THREADS * C8_UNROLL) + threadIdx.x;
  Raw8<T> raw[C8_UNROLL];
  uint32_t row[C8_UNROLL], col[C8_UNROLL];
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const uint32_t i = i0 + u * C8_THREADS;
    group_at(gl, i, row[u], col[u]);
    raw[u] = load8<T, A>(x + (long long)row[u] * ld_x + col[u], i < gl.total ? cols - (int)col[u] : 0);
  }
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const bool in = i0 + u * C8_THREADS < gl.total;
    float v[8];
    unpack8(raw[u], v);
    uint2 codes;
    const int n = in ? cols - (int)col[u] : 0;
    const uint32_t e = c8_encode(v, row[u], col[u], rd, codes);
    if (n > 0) c8_store(c, row[u], (int)col[u], codes, e, status);
  }
}

__device__ __forceinline__ void clamp_finite(float (&v)[8], float) {}
__device__ __forceinline__ void clamp_finite(float (&v)[8], __nv_bfloat16) {}
// code * 2^E can pass the largest half (its block's maximum rounds up): kept finite.  NaN stays.
__device__ __forceinline__ void clamp_finite(float (&v)[8], __half) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (fabsf(v[j]) > 65504.0f) v[j] = copysignf(65504.0f, v[j]);
}

template <typename T, int A>
__global__ void __launch_bounds__(C8_THREADS) ckpt8_restore_kernel(C8View c, int cols, GroupList gl, T* __restrict__ y, long long ld_y) {
  const uint32_t i0 = blockIdx.x * (C8_THREADS * C8_UNROLL) + threadIdx.x;
  uint2 codes[C8_UNROLL];
  uint32_t e[C8_UNROLL], row[C8_UNROLL], col[C8_UNROLL];
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const uint32_t i = i0 + u * C8_THREADS;
    group_at(gl, i, row[u], col[u]);
    if (i < gl.total && (int)col[u] < cols) {
      codes[u] = __ldcs(reinterpret_cast<const uint2*>(c.q + (long long)row[u] * c.ld_q + col[u]));
      e[u] = c.e[(long long)row[u] * c.ld_e + col[u] / C8_BLOCK];
    } else {
      col[u] = (uint32_t)cols;
    }
  }
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const int n = cols - (int)col[u];
    if (n <= 0) continue;
    float v[8];
    c8_decode(codes[u], e[u], v);
    clamp_finite(v, T());
    store8<T, A>(y + (long long)row[u] * ld_y + col[u], pack8(v, T()), n);
  }
}

// ---- activations -----------------------------------------------------------------------------
constexpr int ACT_RELU = 0, ACT_GELU = 1, ACT_SILU = 2;

__device__ __forceinline__ float ex2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Logistic function from e = e^-|h| <= 1 (no overflow).  e^x = 2^(x log2(e)): the product is kept in two terms, its own rounding error
// and the part of log2(e) below FP32's last place (Dekker's product with a constant in two parts, as Cody and Waite reduce arguments), so
// that large |h| keep their digits; the second term enters as 1 + its size.  -1e30 stands for -Inf, whose terms would cancel to NaN (a NaN comes back through the callers' h).
__device__ __forceinline__ float logistic(float h) {
  const float x = fmaxf(-fabsf(h), -1e30f);
  const float t = x * 1.44269504f;
  const float low = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -t));
  float e = ex2_approx(t);
  e = fmaf(e, low * 0.693147181f, e);
  const float r = rcp_approx(1.0f + e);
  return h > 0.0f ? r : e * r;
}
// Normal distribution: E = e^(-h^2/2) and Phi(h).  The upper tail is 0.5 erfc(x / sqrt(2)) = t q(t) E with t = 1 / (1 + 0.34 x), x = |h|;
// q is a least-maximum fit of degree 6 to erfcx(x / sqrt(2)) / (2 t) on 0 <= x <= 13 (relative error 9e-8 at x = 0, growing as
// tail^-0.15), so that one division and one power of two serve the value and the slope.  In FP32 Phi is within 2e-7.
__device__ __forceinline__ float normal_cdf(float h, float& E) {
  const float x = fabsf(h);
  const float t = rcp_approx(fmaf(0.34f, x, 1.0f));
  float q = fmaf(0.0460086847f, t, -0.205629741f);
  q = fmaf(q, t, 0.273061343f);
  q = fmaf(q, t, -0.0389607225f);
  q = fmaf(q, t, 0.16070922f);
  q = fmaf(q, t, 0.128676757f);
  q = fmaf(q, t, 0.136134426f);
  E = ex2_approx(h * h * -0.721347520f);   // log2(e) / 2
  const float tail = q * t * E;
  return h > 0.0f ? 1.0f - tail : tail;
}

template <int KIND>
__device__ __forceinline__ float act_value(float h) {
  if (KIND == ACT_RELU) return h > 0.0f ? h : (h == h ? 0.0f : h);
  if (KIND == ACT_GELU) {
    float E;
    return h * normal_cdf(h, E);
  }
  return h * logistic(h);
}
template <int KIND>
__device__ __forceinline__ float act_slope(float h) {
  if (KIND == ACT_RELU) return h > 0.0f ? 1.0f : (h == h ? 0.0f : h);
  if (KIND == ACT_GELU) {
    float E;
    const float phi = normal_cdf(h, E);
    return fmaf(h * 0.39894228f, E, phi);
  }
  const float sig = logistic(h);
  return sig * fmaf(h, 1.0f - sig, 1.0f);
}

// z = act(h) in the tensor's type (z may be h itself); ch / cz (q nullable): checkpoints of h and of z as stored.
template <typename T, int KIND, int A>
__global__ void __launch_bounds__(C8_THREADS) act_forward_kernel(const T* h, long long ld_h, T* z,
                                                                 long long ld_z, int cols, GroupList gl, C8View ch, C8View cz,
                                                                 C8Rounding rh, C8Rounding rz, uint32_t* __restrict__ status) {
  const C8Round rdh = c8_round(rh), rdz = c8_round(rz);
  const uint32_t i0 = blockIdx.x * (C8_THREADS * C8_UNROLL) + threadIdx.x;
  Raw8<T> raw[C8_UNROLL];
  uint32_t row[C8_UNROLL], col[C8_UNROLL];
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const uint32_t i = i0 + u * C8_THREADS;
    group_at(gl, i, row[u], col[u]);
    raw[u] = load8<T, A>(h + (long long)row[u] * ld_h + col[u], i < gl.total ? cols - (int)col[u] : 0);
  }
#pragma unroll
  for (int u = 0; u < C8_UNROLL; ++u) {
    const int n = i0 + u * C8_THREADS < gl.total ? cols - (int)col[u] : 0;
    float v[8], a[8];
    unpack8(raw[u], v);
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = act_value<KIND>(v[j]);
    const Raw8<T> out = pack8(a, T());
    if (z && n > 0) store8<T, A>(z + (long long)row[u] * ld_z + col[u], out, n);
    uint2 codes;
    if (ch.q) {
      const uint32_t e = c8_encode(v, row[u], col[u], rdh, codes);
      if (n > 0) c8_store(ch, row[u], (int)col[u], codes, e, status);
    }
    if (cz.q) {
      unpack8(out, a);
      const uint32_t e = c8_encode(a, row[u], col[u], rdz, codes);
      if (n > 0) c8_store(cz, row[u], (int)col[u], codes, e, status);
    }
  }
}

// dh = dz * act'(h), h from its checkpoint.  dh may be dz itself.
// A code and an exponent decide the slope: the slopes of the 256 codes for exponents -13 .. 4 (blocks whose maximum lies
// between 2^-7 and 2^11) stand in a table that each CTA computes with the same function, so a value costs a table read
// instead of some 20 operations (229 us against 318 at 32768 x 8192 bfloat16, where HBM needs 206).  Other exponents are computed.
constexpr uint32_t ACT_E0 = 114, ACT_TABLES = 18;
template <typename T, int KIND, int A>
__global__ void __launch_bounds__(C8_THREADS) act_backward_kernel(const T* dz, long long ld_dz, C8View ch, T* dh, long long ld_dh, int cols,
                                                                  GroupList gl) {
  __shared__ float table[KIND == ACT_RELU ? 1 : ACT_TABLES * 256];
  if (KIND != ACT_RELU) {
    for (uint32_t k = threadIdx.x; k < ACT_TABLES * 256; k += C8_THREADS)
      table[k] = act_slope<KIND>((float)(int8_t)(k & 255u) * c8_scale(ACT_E0 + (k >> 8)));
    __syncthreads();
  }
  for (uint32_t i0 = blockIdx.x * (C8_THREADS * C8_UNROLL) + threadIdx.x; i0 < gl.total + threadIdx.x; i0 += gridDim.x * (C8_THREADS * C8_UNROLL)) {
    Raw8<T> raw[C8_UNROLL];
    uint2 codes[C8_UNROLL];
    uint32_t e[C8_UNROLL], row[C8_UNROLL], col[C8_UNROLL];
#pragma unroll
    for (int u = 0; u < C8_UNROLL; ++u) {
      const uint32_t i = i0 + u * C8_THREADS;
      group_at(gl, i, row[u], col[u]);
      if (i >= gl.total || (int)col[u] >= cols) {
        col[u] = (uint32_t)cols;
        continue;
      }
      raw[u] = load8<T, A>(dz + (long long)row[u] * ld_dz + col[u], cols - (int)col[u]);
      codes[u] = __ldcs(reinterpret_cast<const uint2*>(ch.q + (long long)row[u] * ch.ld_q + col[u]));
      e[u] = ch.e[(long long)row[u] * ch.ld_e + col[u] / C8_BLOCK];
    }
#pragma unroll
    for (int u = 0; u < C8_UNROLL; ++u) {
      const int n = cols - (int)col[u];
      if (n <= 0) continue;
      float v[8], g[8];
      unpack8(raw[u], g);
      if (KIND != ACT_RELU && e[u] - ACT_E0 < ACT_TABLES) {
        const float* const of = table + (e[u] - ACT_E0) * 256;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = of[__byte_perm(codes[u].x, 0u, 0x4440 + j)], v[4 + j] = of[__byte_perm(codes[u].y, 0u, 0x4440 + j)];
      } else {
        c8_decode(codes[u], e[u], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = act_slope<KIND>(v[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(g[j], v[j]);
      store8<T, A>(dh + (long long)row[u] * ld_dh + col[u], pack8(g, T()), n);
    }
  }
}

}  // namespace ffi8
