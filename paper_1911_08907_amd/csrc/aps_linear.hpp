// aps_linear.hpp -- device code shared by the linear layer's kernels on
// gfx950: the activations and their derivatives, the 8-bit activation
// checkpoints, and the epilogues of the products.
//
// A checkpoint holds blocks of 32 rows x 128 columns.  As in Algorithm 1 (the
// power-of-two scale from a maximum, then the cast; Sec. 3.3.3) each block's
// exponent is ft = emax - ceil(log2 max), so that the largest magnitude
// lands in the format's top binade without overflow; blocks instead of whole
// layers, since one token's outliers should not cost every other token its
// precision.  32 rows are two steps of a 16-bit matrix instruction's
// contraction, so that the weight gradient, which contracts over the rows,
// decodes with one scalar exponent per step.
//
// Every product keeps its accumulators in fp32; the result is rounded once,
// when it is stored in its type.
#pragma once

#include <type_traits>

#include "aps_common.hpp"
#include "aps_linear.h"

namespace aps {

enum LinOp : int32_t { OP_FWD = APS_LINEAR_FORWARD, OP_DX = APS_LINEAR_GRAD_INPUT, OP_DW = APS_LINEAR_GRAD_WEIGHT };

constexpr int CK_ROWS = APS_CKPT_ROWS, CK_COLS = APS_CKPT_COLS, CK_MAX_FT = APS_CKPT_MAX_EXP;
constexpr int CK_ODD = 1 << 16;  // a block's exponent word: the block has an INF or NaN

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ------------------------------------------------------------------ types

template <class T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

template <class T>
struct TypeEmax {
    static constexpr int value = 127;
};
template <>
struct TypeEmax<_Float16> {
    static constexpr int value = 15;
};

// Four consecutive values at an address aligned for all four.
template <class T>
__device__ __forceinline__ void load4(const T* p, float v[4]) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    const t4 t = *(const t4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
}
template <class T>
__device__ __forceinline__ void store4(T* p, const float v[4]) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    t4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
    *(t4*)p = t;
}

// Up to four values of a row at p, those below `have`; `vec`: the row is
// aligned for four at once.
template <class T>
__device__ __forceinline__ void load_some(const T* p, int64_t have, bool vec, float v[4]) {
    if (vec && have >= 4) {
        load4(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < have ? (float)p[i] : 0.0f;
}
template <class T>
__device__ __forceinline__ void store_some(T* p, int64_t have, bool vec, const float v[4]) {
    if (vec && have >= 4) {
        store4(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) p[i] = (T)v[i];
}
__device__ __forceinline__ uint32_t load_codes4(const uint8_t* p, int64_t have, bool vec) {
    if (vec && have >= 4) return *(const uint32_t*)p;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) w |= (uint32_t)p[i] << (8 * i);
    return w;
}
__device__ __forceinline__ void store_some_codes(uint8_t* p, int64_t have, bool vec, uint32_t w) {
    if (vec && have >= 4) {
        *(uint32_t*)p = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) p[i] = (uint8_t)(w >> (8 * i));
}

// ------------------------------------------------------------ activations
//
// GELU: with h = 1 - Phi(|z|) = erfc(|z| / sqrt 2) / 2,
//   z Phi(z) = max(z, 0) - |z| h,   Phi(z) + z phi(z) = (z < 0 ? h : 1 - h) + z phi(z)
// so that both tails keep h's relative accuracy.  exp(z^2 / 2) h falls slowly,
// from 1/2 at 0 like 0.399 / |z|: it is t times a polynomial in t = 1 / (1 + p |z|),
// whose coefficients were fitted to it over |z| <= 14.5 (beyond, h is below
// fp32's range), and phi is the same exponential.  SiLU: the logistic function by
// one exponential and one reciprocal.
//
// EXACT, for fp32 results: ten terms, fitted for the least relative error (1.3e-8),
// the exponent's roundings carried into the exponential, the reciprocal refined:
// GELU comes out within 3.9e-7 of itself, SiLU 2.8e-7 (over N(0, 1) by norm 3.1e-8
// and 4.6e-8; z (1 + erf) / 2 in fp32 has 3.7e-8 and loses the lower tail).
// Otherwise the result is rounded to 16 bits: six terms, as close where h is large
// (2.2e-7 of h and 1) and within 2.3e-5 relative in the tail, a twentieth of a
// half's rounding; the exponent's roundings stay, 1e-5 of the result at most.
// rcp and exp2 are the hardware's, off by one ulp; exp2 takes a result
// below 2^-126 as zero, so that SiLU below -87.3 (1e-36) is zero.
//
// The limits at +-INF are the functions' own: the factor |z|, or z, that would
// meet a zero is held to where the result is exact already.  NaN stays NaN.

// exp2(y + off) of a small off
__device__ __forceinline__ float exp2_of(float y, float off) {
    return __builtin_amdgcn_exp2f(y) * __builtin_fmaf(off, 0.69314718f, 1.0f);
}
// 1 / d for d in [1, 2^100]
__device__ __forceinline__ float rcp_refined(float d) {
    const float r = __builtin_amdgcn_rcpf(d);
    return __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
}
// |z|, at most lim; NaN stays
__device__ __forceinline__ float magnitude_to(float z, float lim) {
    const float a = __builtin_fabsf(z);
    return a > lim ? lim : a;
}

struct Tail {
    float h, e;  // 1 - Phi(|z|), exp(-z^2 / 2)
};
template <bool EXACT>
__device__ __forceinline__ Tail normal_tail(float z) {
    if constexpr (EXACT) {
        const float a = magnitude_to(z, 15.0f), s = a * a;  // exp(-15^2 / 2) is zero already
        const float t = rcp_refined(__builtin_fmaf(0.375f, a, 1.0f));
        // z^2 / 2 log2(e) = y + off: the square's rounding, the product's, the constant's
        constexpr float c = 0.721347511f, c_lo = 9.62981517e-09f;
        const float y = s * -c;
        const float off = __builtin_fmaf(__builtin_fmaf(a, a, -s), -c, __builtin_fmaf(s, -c_lo, __builtin_fmaf(s, -c, -y)));
        const float e = exp2_of(y, off);
        float w = __builtin_fmaf(0.0208993945f, t, -0.134001285f);
        w = __builtin_fmaf(w, t, 0.344836205f);
        w = __builtin_fmaf(w, t, -0.424009472f);
        w = __builtin_fmaf(w, t, 0.215563744f);
        w = __builtin_fmaf(w, t, -0.0561585128f);
        w = __builtin_fmaf(w, t, 0.108109742f);
        w = __builtin_fmaf(w, t, 0.125283062f);
        w = __builtin_fmaf(w, t, 0.14988403f);
        w = __builtin_fmaf(w, t, 0.14959307f);
        return {w * t * e, e};
    } else {
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, __builtin_fabsf(z), 1.0f));
        const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
        float w = __builtin_fmaf(-0.0788610998f, t, 0.220412575f);
        w = __builtin_fmaf(w, t, -0.0207146197f);
        w = __builtin_fmaf(w, t, 0.14547459f);
        w = __builtin_fmaf(w, t, 0.1136206f);
        w = __builtin_fmaf(w, t, 0.120067733f);
        return {w * t * e, e};
    }
}

// The logistic function of z and of -z.
struct Logistic {
    float s, u;
};
// EXACT: from exp(-|z|), which neither overflows nor cancels.
template <bool EXACT>
__device__ __forceinline__ Logistic logistic(float z) {
    if constexpr (EXACT) {
        constexpr float c = 1.44269502f, c_lo = 1.92596303e-08f;
        const float a = magnitude_to(z, 104.0f), y = a * -c;
        const float e = exp2_of(y, __builtin_fmaf(a, -c_lo, __builtin_fmaf(a, -c, -y)));
        const float r = rcp_refined(1.0f + e), q = e * r;
        return {z < 0.0f ? q : r, z < 0.0f ? r : q};
    } else {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return {s, 1.0f - s};
    }
}

template <int ACT, bool EXACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == APS_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == APS_ACT_GELU)
        return __builtin_fmaf(-__builtin_fminf(__builtin_fabsf(z), 15.0f), normal_tail<EXACT>(z).h, __builtin_fmaxf(z, 0.0f));
    if constexpr (ACT == APS_ACT_SILU) return (z < -104.0f ? -104.0f : z) * logistic<EXACT>(z).s;
    return z;
}

template <int ACT, bool EXACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == APS_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if constexpr (ACT == APS_ACT_GELU) {
        const Tail n = normal_tail<EXACT>(z);
        return __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -15.0f, 15.0f), n.e * 0.39894228f, z < 0.0f ? n.h : 1.0f - n.h);
    }
    if constexpr (ACT == APS_ACT_SILU) {
        const Logistic l = logistic<EXACT>(z);
        return l.s * __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -104.0f, 104.0f), l.u, 1.0f);
    }
    return 1.0f;
}

// whether results of type T take the EXACT form
template <class T>
constexpr bool exact_act = sizeof(T) == 4;

// f(std::integral_constant<int, ACT>) of a call's activation: one copy of the
// code each, chosen once.
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case APS_ACT_RELU: f(std::integral_constant<int, APS_ACT_RELU>()); break;
        case APS_ACT_GELU: f(std::integral_constant<int, APS_ACT_GELU>()); break;
        case APS_ACT_SILU: f(std::integral_constant<int, APS_ACT_SILU>()); break;
        default: f(std::integral_constant<int, APS_ACT_NONE>()); break;
    }
}

// ------------------------------------------------------------ checkpoints

// The largest format value, times a power of two, that T holds; the format's emax.
template <class T, bool E5>
constexpr float ck_limit() {
    return (E5 ? 1.75f : 1.875f) * (TypeEmax<T>::value == 15 ? 0x1p15f : 0x1p127f);
}
template <bool E5>
constexpr int ck_emax() {
    return E5 ? 15 : 7;
}

// A finite magnitude at most lim, the largest format value that T holds;
// INF and NaN stay.
__device__ __forceinline__ float ck_clamp(float x, float lim) {
    return __builtin_fabsf(x) < __builtin_inff() ? __builtin_amdgcn_fmed3f(x, -lim, lim) : x;
}

// A block's maximum as an unsigned word: the largest finite magnitude's bits,
// and in bit 31 whether an element is INF or NaN.
__device__ __forceinline__ uint32_t ck_max_bits(float x) {
    const uint32_t a = f2u(x) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0x80000000u;
}
__device__ __forceinline__ uint32_t ck_max_join(uint32_t a, uint32_t b) {
    return max(a & 0x7FFFFFFFu, b & 0x7FFFFFFFu) | ((a | b) & 0x80000000u);
}

// The block's exponent word from its maximum.
__device__ __forceinline__ int32_t ck_word(uint32_t mx, int emax) {
    const uint32_t a = mx & 0x7FFFFFFFu;
    const int ft = a ? min(emax - ceil_log2_bits(a), CK_MAX_FT) : 0;
    return (ft & 0xFFFF) | ((mx >> 31) ? CK_ODD : 0);
}
__device__ __forceinline__ int ck_ft(int32_t word) { return (int)(int16_t)word; }

// 2^e; the exponents of a block are within +-126 of zero
__device__ __forceinline__ float pow2_of(int e) { return u2f((uint32_t)(e + 127) << 23); }

// The codes of four scaled values.
template <bool E5>
__device__ __forceinline__ uint32_t ck_encode4(const float v[4]) {
    if constexpr (E5) return encode4_e5m2(v[0], v[1], v[2], v[3]);
    return encode4_e4m3(v[0], v[1], v[2], v[3]);
}

// The same for finite values within the format's largest magnitude.
template <bool E5>
__device__ __forceinline__ uint32_t ck_encode4_finite(const float v[4]) {
    if constexpr (E5)
        return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_bf8_f32(v[0], v[1], 0, false), true);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), true);
}

// 1-4-3's INF and NaN among four codes: v where a code is one.
__device__ __forceinline__ void ck_odd_e4m3(uint32_t w, float v[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (w >> (8 * i)) & 0x7Fu;
        if (c >= 0x78u) v[i] = c > 0x78u ? __builtin_nanf("") : __builtin_copysignf(__builtin_inff(), v[i]);
    }
}

// The values of four codes of a block.  inv = 2^-ft.
template <bool E5>
__device__ __forceinline__ void ck_decode4(uint32_t w, float inv, bool odd, float v[4]) {
    f32x2 lo, hi;
    if constexpr (E5) {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8(w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8(w, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    }
    v[0] = lo[0] * inv;
    v[1] = lo[1] * inv;
    v[2] = hi[0] * inv;
    v[3] = hi[1] * inv;
    if (!E5 && odd) ck_odd_e4m3(w, v);
}

// ------------------------------------------------------------- a product
//
// Every product is out[q][p] = sum over c of P[p][c] * Q[q][c], p the output's
// contiguous axis: P is the weights or the checkpoint's codes, Q the
// activations or the output gradients.  P and Q say where the contraction
// runs in memory: along a row (contiguous), or from row to row.
//
//   forward      out Y  [M][N]: p = n, q = m, c = k: P = W along rows, Q = X along rows
//   grad_input   out dX [M][K]: p = k, q = m, c = n: P = W row to row, Q = dZ along rows
//   grad_weight  out dW [N][K]: p = k, q = n, c = m: P = codes row to row, Q = dZ row to row

// which rows are aligned for four elements at once
enum LinVec : uint32_t { LV_OUT = 1, LV_R = 2, LV_CODES = 4, LV_BIAS = 8, LV_ZC = 16 };

struct LinArgs {
    const void* __restrict__ P;  // weights, or codes
    const void* __restrict__ Q;
    int64_t ldp, ldq;            // row strides in elements
    int64_t np, nq, nc;          // p, q and contraction lengths
    const void* bias;            // forward, or NULL
    const void* R;               // added residual, or NULL; may be out
    int64_t ldr;
    void* out;
    int64_t ldo;
    uint8_t* codes;              // forward: the checkpoint of z, or NULL
    int64_t ldcodes;
    int32_t* exps;               // its blocks' exponent words
    const uint8_t* zc;           // grad_input: the checkpoint of z, or NULL
    int64_t ldzc;
    const int32_t* zexps;        // ... its exponent words (grad_weight: those of P)
    float* dbias;                // grad_weight, or NULL
    float* part;                 // split products: partial sums [split][nq][ldpart]
    float* part_bias;            // ... of dbias [split][nq]
    int64_t ldpart;
    int32_t act;
    int32_t split;               // pieces of the contraction
    int64_t piece;               // contraction length of one
    uint32_t vec;                // LinVec
    uint32_t accumulate;         // grad_weight: add to out
};

// A wave's join of its lanes' block maxima, in every lane.
__device__ __forceinline__ uint32_t ck_wave_max(uint32_t m) {
#pragma unroll
    for (int o = 32; o; o >>= 1) m = ck_max_join(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

// What the epilogue reads besides the sums, for N consecutive p of row q.
template <class T, int OP, int N>
struct LinRead {
    typedef T t4 __attribute__((ext_vector_type(4)));
    t4 r[OP == OP_DW ? 1 : N / 4];
    uint32_t c[OP == OP_DX ? N / 4 : 1];
    int32_t word;
    static __device__ __forceinline__ t4 load_raw(const T* s, int64_t have, bool vec) {
        if (vec && have >= 4) return *(const t4*)s;
        t4 v = {};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) v[i] = s[i];
        return v;
    }
    // the first `have` of the N; p within one block of columns
    __device__ __forceinline__ void read(const LinArgs& a, int64_t q, int64_t p, int64_t have) {
        if constexpr (OP != OP_DW) {
            if (a.R)
#pragma unroll
                for (int i = 0; i < N; i += 4) r[i / 4] = load_raw((const T*)a.R + q * a.ldr + p + i, have - i, a.vec & LV_R);
        }
        if constexpr (OP == OP_DX) {
            word = 0;
            if (a.zc) {
#pragma unroll
                for (int i = 0; i < N; i += 4) c[i / 4] = load_codes4(a.zc + q * a.ldzc + p + i, have - i, a.vec & LV_ZC);
                if (have > 0) word = a.zexps[(q / CK_ROWS) * ((a.np + CK_COLS - 1) / CK_COLS) + p / CK_COLS];
            }
        }
    }
};

// The stored result of N consecutive p of row q (the first `have` of them),
// v being the finished sums: bias already added in the forward pass.
template <class T, int OP, bool E5, int N, int ACT>
__device__ __forceinline__ void lin_finish(const LinArgs& a, const LinRead<T, OP, N>& in, int64_t q, int64_t p, int64_t have,
                                           const float v[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float y[4];
        if constexpr (OP == OP_DW) {
            float* o = (float*)a.out + q * a.ldo + p + i;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = 0.0f;
            if (a.accumulate) load_some(o, have - i, a.vec & LV_OUT, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = a.accumulate ? y[e] + v[i + e] : v[i + e];
            store_some(o, have - i, a.vec & LV_OUT, y);
            continue;
        }
        if constexpr (OP == OP_FWD) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = act_value<ACT, exact_act<T>>(v[i + e]);
        } else if constexpr (OP == OP_DX) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = v[i + e];
            if constexpr (ACT != APS_ACT_NONE) {
                float z[4];
                ck_decode4<E5>(in.c[i / 4], pow2_of(-ck_ft(in.word)), in.word & CK_ODD, z);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] *= act_slope<ACT, exact_act<T>>(z[e]);
            }
        }
        if constexpr (OP != OP_DW) {
            if (a.R)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += (float)in.r[i / 4][e];
            store_some((T*)a.out + q * a.ldo + p + i, have - i, a.vec & LV_OUT, y);
        }
    }
}

template <class T>
__device__ __forceinline__ void lin_bias4(const LinArgs& a, int64_t p, int64_t have, float b[4]) {
    if (a.bias)
        load_some((const T*)a.bias + p, have, a.vec & LV_BIAS, b);
    else
        b[0] = b[1] = b[2] = b[3] = 0.0f;
}

// The codes of four values of z at row q, with the block's word known.
template <class T, bool E5>
__device__ __forceinline__ void lin_save4(const LinArgs& a, int64_t q, int64_t p, int64_t have, int32_t word, const float z[4]) {
    constexpr float lim = ck_limit<T, E5>();
    const float s = pow2_of(ck_ft(word));
    float v[4];
    uint32_t c;
    if (word & CK_ODD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ck_clamp(z[i], lim) * s;
        c = ck_encode4<E5>(v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_fmed3f(z[i], -lim, lim) * s;
        c = ck_encode4_finite<E5>(v);
    }
    store_some_codes(a.codes + q * a.ldcodes + p, have, a.vec & LV_CODES, c);
}

// ------------------------------------------------------------ host checks

constexpr int64_t LIN_MAX_LD = (1LL << 31) - 1;
constexpr int64_t LIN_MAX_BLOCKS = 1 << 22;  // blocks of 32 x 128: a launch's size stays within HIP's

static inline int lin_elem_bytes(int dtype) { return dtype == APS_DTYPE_F32 ? 4 : 2; }

static inline bool lin_aligned(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

static inline bool lin_act_known(int act) { return act >= APS_ACT_NONE && act <= APS_ACT_SILU; }

static inline bool lin_too_large(int64_t cols, int64_t rows) {
    return ((cols + CK_COLS - 1) / CK_COLS) * ((rows + CK_ROWS - 1) / CK_ROWS) > LIN_MAX_BLOCKS;
}

// Of a product (M, N, K), or of a matrix (M, N, 0).
static inline int lin_check_dims(int32_t M, int32_t N, int32_t K, int32_t dtype) {
    if (M < 0 || N < 0 || K < 0 || M > APS_MAX_GEMM_DIM || N > APS_MAX_GEMM_DIM || K > APS_MAX_GEMM_DIM)
        return APS_ERR_SIZE;
    if (lin_too_large(N, M) || lin_too_large(K, M) || lin_too_large(K, N)) return APS_ERR_SIZE;
    if (dtype != APS_DTYPE_F32 && dtype != APS_DTYPE_BF16 && dtype != APS_DTYPE_F16) return APS_ERR_UNSUPPORTED;
    return APS_OK;
}

// A matrix of rows x cols elements of `bytes`; nothing is asked of an empty one.
static inline int lin_check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int bytes) {
    if (rows == 0 || cols == 0) return APS_OK;
    if (!p) return APS_ERR_NULL;
    if (ld < cols || ld > LIN_MAX_LD) return APS_ERR_SIZE;
    return lin_aligned(p, bytes) ? APS_OK : APS_ERR_ALIGN;
}

static inline int lin_check_checkpoint(aps_format f, const void* codes, int64_t ldc, const void* exps, int64_t rows,
                                       int64_t cols, bool& e5) {
    int st = fmt_status(f);
    if (st != APS_OK) return st;
    const int hw = make_fmtk(f).hw;
    if (hw != HW_E5M2 && hw != HW_E4M3) return APS_ERR_UNSUPPORTED;
    e5 = hw == HW_E5M2;
    st = lin_check_matrix(codes, ldc, rows, cols, 1);
    if (st != APS_OK) return st;
    if (rows == 0 || cols == 0) return APS_OK;
    if (!exps) return APS_ERR_NULL;
    return lin_aligned(exps, 4) ? APS_OK : APS_ERR_ALIGN;
}

#define APS_LIN_TRY(x)                   \
    do {                                 \
        const int st_ = (x);             \
        if (st_ != APS_OK) return st_;   \
    } while (0)

// ------------------------------------------------------------ the launches

// dtype is one of APS_DTYPE_*; the format is 1-5-2 (e5) or 1-4-3.
void launch_lin_general(int op, int dtype, bool e5, const LinArgs& a, hipStream_t s);
void launch_lin_join(int op, int dtype, bool e5, const LinArgs& a, hipStream_t s);

constexpr int LIN_FEW = 32;  // rows that the decode kernel takes at most
void launch_lin_decode(int dtype, bool fast, const LinArgs& a, hipStream_t s);
// Its time in us; fast: rows of whole chunks that start on them.
double lin_decode_us(int64_t np, int64_t nq, int64_t nc, bool f32, bool fast);

// One operand's copy into aligned rows (src NULL: none).
struct LinCopy {
    const void* src;
    void* dst;
    int64_t lds, ldd, rows, cols;  // row strides in elements; ldd is whole 16-byte chunks
    int32_t elem;                  // bytes
};
void launch_lin_align(const LinCopy& p, const LinCopy& q, hipStream_t s);
double lin_align_us(uint64_t bytes);  // of copies that take `bytes`

// A choice for an output and a contraction: the tile kernel's shape, the pieces
// of the contraction, and the model's time in us.
enum LinShape : int32_t { LIN_BIG, LIN_MIDDLE, LIN_SMALL };
struct LinTile {
    int shape, split;
    double us;
};
LinTile lin_tile(int op, int64_t np, int64_t nq, int64_t nc, bool f32);
LinTile lin_general(int op, int64_t np, int64_t nq, int64_t nc, bool f32);
void launch_lin_tile(int op, int dtype, bool e5, int shape, const LinArgs& a, hipStream_t s);

}  // namespace aps

// Launch kernel K of the operator and format.
#define APS_LIN_OPS(K, T, ...)                                                              \
    switch (op * 2 + (e5 ? 1 : 0)) {                                                        \
        case OP_FWD * 2: hipLaunchKernelGGL((K<T, OP_FWD, false>), __VA_ARGS__); break;     \
        case OP_FWD * 2 + 1: hipLaunchKernelGGL((K<T, OP_FWD, true>), __VA_ARGS__); break;  \
        case OP_DX * 2: hipLaunchKernelGGL((K<T, OP_DX, false>), __VA_ARGS__); break;       \
        case OP_DX * 2 + 1: hipLaunchKernelGGL((K<T, OP_DX, true>), __VA_ARGS__); break;    \
        case OP_DW * 2: hipLaunchKernelGGL((K<T, OP_DW, false>), __VA_ARGS__); break;       \
        default: hipLaunchKernelGGL((K<T, OP_DW, true>), __VA_ARGS__); break;               \
    }
