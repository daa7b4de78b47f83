// aps_ckpt.hip -- activation checkpoints in 8 bits: saving and loading them,
// and the activation's gradient at a checkpointed pre-activation.
//
// A wave works within one block of 32 rows x 128 columns, so that the block's
// exponent is a scalar.  A lane takes 16 bytes of the activations' type at a
// time (8 or 4 elements), a wave 4 or 2 rows; its loads are all issued before
// the first is used.  Saving reads each element once and keeps it in
// registers between the block's maximum and the cast.
#include "aps_linear.hpp"

namespace aps {

namespace {

constexpr int CTHREADS = 256;
constexpr int LOAD_STEPS = 2;
constexpr int SAVE_WAVES = CTHREADS / 64;

struct CkArgs {
    const void* X;  // save: the activations; act_grad: dY
    int64_t ldx;
    void* out;      // load: the activations; act_grad: dZ
    int64_t ldo;
    uint8_t* codes;
    int64_t ldc;
    int32_t* exps;
    int64_t M, C;
    int32_t act;
};

// One lane's place in its wave's block.
template <class T>
struct Walk {
    static constexpr int E = 16 / (int)sizeof(T);      // elements of a lane's share of a row
    static constexpr int LANES = CK_COLS / E;          // lanes of a row
    static constexpr int STEP = 64 / LANES;            // rows at a time
    static constexpr int STEPS = CK_ROWS / STEP;
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> word_t;
    typedef word_t bits __attribute__((ext_vector_type(E)));
    static constexpr word_t MAGNITUDE = (word_t)~((word_t)1 << (8 * sizeof(T) - 1));
    static __device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(word_t, (T)v); }
    static __device__ __forceinline__ float value_of(uint32_t b) { return (float)__builtin_bit_cast(T, (word_t)b); }
    int64_t row, col, have;
    int64_t block;
    // the wave's rows of a block that `waves` waves share
    __device__ __forceinline__ bool place(const CkArgs& a, int waves) {
        const int64_t nb = (a.C + CK_COLS - 1) / CK_COLS;
        const int64_t k = (int64_t)blockIdx.x * (CTHREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t rows = k / nb;  // neighbouring waves take neighbouring columns
        const int64_t r0 = rows * (CK_ROWS / waves);
        block = r0 / CK_ROWS * nb + k % nb;
        const int lane = threadIdx.x & 63;
        row = r0 + lane / LANES;
        col = k % nb * CK_COLS + lane % LANES * E;
        have = a.C - col;
        return r0 < a.M;
    }
    // the same where a workgroup's waves share its block
    __device__ __forceinline__ void place_shared(const CkArgs& a) {
        const int64_t nb = (a.C + CK_COLS - 1) / CK_COLS;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        block = blockIdx.x;
        row = block / nb * CK_ROWS + wave * (CK_ROWS / SAVE_WAVES) + lane / LANES;
        col = block % nb * CK_COLS + lane % LANES * E;
        have = a.C - col;
    }
};

// A lane's E elements at p; VEC: rows are aligned for all of them at once.
template <class T, bool VEC>
__device__ __forceinline__ typename Walk<T>::vec load_share(const T* p, int64_t have) {
    if (VEC && have >= Walk<T>::E) return *(const typename Walk<T>::vec*)p;
    typename Walk<T>::vec v = {};
#pragma unroll
    for (int i = 0; i < Walk<T>::E; ++i)
        if (i < have) v[i] = p[i];
    return v;
}

template <int E>
struct CodeVec;
template <>
struct CodeVec<4> {
    typedef uint32_t type;
    static __device__ __forceinline__ uint32_t word(type v, int) { return v; }
};
template <>
struct CodeVec<8> {
    typedef u2v type;
    static __device__ __forceinline__ uint32_t word(type v, int i) { return v[i]; }
};

template <class T, bool VEC>
__device__ __forceinline__ typename CodeVec<Walk<T>::E>::type load_share_codes(const uint8_t* p, int64_t have) {
    typedef typename CodeVec<Walk<T>::E>::type C;
    if (VEC && have >= Walk<T>::E) return *(const C*)p;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < Walk<T>::E; ++i)
        if (i < have) w[i / 4] |= (uint32_t)p[i] << (i % 4 * 8);
    if constexpr (Walk<T>::E == 8)
        return C{w[0], w[1]};
    else
        return w[0];
}

// The waves of a workgroup share a block, 8 rows each: 33 x 1001 fp32 takes 4.4
// us, with a block to a wave 8.6; 16384 x 4096 bf16 39.6 (5.1 TB/s, a large
// copy's rate) and 40.2.
template <class T, bool E5, bool VEC>
__global__ __launch_bounds__(CTHREADS) void k_ckpt_save(CkArgs a) {
    typedef Walk<T> Wk;
    constexpr int E = Wk::E;
    constexpr float lim = ck_limit<T, E5>();
    constexpr int STEPS = Wk::STEPS / SAVE_WAVES;
    __shared__ uint32_t red[2][SAVE_WAVES];
    const int wave = threadIdx.x >> 6;
    Wk w;
    w.place_shared(a);
    typename Wk::vec x[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int64_t r = w.row + s * Wk::STEP;
        x[s] = load_share<T, VEC>((const T*)a.X + r * a.ldx + w.col, r < a.M ? w.have : 0);
    }
    // the maximum on the magnitudes' bits, in which the values order
    typename Wk::bits top = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
        top = __builtin_elementwise_max(top, __builtin_bit_cast(typename Wk::bits, x[s]) & Wk::MAGNITUDE);
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) mx = max(mx, (uint32_t)top[i]);
#pragma unroll
    for (int o = 32; o; o >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o));
    if ((threadIdx.x & 63) == 0) red[0][wave] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SAVE_WAVES; ++i) mx = max(mx, red[0][i]);
    mx = __builtin_amdgcn_readfirstlane(mx);
    // INF, NaN or more than lim in the block: each element is looked at
    const bool careful = mx > Wk::bits_of(lim);
    mx = f2u(Wk::value_of(mx));
    if (careful) {
        mx = 0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < E; ++i) mx = ck_max_join(mx, ck_max_bits(ck_clamp((float)x[s][i], lim)));
        mx = ck_wave_max(mx);
        if ((threadIdx.x & 63) == 0) red[1][wave] = mx;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SAVE_WAVES; ++i) mx = ck_max_join(mx, red[1][i]);
    }
    const int32_t word = ck_word(mx, ck_emax<E5>());
    if (threadIdx.x == 0) a.exps[w.block] = word;
    const float up = pow2_of(ck_ft(word));
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int64_t r = w.row + s * Wk::STEP;
        if (r >= a.M) break;
        uint32_t c[2] = {0, 0};
#pragma unroll
        for (int g = 0; g < E / 4; ++g) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (float)x[s][4 * g + i];
            if (careful) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = ck_clamp(v[i], lim) * up;
                c[g] = ck_encode4<E5>(v);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] *= up;
                c[g] = ck_encode4_finite<E5>(v);
            }
        }
        uint8_t* o = a.codes + r * a.ldc + w.col;
        if (VEC && w.have >= E) {
            if constexpr (E == 8)
                *(u2v*)o = u2v{c[0], c[1]};
            else
                *(uint32_t*)o = c[0];
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < w.have) o[i] = (uint8_t)(c[i / 4] >> (i % 4 * 8));
        }
    }
}

// GRAD: out = X * act'(z); otherwise out = act(z), z the checkpoint's values.
// 16384 x 4096 bf16 loads in 30 us, and GELU's gradient of 8192 x 4096 takes 31
// (5.4 TB/s): bound by HBM; a few rows by latency, 4 us.  In fp32 GELU's 33
// operations bound it: 8192 x 4096 loads in 41 us, its gradient takes 52.
// A wave takes LOAD_STEPS of a block's steps: nothing ties the rows together,
// and more waves hide the activations' arithmetic and a few rows' latency.
template <class T, bool E5, bool VEC, bool GRAD>
__global__ __launch_bounds__(CTHREADS) void k_ckpt_load(CkArgs a) {
    typedef Walk<T> Wk;
    constexpr int E = Wk::E;
    Wk w;
    if (!w.place(a, Wk::STEPS / LOAD_STEPS)) return;
    const int32_t word = a.exps[w.block];
    const float inv = pow2_of(-ck_ft(word));
    typename CodeVec<E>::type c[LOAD_STEPS];
    typename Wk::vec x[GRAD ? LOAD_STEPS : 1];
#pragma unroll
    for (int s = 0; s < LOAD_STEPS; ++s) {
        const int64_t r = w.row + s * Wk::STEP;
        const int64_t have = r < a.M ? w.have : 0;
        c[s] = load_share_codes<T, VEC>(a.codes + r * a.ldc + w.col, have);
        if constexpr (GRAD) x[s] = load_share<T, VEC>((const T*)a.X + r * a.ldx + w.col, have);
    }
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int s = 0; s < LOAD_STEPS; ++s) {
            const int64_t r = w.row + s * Wk::STEP;
            if (r >= a.M) break;
            typename Wk::vec y;
#pragma unroll
            for (int g = 0; g < E / 4; ++g) {
                float z[4];
                ck_decode4<E5>(CodeVec<E>::word(c[s], g), inv, word & CK_ODD, z);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[4 * g + i] = (T)(GRAD ? (float)x[GRAD ? s : 0][4 * g + i] * act_slope<act.value, exact_act<T>>(z[i])
                                            : act_value<act.value, exact_act<T>>(z[i]));
            }
            T* o = (T*)a.out + r * a.ldo + w.col;
            if (VEC && w.have >= E) {
                *(typename Wk::vec*)o = y;
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (i < w.have) o[i] = y[i];
            }
        }
    });
}

// `waves` of a block
dim3 grid_of(const CkArgs& a, int waves) {
    const int64_t blocks = ((a.M + CK_ROWS - 1) / CK_ROWS) * ((a.C + CK_COLS - 1) / CK_COLS) * waves;
    return dim3((unsigned)((blocks + CTHREADS / 64 - 1) / (CTHREADS / 64)));
}

// rows of `ld` elements of `bytes` from p, aligned for a lane's share at once
bool rows_of_shares(const void* p, int64_t ld, int64_t bytes, int64_t share) {
    return (uintptr_t)p % (uintptr_t)(bytes * share) == 0 && ld % share == 0;
}

#define APS_CK_TYPE(F, T, ...)                      \
    if (e5) {                                       \
        if (vec) F(T, true, true, __VA_ARGS__)      \
        else F(T, true, false, __VA_ARGS__)         \
    } else {                                        \
        if (vec) F(T, false, true, __VA_ARGS__)     \
        else F(T, false, false, __VA_ARGS__)        \
    }
#define APS_CK_TYPES(F, ...)                        \
    if (dtype == APS_DTYPE_BF16) {                  \
        APS_CK_TYPE(F, __bf16, __VA_ARGS__)         \
    } else if (dtype == APS_DTYPE_F16) {            \
        APS_CK_TYPE(F, _Float16, __VA_ARGS__)       \
    } else {                                        \
        APS_CK_TYPE(F, float, __VA_ARGS__)          \
    }
#define APS_CK_SAVE(T, e, v, ...) { hipLaunchKernelGGL((k_ckpt_save<T, e, v>), __VA_ARGS__); }
#define APS_CK_LOAD(T, e, v, ...) { hipLaunchKernelGGL((k_ckpt_load<T, e, v, false>), __VA_ARGS__); }
#define APS_CK_GRAD(T, e, v, ...) { hipLaunchKernelGGL((k_ckpt_load<T, e, v, true>), __VA_ARGS__); }

}  // namespace

}  // namespace aps

using namespace aps;

extern "C" int aps_checkpoint_save(const void* X, int64_t ldx, int32_t M, int32_t C, int32_t dtype, aps_format fmt,
                                   uint8_t* codes, int64_t ldc, int32_t* ckpt_exp, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, C, 0, dtype));
    const int es = lin_elem_bytes(dtype), share = 16 / es;
    bool e5 = false;
    APS_LIN_TRY(lin_check_matrix(X, ldx, M, C, es));
    APS_LIN_TRY(lin_check_checkpoint(fmt, codes, ldc, ckpt_exp, M, C, e5));
    if (M == 0 || C == 0) return APS_OK;
    const CkArgs a{X, ldx, nullptr, 0, codes, ldc, ckpt_exp, M, C, APS_ACT_NONE};
    const bool vec = rows_of_shares(X, ldx, es, share) && rows_of_shares(codes, ldc, 1, share);
    APS_CK_TYPES(APS_CK_SAVE, grid_of(a, SAVE_WAVES), dim3(CTHREADS), 0, (hipStream_t)stream, a)
    return launched();
}

extern "C" int aps_checkpoint_load(const uint8_t* codes, int64_t ldc, const int32_t* ckpt_exp, int32_t M, int32_t C,
                                   aps_format fmt, int32_t act, void* X, int64_t ldx, int32_t dtype, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, C, 0, dtype));
    if (!lin_act_known(act)) return APS_ERR_UNSUPPORTED;
    const int es = lin_elem_bytes(dtype), share = 16 / es;
    bool e5 = false;
    APS_LIN_TRY(lin_check_checkpoint(fmt, codes, ldc, ckpt_exp, M, C, e5));
    APS_LIN_TRY(lin_check_matrix(X, ldx, M, C, es));
    if (M == 0 || C == 0) return APS_OK;
    const CkArgs a{nullptr, 0, X, ldx, (uint8_t*)codes, ldc, (int32_t*)ckpt_exp, M, C, act};
    const bool vec = rows_of_shares(X, ldx, es, share) && rows_of_shares(codes, ldc, 1, share);
    APS_CK_TYPES(APS_CK_LOAD, grid_of(a, CK_ROWS / (64 / (CK_COLS / share)) / LOAD_STEPS), dim3(CTHREADS), 0, (hipStream_t)stream, a)
    return launched();
}

extern "C" int aps_activation_grad(const void* dY, int64_t lddy, int32_t act, aps_format fmt, const uint8_t* codes,
                                   int64_t ldc, const int32_t* ckpt_exp, void* dZ, int64_t lddz, int32_t M, int32_t C,
                                   int32_t dtype, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, C, 0, dtype));
    if (!lin_act_known(act)) return APS_ERR_UNSUPPORTED;
    const int es = lin_elem_bytes(dtype), share = 16 / es;
    bool e5 = false;
    APS_LIN_TRY(lin_check_matrix(dY, lddy, M, C, es));
    APS_LIN_TRY(lin_check_checkpoint(fmt, codes, ldc, ckpt_exp, M, C, e5));
    APS_LIN_TRY(lin_check_matrix(dZ, lddz, M, C, es));
    if (M == 0 || C == 0) return APS_OK;
    const CkArgs a{dY, lddy, dZ, lddz, (uint8_t*)codes, ldc, (int32_t*)ckpt_exp, M, C, act};
    const bool vec = rows_of_shares(dY, lddy, es, share) && rows_of_shares(dZ, lddz, es, share) &&
                     rows_of_shares(codes, ldc, 1, share);
    APS_CK_TYPES(APS_CK_GRAD, grid_of(a, CK_ROWS / (64 / (CK_COLS / share)) / LOAD_STEPS), dim3(CTHREADS), 0, (hipStream_t)stream, a)
    return launched();
}
