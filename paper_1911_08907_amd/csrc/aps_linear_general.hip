// aps_linear_general.hip -- the linear layer's products for any type,
// alignment and length, and the join of a split contraction.
//
// k_lin_general: a workgroup of four waves forms a tile of 128 p x 64 q, each
// wave 64 x 32 of it in two 32 x 32 accumulators.  The contraction is staged
// 64 bytes deep: elements are read one by one with their bounds checked (zero
// outside), converted where the operand is a checkpoint, and laid along the
// contraction in LDS, whose rows of 64 + 16 bytes spread the 16-byte fragment
// reads over the banks.  A fragment's 16 bytes are one 16-bit matrix
// instruction's eight contraction elements, or four fp32 instructions' one.
// The next stage's elements are in flight while the present ones multiply.
// 77 x 777 x 1001 fp32 in seven pieces takes 15.8 us, bound by a stage's latency.
#include "aps_linear.hpp"

namespace aps {

namespace {

constexpr int GP = 128, GQ = 64;  // a workgroup's tile
constexpr int GTHREADS = 256;

template <class T>
struct Frag;
template <>
struct Frag<__bf16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x16 mma(bf16x8 p, bf16x8 q, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(p, q, c, 0, 0, 0);
    }
};
template <>
struct Frag<_Float16> {
    typedef f16x8 type;
    static __device__ __forceinline__ f32x16 mma(f16x8 p, f16x8 q, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(p, q, c, 0, 0, 0);
    }
};
template <>
struct Frag<float> {
    typedef f32x4 type;
    static __device__ __forceinline__ f32x16 mma(f32x4 p, f32x4 q, f32x16 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(p[i], q[i], c, 0, 0, 0);
        return c;
    }
};

// One stage of an operand of R rows: each thread's share of its R x BK elements.
template <class T, int R, bool ALONG>
struct Stage {
    static constexpr int BK = 64 / (int)sizeof(T);
    static constexpr int N = R * BK / GTHREADS;
    static constexpr int LDS_ROW = BK + 16 / (int)sizeof(T);
    T v[N];

    // thread t's n-th element: its row and its place in the stage
    static __device__ __forceinline__ int row(int n) {
        return ALONG ? (int)threadIdx.x / BK + n * (GTHREADS / BK) : (int)threadIdx.x % R;
    }
    static __device__ __forceinline__ int at(int n) {
        return ALONG ? (int)threadIdx.x % BK : (int)threadIdx.x / R + n * (GTHREADS / R);
    }
    __device__ __forceinline__ void read(const T* base, int64_t ld, int64_t r0, int64_t nr, int64_t c0, int64_t nc) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int64_t r = r0 + row(n), c = c0 + at(n);
            v[n] = (r < nr && c < nc) ? (ALONG ? base[r * ld + c] : base[c * ld + r]) : (T)0.0f;
        }
    }
    // the codes of a checkpoint, [c][r]; the stage lies in one block of rows,
    // the tile in one block of columns
    template <bool E5>
    __device__ __forceinline__ void read_codes(const uint8_t* base, int64_t ld, const int32_t* exps, int64_t r0,
                                               int64_t nr, int64_t c0, int64_t nc) {
        static_assert(!ALONG, "the contraction runs over a checkpoint's rows");
        const int64_t nb = (nr + CK_COLS - 1) / CK_COLS;
        const int32_t word = c0 < nc ? exps[(c0 / CK_ROWS) * nb + r0 / CK_COLS] : 0;
        const float inv = pow2_of(-ck_ft(word));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int64_t r = r0 + row(n), c = c0 + at(n);
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (r < nr && c < nc) ck_decode4<E5>(base[c * ld + r], inv, word & CK_ODD, d);
            v[n] = (T)d[0];
        }
    }
    __device__ __forceinline__ void write(T* lds) const {
#pragma unroll
        for (int n = 0; n < N; ++n) lds[row(n) * LDS_ROW + at(n)] = v[n];
    }
};

template <class T, int OP, bool E5>
__global__ __launch_bounds__(GTHREADS) void k_lin_general(LinArgs a) {
    typedef Stage<T, GP, OP == OP_FWD> SP;
    typedef Stage<T, GQ, OP != OP_DW> SQ;
    constexpr int BK = SP::BK, ROW = SP::LDS_ROW;
    __shared__ __align__(16) T lp[GP * ROW];
    __shared__ __align__(16) T lq[GQ * ROW];
    __shared__ uint32_t red[GTHREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wp = wave & 1, wq = wave >> 1;
    const int64_t tp = (a.np + GP - 1) / GP, tq = (a.nq + GQ - 1) / GQ;
    const int64_t tile = blockIdx.x % (tp * tq), piece = blockIdx.x / (tp * tq);
    const int64_t p0 = (tile % tp) * GP, q0 = (tile / tp) * GQ;
    const int64_t cb = piece * a.piece, ce = min(a.nc, cb + a.piece);

    SP sp;
    SQ sq;
    const auto read = [&](int64_t c) {
        if constexpr (OP == OP_DW)
            sp.template read_codes<E5>((const uint8_t*)a.P, a.ldp, a.zexps, p0, a.np, c, ce);
        else
            sp.read((const T*)a.P, a.ldp, p0, a.np, c, ce);
        sq.read((const T*)a.Q, a.ldq, q0, a.nq, c, ce);
    };
    f32x16 acc[2] = {};
    float db = 0.0f;
    const bool sums = OP == OP_DW && a.dbias && p0 == 0;
    if (cb < ce) read(cb);
    for (int64_t c = cb; c < ce; c += BK) {
        __syncthreads();
        sp.write(lp);
        sq.write(lq);
        __syncthreads();
        if (c + BK < ce) read(c + BK);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            typedef typename Frag<T>::type F;
            const int at = (k * 32 + (lane >> 5) * 16) / (int)sizeof(T);
            const F q = *(const F*)(lq + (wq * 32 + (lane & 31)) * ROW + at);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                acc[i] = Frag<T>::mma(*(const F*)(lp + (wp * 64 + i * 32 + (lane & 31)) * ROW + at), q, acc[i]);
        }
        if (sums && threadIdx.x < GQ)
            for (int k = 0; k < BK; ++k) db += (float)lq[threadIdx.x * ROW + k];
    }

    const int64_t q = q0 + wq * 32 + (lane & 31);
    const int64_t pl = p0 + wp * 64 + (lane >> 5) * 4;  // of accumulator i's group g: + 32 i + 8 g
    if (a.split > 1) {
        if (q < a.nq) {
            float* o = a.part + (piece * a.nq + q) * a.ldpart;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t p = pl + 8 * i;
                if (p < a.ldpart)  // ldpart is a multiple of 4
                    *(f32x4*)(o + p) = f32x4{acc[i / 4][i % 4 * 4], acc[i / 4][i % 4 * 4 + 1], acc[i / 4][i % 4 * 4 + 2],
                                            acc[i / 4][i % 4 * 4 + 3]};
            }
        }
        if (sums && threadIdx.x < GQ && q0 + threadIdx.x < a.nq) a.part_bias[piece * a.nq + q0 + threadIdx.x] = db;
        return;
    }
    if (sums && threadIdx.x < GQ && q0 + threadIdx.x < a.nq) {
        float* o = a.dbias + q0 + threadIdx.x;
        *o = a.accumulate ? *o + db : db;
    }
    if constexpr (OP == OP_FWD) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float b[4];
            lin_bias4<T>(a, pl + 8 * i, a.np - pl - 8 * i, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i / 4][i % 4 * 4 + e] += b[e];
        }
        if (a.codes) {
            uint32_t mx = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (q < a.nq && pl + 8 * (i / 4) + i % 4 < a.np)
                    mx = ck_max_join(mx, ck_max_bits(ck_clamp(acc[i / 16][i % 16], ck_limit<T, E5>())));
            mx = ck_wave_max(mx);
            if (lane == 0) red[wave] = mx;
            __syncthreads();
            const int32_t word = ck_word(ck_max_join(red[2 * wq], red[2 * wq + 1]), ck_emax<E5>());
            const int64_t qb = q0 / CK_ROWS + wq;
            if (wp == 0 && lane == 0 && qb * CK_ROWS < a.nq)
                a.exps[qb * ((a.np + CK_COLS - 1) / CK_COLS) + p0 / CK_COLS] = word;
            if (q < a.nq)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z[4] = {acc[i / 4][i % 4 * 4], acc[i / 4][i % 4 * 4 + 1], acc[i / 4][i % 4 * 4 + 2],
                                        acc[i / 4][i % 4 * 4 + 3]};
                    lin_save4<T, E5>(a, q, pl + 8 * i, a.np - pl - 8 * i, word, z);
                }
        }
    }
    if (q < a.nq)
        with_act(OP == OP_DW ? APS_ACT_NONE : a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t p = pl + 8 * i;
                const float v[4] = {acc[i / 4][i % 4 * 4], acc[i / 4][i % 4 * 4 + 1], acc[i / 4][i % 4 * 4 + 2],
                                    acc[i / 4][i % 4 * 4 + 3]};
                if (p >= a.np) break;
                LinRead<T, OP, 4> in;
                in.read(a, q, p, a.np - p);
                lin_finish<T, OP, E5, 4, act.value>(a, in, q, p, a.np - p, v);
            }
        });
}

// The sum of a split contraction's pieces, in their order, and the epilogue:
// a workgroup finishes one checkpoint block of 32 q x 128 p, a thread four p.
// Four pieces of 4096 x 1024 take 14 us (84 MB, 6 TB/s); with four rows to a
// thread, seven pieces of 77 x 777 took 17 us, now 7.
constexpr int JTHREADS = 1024;

template <class T, int OP, bool E5>
__global__ __launch_bounds__(JTHREADS) void k_lin_join(LinArgs a) {
    __shared__ uint32_t red[JTHREADS / 64];
    const int64_t tp = (a.np + CK_COLS - 1) / CK_COLS;
    const int64_t pb = blockIdx.x % tp, qb = blockIdx.x / tp;
    const int64_t p = pb * CK_COLS + threadIdx.x % 32 * 4, q = qb * CK_ROWS + threadIdx.x / 32;
    const int64_t have = q < a.nq ? a.np - p : 0;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    LinRead<T, OP, 4> in;
    in.read(a, q, p, have);
    if (have > 0) {
        const int64_t step = a.nq * a.ldpart;
        const float* x = a.part + q * a.ldpart + p;
        int s = 0;
        for (; s + 4 <= a.split; s += 4, x += 4 * step) {  // four pieces in flight
            const f32x4 x0 = *(const f32x4*)x, x1 = *(const f32x4*)(x + step), x2 = *(const f32x4*)(x + 2 * step),
                        x3 = *(const f32x4*)(x + 3 * step);
            v = (((v + x0) + x1) + x2) + x3;
        }
        for (; s < a.split; ++s, x += step) v += *(const f32x4*)x;
    }
    if (OP == OP_FWD) {
        float b[4];
        lin_bias4<T>(a, p, have, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += b[e];
    }
    if (OP == OP_DW && a.dbias && pb == 0 && threadIdx.x < 32 && qb * CK_ROWS + threadIdx.x < a.nq) {
        const int64_t r = qb * CK_ROWS + threadIdx.x;
        float db = 0.0f;
        for (int s = 0; s < a.split; ++s) db += a.part_bias[s * a.nq + r];
        a.dbias[r] = a.accumulate ? a.dbias[r] + db : db;
    }
    int32_t word = 0;
    if (OP == OP_FWD && a.codes) {
        uint32_t mx = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) mx = ck_max_join(mx, ck_max_bits(ck_clamp(v[e], ck_limit<T, E5>())));
        mx = ck_wave_max(mx);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = mx;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < JTHREADS / 64; ++w) mx = ck_max_join(mx, red[w]);
        word = ck_word(mx, ck_emax<E5>());
        if (threadIdx.x == 0) a.exps[qb * tp + pb] = word;
    }
    if (have <= 0) return;
    const float z[4] = {v[0], v[1], v[2], v[3]};
    if (OP == OP_FWD && a.codes) lin_save4<T, E5>(a, q, p, have, word, z);
    with_act(OP == OP_DW ? APS_ACT_NONE : a.act,
             [&](auto act) { lin_finish<T, OP, E5, 4, act.value>(a, in, q, p, have, z); });
}

}  // namespace

// Pieces of the contraction: where the tiles are fewer than two workgroups
// per CU, enough pieces for that many, of at least 128 contraction elements:
// up to 512.  The time in us: a launch and the first stage's way in; per stage of
// 64 bytes its latency or its share for each tile at work; for a split the join's
// launch, its serial sum and the partial sums' way out and in.  Fitted to graph
// replays of 480 products, half of them with rows off their chunks, beside the
// other kernels: two stages take 8.7, 118 x 2307 of 7669 in 13 pieces 41, 8000 x
// 4095 of 4095 894, bf16; a weight gradient of 4868 rows, 256 x 3264, 234; 21568
// in 168 pieces, fp32, 32.
LinTile lin_general(int op, int64_t np, int64_t nq, int64_t nc, bool f32) {
    static const struct {
        double stage, share;
    } plain[] = {{1.3, 0.0025}, {1.1, 0.0036}}, decodes[] = {{3.3, 0.0115}, {2.1, 0.0073}};
    const auto& m = (op == OP_DW ? decodes : plain)[f32];
    const int64_t tiles = ((np + GP - 1) / GP) * ((nq + GQ - 1) / GQ);
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(tiles, 1), nc / 128));
    const int64_t stages = (nc + (f32 ? 15 : 31)) / (f32 ? 16 : 32);
    const double us = 6.5 + std::ceil((double)stages / split) * std::max(m.stage, m.share * tiles * split) +
                      (split > 1 ? 2.0 + 0.08 * split + (double)split * np * nq * 8 / 6.0e6 : 0.0);
    return {LIN_SMALL, (int)split, us};
}

#define APS_LIN_TYPES(K, ...)                                              \
    if (dtype == APS_DTYPE_BF16) {                                         \
        APS_LIN_OPS(K, __bf16, __VA_ARGS__)                                \
    } else if (dtype == APS_DTYPE_F16) {                                   \
        APS_LIN_OPS(K, _Float16, __VA_ARGS__)                              \
    } else {                                                               \
        APS_LIN_OPS(K, float, __VA_ARGS__)                                 \
    }

void launch_lin_general(int op, int dtype, bool e5, const LinArgs& a, hipStream_t s) {
    const int64_t tiles = ((a.np + GP - 1) / GP) * ((a.nq + GQ - 1) / GQ);
    const dim3 grid((unsigned)(tiles * a.split));
    APS_LIN_TYPES(k_lin_general, grid, dim3(GTHREADS), 0, s, a)
}

void launch_lin_join(int op, int dtype, bool e5, const LinArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)(((a.np + CK_COLS - 1) / CK_COLS) * ((a.nq + CK_ROWS - 1) / CK_ROWS)));
    APS_LIN_TYPES(k_lin_join, grid, dim3(JTHREADS), 0, s, a)
}

}  // namespace aps
