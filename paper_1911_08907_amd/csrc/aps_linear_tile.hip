// aps_linear_tile.hip -- the linear layer's products of operands whose rows
// are aligned to 16 bytes.
//
// A workgroup forms a tile of 256 p x 256 q with eight waves (two on each
// SIMD), 128 x 128 with four, or 128 x 64 with four; each wave two by four, two
// or one 32 x 32 accumulators.  The contraction is staged 128 bytes
// deep (64 c of a 16-bit type, 32 of fp32) in two buffers of LDS that the loads fill directly.  A stage's loads are issued
// in the first half of the stage before, so one barrier per stage suffices: it
// says both that the stage has landed and that the other buffer is read out.
// Within a stage a fragment is read one of four steps before its products.
//
// In LDS a stage lies as it does in memory, each 16-byte chunk of a row at a
// place exclusive-ored with a few bits of the row, which the loading lane
// chooses by the chunk it asks for:
//   along rows   [rows][128 bytes]: a fragment is one 16-byte read per lane;
//                chunk ^ (row / 2) & 7 gives 16 lanes 64 different banks
//   row to row   [c][p]: a fragment is two transposing reads of 4 c x 16 p per
//                16 lanes; chunk ^ 4 (c & 3) gives 32 lanes all banks.  fp32: four
//                reads of one c x 32 p; chunk ^ 8 (c / 8 & 1) parts the halves
//   codes        [c][p] bytes: one transposing read of 8 c x 16 p per 16
//                lanes, chunk ^ 2 (c & 7) (rows of 256; half of that for 128);
//                then four conversions of two codes, with the block's power of
//                two, to the matrix type: exact
// An fp32 step is 8 c by four instructions of 2: a lane's half h holds 4 c from
// 16 (s / 2) + 8 h + 4 (s & 1) on in step s, so that two steps are one read of codes.
//
// Measured, bf16: 16384 x 1024 x 4096 forward 116 us (1.18 PFLOP/s; the matrix
// units 55 % busy at the 2.0 GHz that their power leaves), 4096 x 4096 x 1024
// 37, with GELU and a checkpoint 54; the weight gradient of 16384 x 4096 x 1024 127
// us in four pieces.  With every load a hit in L2 8192^3 gains 9 %, without LDS
// reads 5 %: neither alone bounds it.  fp32 4096 x 4096 x 1024 252 us, 136 TFLOP/s.
// Elements past an operand's end are read as zero by the buffer loads' own
// range check, through an offset that is out of range.
#include "aps_linear.hpp"

namespace aps {

namespace {

template <class T>
constexpr int TK_OF = 128 / (int)sizeof(T);  // contraction elements of a stage

// FQ accumulators of 32 q by two of 32 p a wave, WP x WQ waves.
template <int FQ_, int WP_, int WQ_>
struct Shape {
    static constexpr int FQ = FQ_, WP = WP_, WQ = WQ_;
    static constexpr int WAVES = WP * WQ, THREADS = 64 * WAVES, TP = 64 * WP, TQ = 32 * FQ * WQ;
};
typedef Shape<4, 4, 2> Big;     // 256 p x 256 q
typedef Shape<2, 2, 2> Middle;  // 128 x 128
typedef Shape<1, 2, 2> Small;   // 128 x 64

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;  // as a byte offset; the loads' range ends there
constexpr int WAIT_LOADS = 0x0F70;              // s_waitcnt vmcnt(0)

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

#define APS_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))

template <class T>
struct Mat;
template <>
struct Mat<__bf16> {
    typedef bf16x8 frag;
    static __device__ __forceinline__ f32x16 mma(frag p, frag q, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(p, q, c, 0, 0, 0);
    }
    template <bool E5, bool HI>
    static __device__ __forceinline__ uint32_t two(uint32_t w, float inv) {
        if constexpr (E5) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, inv, HI));
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, inv, HI));
    }
    static constexpr uint32_t INF = 0x7F80u, NAN_ = 0x7FC0u;
    static __device__ __forceinline__ float add2(uint32_t w, float s) {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, s, false);
    }
};
template <>
struct Mat<_Float16> {
    typedef f16x8 frag;
    static __device__ __forceinline__ f32x16 mma(frag p, frag q, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(p, q, c, 0, 0, 0);
    }
    template <bool E5, bool HI>
    static __device__ __forceinline__ uint32_t two(uint32_t w, float inv) {
        if constexpr (E5) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, inv, HI));
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, inv, HI));
    }
    static constexpr uint32_t INF = 0x7C00u, NAN_ = 0x7E00u;
    static __device__ __forceinline__ float add2(uint32_t w, float s) {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.0f, (_Float16)1.0f}, s, false);
    }
};

template <>
struct Mat<float> {
    typedef f32x4 frag;
    static __device__ __forceinline__ f32x16 mma(frag p, frag q, f32x16 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(p[i], q[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ float add2(uint32_t w, float s) { return s + u2f(w); }
};

enum Kind { ALONG, ACROSS, CODES };

// What the place of a row-to-row operand's chunk is exclusive-ored with, in
// chunks: R elements of ELEM bytes a row.  Rows shorter than the 256 bytes of
// the banks take turns by themselves.
template <int R, int ELEM>
__device__ __forceinline__ int across_xor(int c) {
    constexpr int PER = 256 / (R * ELEM) > 1 ? 256 / (R * ELEM) : 1;  // rows of 256 bytes
    if constexpr (ELEM == 4) return (c / 8 & 1) * 8;
    if constexpr (ELEM == 1) return (c / PER & (8 / PER - 1)) * 2;
    return (c / PER & (4 / PER - 1)) * 4;
}

// One operand's R rows (p or q): what a lane loads.
template <class T, Kind KIND, int R, int WAVES>
struct Operand {
    static constexpr int ELEM = KIND == CODES ? 1 : sizeof(T), TK = TK_OF<T>;
    static constexpr int BYTES = R * TK * ELEM;  // of a stage
    static constexpr int LOADS = BYTES / (WAVES * 1024);
    static_assert(LOADS * WAVES * 1024 == BYTES, "whole loads of every wave");
    const char* base;   // of the tile's first row and the stage's first c (scalar)
    int64_t step;       // bytes from stage to stage
    uint32_t off[LOADS];
    int c_of;           // along: the lane's c in a stage; across: its first row c
    int c_step;         // across: c from load to load

    __device__ __forceinline__ void place(const void* p, int64_t ld, int64_t r0, int64_t nr, int64_t c0) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if constexpr (KIND == ALONG) {
            base = (const char*)p + (r0 * ld + c0) * ELEM;
            step = TK * ELEM;
            const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
            c_of = chunk * (16 / ELEM);
            c_step = 0;
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                const int row = (WAVES * n + wave) * 8 + (lane >> 3);
                off[n] = r0 + row < nr ? (uint32_t)row * (uint32_t)(ld * ELEM) + chunk * 16 : OUT_OF_RANGE;
            }
        } else {
            constexpr int PER_ROW = R * ELEM / 16;        // chunks of a row
            constexpr int ROWS = 64 / PER_ROW;            // rows of one load
            base = (const char*)p + (c0 * ld + r0) * ELEM;
            step = TK * ld * ELEM;
            const int c = ROWS * wave + lane / PER_ROW;
            c_of = c;
            c_step = WAVES * ROWS;
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                const int chunk = (lane % PER_ROW) ^ across_xor<R, ELEM>(c + n * c_step);
                off[n] = r0 + chunk * (16 / ELEM) < nr
                             ? (uint32_t)(c + n * c_step) * (uint32_t)(ld * ELEM) + chunk * 16
                             : OUT_OF_RANGE;
            }
        }
    }
    // The n-th load of a stage into LDS; `left` c's are left, none or fewer
    // behind the contraction's end.
    __device__ __forceinline__ void load(char* lds, int n, int left) const {
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)OUT_OF_RANGE, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t o = c_of + n * c_step < left ? off[n] : OUT_OF_RANGE;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, APS_LDS(void, lds + (WAVES * n + wave) * 1024), 16, o, 0, 0, 0);
    }
    __device__ __forceinline__ void next() { base += step; }
};

// A wave's fragments of an operand: N of 32 rows each from row r on.  The places
// differ from fragment to fragment and from 16 c to 16 c by constants, but for
// the exclusive-or: along rows it depends on the 16 c, otherwise on the
// fragment's rows.
template <class T, Kind KIND, int R, int N>
struct Reader {
    static constexpr int BASES = KIND == ALONG ? 4 : N;
    int at[BASES];
    __device__ __forceinline__ void place(int r) {
        const int lane = threadIdx.x & 63, half = lane >> 5, i = lane & 15;
#pragma unroll
        for (int b = 0; b < BASES; ++b) {
            if constexpr (KIND == ALONG) {
                const int row = lane & 31;
                const int chunk = sizeof(T) == 4 ? b / 2 * 4 + half * 2 + b % 2 : 2 * b + half;
                at[b] = (r + row) * 128 + (chunk ^ ((row >> 1) & 7)) * 16;
            } else if constexpr (KIND == ACROSS && sizeof(T) == 4) {
                const int c = half * 8, p = r + 32 * b + (lane & 31);
                at[b] = c * (4 * R) + ((p >> 2) ^ across_xor<R, 4>(c)) * 16 + (p & 3) * 4;
            } else if constexpr (KIND == ACROSS) {
                const int c = half * 8 + (i >> 2), p = r + 32 * b + (lane & 16) + (i & 3) * 4;
                at[b] = c * (2 * R) + ((p >> 3) ^ across_xor<R, 2>(c)) * 16 + (p & 7) * 2;
            } else {
                const int c = half * 8 + (i >> 1), p = r + 32 * b + (lane & 16) + (i & 1) * 8;
                at[b] = c * R + ((p >> 4) ^ across_xor<R, 1>(c)) * 16 + (p & 15);
            }
        }
    }
    // fragment n of step s
    __device__ __forceinline__ typename Mat<T>::frag read(const char* lds, int n, int s) const {
        typedef typename Mat<T>::frag F;
        if constexpr (KIND == ALONG) return *(const F*)(lds + at[s] + n * 32 * 128);
        if constexpr (sizeof(T) == 4) {
            const char* p = lds + at[KIND == ALONG ? 0 : n] + (s / 2 * 16 + s % 2 * 4) * (4 * R);
            F v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *(const float*)(p + i * (4 * R));
            return v;
        }
        const char* p = lds + at[KIND == ALONG ? 0 : n] + s * 16 * (2 * R);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(APS_LDS(s16x4, p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(APS_LDS(s16x4, p + 4 * (2 * R)));
        struct { s16x4 a, b; } both = {lo, hi};
        return __builtin_bit_cast(F, both);
    }
    // fragment n's codes of the s-th 16 c
    __device__ __forceinline__ i32x2 read_codes(const char* lds, int n, int s) const {
        return __builtin_amdgcn_ds_read_tr8_b64_v2i32(APS_LDS(i32x2, lds + at[n] + s * 16 * R));
    }
};

template <class T, bool E5>
__device__ __forceinline__ typename Mat<T>::frag decode_fragment(i32x2 w, int32_t word, int s) {
    typedef Mat<T> M;
    const float inv = pow2_of(-ck_ft(word));
    if constexpr (sizeof(T) == 4) {
        float z[4];
        ck_decode4<E5>((uint32_t)w[s % 2], inv, word & CK_ODD, z);
        return f32x4{z[0], z[1], z[2], z[3]};
    } else {
        u4v v = {M::template two<E5, false>(w[0], inv), M::template two<E5, true>(w[0], inv),
                 M::template two<E5, false>(w[1], inv), M::template two<E5, true>(w[1], inv)};
        if (!E5 && (word & CK_ODD)) {  // the conversion knows no INF of 1-4-3
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = ((uint32_t)w[i / 4] >> (i % 4 * 8)) & 0xFFu, sh = i % 2 * 16;
                const uint32_t x = ((c & 0x80u) << 8) | ((c & 0x7Fu) > 0x78u ? M::NAN_ : M::INF);
                if ((c & 0x7Fu) >= 0x78u) v[i / 2] = (v[i / 2] & ~(0xFFFFu << sh)) | (x << sh);
            }
        }
        return __builtin_bit_cast(typename M::frag, v);
    }
}

// Which tile and piece a workgroup forms.  Workgroups go to the eight XCDs in
// turn, each with an L2 of its own: an XCD takes a run of consecutive tiles,
// and consecutive tiles fill strips of four q by all p, so that those at work
// at a time share their operands' rows.
struct TilePlace {
    int64_t p, q, piece;
};
__device__ __forceinline__ TilePlace tile_place(int64_t tp, int64_t tq) {
    const int64_t n = gridDim.x, b = blockIdx.x, xcd = b % 8, each = n / 8, more = n % 8;
    const int64_t k = xcd * each + min(xcd, more) + b / 8;
    const int64_t t = k % (tp * tq), strip = t / (4 * tp), first = strip * 4, high = min(tq - first, (int64_t)4);
    const int64_t in = t - strip * 4 * tp;
    return {in / high, first + in % high, k / (tp * tq)};
}

template <class T, int OP, bool E5, class S>
__global__ __launch_bounds__(S::THREADS, 2) void k_lin_tile(LinArgs a) {
    constexpr int FQ = S::FQ, WP = S::WP, TP = S::TP, TQ = S::TQ, TK = TK_OF<T>;
    constexpr Kind KP = OP == OP_FWD ? ALONG : (OP == OP_DX ? ACROSS : CODES);
    constexpr Kind KQ = OP == OP_DW ? ACROSS : ALONG;
    typedef Operand<T, KP, TP, S::WAVES> OpP;
    typedef Operand<T, KQ, TQ, S::WAVES> OpQ;
    typedef typename Mat<T>::frag F;
    // the epilogue turns a wave's accumulators through LDS, RF of its FQ at a time
    constexpr int RF = FQ < 2 ? FQ : 2, TURN = RF * 32 * 64 * 4;
    constexpr int STAGE = std::max(OpP::BYTES + OpQ::BYTES, S::WAVES * TURN / 2);
    __shared__ __align__(1024) char lds0[STAGE];
    __shared__ __align__(1024) char lds1[STAGE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave % WP, wq = wave / WP;
    const TilePlace at = tile_place((a.np + TP - 1) / TP, (a.nq + TQ - 1) / TQ);
    const int64_t p0 = at.p * TP, q0 = at.q * TQ, piece = at.piece;
    const int cb = (int)(piece * a.piece), ce = (int)min(a.nc, (piece + 1) * a.piece);

    OpP P;
    OpQ Q;
    P.place(a.P, a.ldp, p0, a.np, cb);
    Q.place(a.Q, a.ldq, q0, a.nq, cb);
    // the sums begin with the bias: p = 32 i + 8 g + 4 (lane / 32) + e of
    // accumulator i's element 4 g + e
    f32x16 acc[2][FQ];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f32x16 b = {};
        if (OP == OP_FWD && a.split == 1 && a.bias)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t p = p0 + wp * 64 + i * 32 + g * 8 + (lane >> 5) * 4;
                float v[4];
                lin_bias4<T>(a, p, a.np - p, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) b[4 * g + e] = v[e];
            }
#pragma unroll
        for (int j = 0; j < FQ; ++j) acc[i][j] = b;
    }
    // dbias: where it is asked for, the tiles of the first p sum Q's columns,
    // each wave those of one fragment
    const bool sums = OP == OP_DW && a.dbias && p0 == 0;
    float sum = 0.0f;
    Reader<T, KQ, TQ, 1> RS;
    RS.place(wq * (32 * FQ) + (wp < FQ ? wp : 0) * 32);

    Reader<T, KP, TP, 2> RP;
    Reader<T, KQ, TQ, FQ> RQ;
    RP.place(wp * 64);
    RQ.place(wq * (32 * FQ));
    const int64_t nb = (a.np + CK_COLS - 1) / CK_COLS, pb = min(p0 / CK_COLS + wp / 2, nb - 1);

    // a stage's loads go out with its first two steps
    constexpr auto first = [](int s, int loads) { return s < 2 ? s * loads / 2 : loads; };
    // One stage: the products of `use`, and in their shade the next stage's
    // loads into `fill` and each 16 c's fragments before they are needed.
    const auto stage = [&](char* __restrict fill, const char* __restrict use, int c) {
        __builtin_amdgcn_s_waitcnt(WAIT_LOADS);
        __syncthreads();
        const int left = ce - c - TK;
        int32_t word[2] = {0, 0};
        if constexpr (OP == OP_DW) {
            word[0] = cld(a.zexps, c / CK_ROWS * nb + pb);
            word[1] = cld(a.zexps, min(c / CK_ROWS + 1, (int)(a.nc - 1) / CK_ROWS) * nb + pb);
        }
        F p[2][2], q[2][FQ];
        // codes stay codes until their step, so that nothing waits for a read
        // just issued; fp32 has two steps from one read
        i32x2 codes[2][2];
        constexpr int per = sizeof(T) == 4 ? 2 : 1;
        const auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if constexpr (OP == OP_DW) {
                    if (s % per == 0) codes[s / per & 1][i] = RP.read_codes(use, i, s / per);
                } else {
                    p[s & 1][i] = RP.read(use, i, s);
                }
            }
#pragma unroll
            for (int j = 0; j < FQ; ++j) q[s & 1][j] = RQ.read(use + OpP::BYTES, j, s);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int n = first(s, OpP::LOADS); n < first(s + 1, OpP::LOADS); ++n) P.load(fill, n, left);
#pragma unroll
            for (int n = first(s, OpQ::LOADS); n < first(s + 1, OpQ::LOADS); ++n) Q.load(fill + OpP::BYTES, n, left);
            if (s < 3) read(s + 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (OP == OP_DW)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    p[s & 1][i] = decode_fragment<T, E5>(codes[s / per & 1][i], word[sizeof(T) == 4 ? 0 : s / 2], s);
#pragma unroll
            for (int j = 0; j < FQ; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][j] = Mat<T>::mma(p[s & 1][i], q[s & 1][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        P.next();
        Q.next();
        if (OP == OP_DW && sums) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const u4v w = __builtin_bit_cast(u4v, RS.read(use + OpP::BYTES, 0, s));
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = Mat<T>::add2(w[i], sum);
            }
        }
    };
    if (cb < ce) {
        const int left = ce - cb;
#pragma unroll
        for (int n = 0; n < OpP::LOADS; ++n) P.load(lds0, n, left);
#pragma unroll
        for (int n = 0; n < OpQ::LOADS; ++n) Q.load(lds0 + OpP::BYTES, n, left);
        P.next();
        Q.next();
    }
    for (int c = cb; c < ce; c += 2 * TK) {
        stage(lds1, lds0, c);
        if (c + TK < ce) stage(lds0, lds1, c + TK);
    }

    // accumulator [i][j]: q = its lane of 32, p = 4 elements of each 8, by the lane's half
    const int64_t ql = q0 + wq * (32 * FQ);
    if constexpr (OP == OP_DW) {
        sum += __shfl_xor(sum, 32);
        const int64_t q = ql + wp * 32 + lane;
        if (sums && wp < FQ && lane < 32 && q < a.nq) {
            if (a.split > 1)
                a.part_bias[piece * a.nq + q] = sum;
            else
                a.dbias[q] = a.accumulate ? a.dbias[q] + sum : sum;
        }
    }
    // the stages are read out, and the loads behind the contraction's end, which
    // write zeros, have written them
    __builtin_amdgcn_s_waitcnt(WAIT_LOADS);
    __syncthreads();
    int32_t word[FQ] = {};
    if constexpr (OP == OP_FWD) {
        if (a.codes) {
            // a block of 32 q x 128 p is two waves': its maximum goes by LDS
            uint32_t* red = (uint32_t*)lds0;
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
                float m = 0.0f, bad = 0.0f;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        m = __builtin_fmaxf(m, __builtin_fabsf(acc[i][j][e]));
                        bad = __builtin_fmaf(acc[i][j][e], 0.0f, bad);
                    }
                uint32_t mx = f2u(__builtin_fminf(m, ck_limit<T, E5>()));
                if (bad != 0.0f) {  // an INF or NaN: the maximum of the others
                    mx = 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            mx = ck_max_join(mx, ck_max_bits(ck_clamp(acc[i][j][e], ck_limit<T, E5>())));
                }
                mx = ck_wave_max(ql + j * 32 + (lane & 31) < a.nq ? mx : 0);
                if (lane == 0) red[wave * FQ + j] = mx;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
                word[j] = ck_word(ck_max_join(red[wave * FQ + j], red[(wave ^ 1) * FQ + j]), ck_emax<E5>());
                const int64_t qb = ql / CK_ROWS + j;
                if ((wp & 1) == 0 && lane == 0 && qb * CK_ROWS < a.nq && p0 + wp * 64 < a.np)
                    a.exps[qb * nb + p0 / CK_COLS + wp / 2] = word[j];
            }
            __syncthreads();
        }
    }
    // Each wave turns its accumulators through LDS of its own, 32 RF q x 64 p
    // at a time, so that eight lanes store a row's 64 p; a 16-byte chunk of row
    // q lies at chunk ^ q & 15.
    char* turn = (wave < S::WAVES / 2 ? lds0 : lds1) + wave % (S::WAVES / 2) * TURN;
    const int64_t p = p0 + wp * 64 + (lane & 7) * 8, have = a.np - p;
    with_act(OP == OP_DW || a.split > 1 ? APS_ACT_NONE : a.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < FQ / RF; ++r) {
            const int64_t qr = ql + r * (32 * RF);
            if (qr >= a.nq) break;
            LinRead<T, OP, 8> in[4 * RF];
            if (a.split == 1)
#pragma unroll
                for (int k = 0; k < 4 * RF; ++k) {
                    const int64_t q = qr + k * 8 + (lane >> 3);
                    in[k].read(a, q, p, q < a.nq ? have : 0);
                }
#pragma unroll
            for (int j = 0; j < RF; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f32x16& v = acc[i / 4][RF * r + j];
                    const int row = j * 32 + (lane & 31), chunk = (i / 4) * 8 + (i % 4) * 2 + (lane >> 5);
                    *(f32x4*)(turn + row * 256 + (chunk ^ (row & 15)) * 16) =
                        f32x4{v[i % 4 * 4], v[i % 4 * 4 + 1], v[i % 4 * 4 + 2], v[i % 4 * 4 + 3]};
                }
            wave_lds_sync();
#pragma unroll
            for (int k = 0; k < 4 * RF; ++k) {
                const int row = k * 8 + (lane >> 3);
                const int64_t q = qr + row;
                const f32x4 lo = *(const f32x4*)(turn + row * 256 + (((lane & 7) * 2) ^ (row & 15)) * 16);
                const f32x4 hi = *(const f32x4*)(turn + row * 256 + (((lane & 7) * 2 + 1) ^ (row & 15)) * 16);
                const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                if (q >= a.nq || have <= 0) continue;
                if (a.split > 1) {
                    float* o = a.part + (piece * a.nq + q) * a.ldpart + p;  // ldpart is a multiple of 4
                    *(f32x4*)o = lo;
                    if (have > 4) *(f32x4*)(o + 4) = hi;
                    continue;
                }
                if (OP == OP_FWD && a.codes) {
                    const int32_t wd = word[RF * r + k / 4];
                    lin_save4<T, E5>(a, q, p, have, wd, v);
                    lin_save4<T, E5>(a, q, p + 4, have - 4, wd, v + 4);
                }
                lin_finish<T, OP, E5, 8, act.value>(a, in[k], q, p, have, v);
            }
            wave_lds_sync();
        }
    });
}

}  // namespace

// The shape and the pieces of the contraction that a model of the time finds
// fastest, in us: a launch; per stage the latency of one tile's stage or,
// where more tiles are at work, their share of the GPU; per tile its epilogue;
// for a split the join's launch and the partial sums' way out and in.  The
// terms were fitted to graph replays of 40 products from 64 x 64 x 16384 to
// 16384 x 4096 x 1024, where the model's choice took at most 1.17 times the best
// of all shapes with 1 to 32 pieces (in us: 512 x 4096 x 1024 bf16, small 9.8, middle
// 12.1, big 27.8; 4096 x 4096 x 1024, small 50.5, middle 43.5, big 36.5; 64 x
// 1024 x 4096, small in 8 pieces 10.4, in 2 17.7).
LinTile lin_tile(int op, int64_t np, int64_t nq, int64_t nc, bool f32) {
    static const struct {
        int shape, tp, tq, fill;       // tiles at work at a time
        double launch, stage, decode;  // once; a stage alone; one that decodes
        double share, tile;            // a stage per tile; a tile
    } half[] = {{LIN_BIG, 256, 256, 256, 6.5, 1.3, 1.5, 0.0063, 0.02},
                {LIN_MIDDLE, 128, 128, 512, 4.5, 0.42, 1.0, 0.0020, 0.008},
                {LIN_SMALL, 128, 64, 768, 3.2, 0.35, 0.8, 0.00125, 0.004}},
      full[] = {{LIN_MIDDLE, 128, 128, 512, 4.5, 2.0, 2.2, 0.0077, 0.008},
                {LIN_MIDDLE, 128, 128, 512, 4.5, 2.0, 2.2, 0.0077, 0.008},
                {LIN_SMALL, 128, 64, 768, 3.2, 1.1, 1.3, 0.0039, 0.004}};
    LinTile best{LIN_SMALL, 1, 1e300};
    const int64_t stages = (nc + (f32 ? 31 : 63)) / (f32 ? 32 : 64);
    for (const auto& m : f32 ? full : half) {
        const int64_t tiles = ((np + m.tp - 1) / m.tp) * ((nq + m.tq - 1) / m.tq);
        for (int64_t split = 1; split <= 64 && split * 4 <= std::max<int64_t>(stages, 4); split += split < 4 ? 1 : split / 2) {
            const double n = (double)(tiles * split);
            if (split > 1 && n > 2 * m.fill) break;
            const double turns = std::ceil(n / m.fill);  // a last turn that is not full takes half a full one's time
            const double work = std::max(n, (turns - 1) * m.fill + std::min(n, 0.5 * m.fill));
            double t = m.launch + std::ceil((double)stages / split) * std::max(op == OP_DW ? m.decode : m.stage, m.share * work) +
                       m.tile * n;
            if (split > 1) t += 4.0 + (double)split * np * nq * 8 / 6.0e6;
            if (t < best.us) best = {m.shape, (int)split, t};
        }
    }
    return best;
}

template <class T, int OP, bool E5>
static void launch_shape(int shape, const LinArgs& a, hipStream_t s) {
    const auto go = [&](auto sh) {
        typedef decltype(sh) S;
        const int64_t tiles = ((a.np + S::TP - 1) / S::TP) * ((a.nq + S::TQ - 1) / S::TQ);
        hipLaunchKernelGGL((k_lin_tile<T, OP, E5, S>), dim3((unsigned)(tiles * a.split)), dim3(S::THREADS), 0, s, a);
    };
    if constexpr (sizeof(T) == 2)
        if (shape == LIN_BIG) return go(Big());
    if (shape == LIN_MIDDLE)
        go(Middle());
    else
        go(Small());
}

void launch_lin_tile(int op, int dtype, bool e5, int shape, const LinArgs& a, hipStream_t s) {
    const auto with = [&](auto t) {
        typedef decltype(t) T;
        if (op == OP_FWD)
            e5 ? launch_shape<T, OP_FWD, true>(shape, a, s) : launch_shape<T, OP_FWD, false>(shape, a, s);
        else if (op == OP_DX)
            e5 ? launch_shape<T, OP_DX, true>(shape, a, s) : launch_shape<T, OP_DX, false>(shape, a, s);
        else
            e5 ? launch_shape<T, OP_DW, true>(shape, a, s) : launch_shape<T, OP_DW, false>(shape, a, s);
    };
    if (dtype == APS_DTYPE_BF16)
        with((__bf16)0.0f);
    else if (dtype == APS_DTYPE_F16)
        with((_Float16)0.0f);
    else
        with(0.0f);
}

}  // namespace aps
