// aps_linear_decode.hip -- the linear layer's forward product for a few rows
// (single tokens, small batches): bound by the weights' bytes and by latency.
//
// A workgroup of sixteen waves finishes 16 p for all q: its waves take the
// contraction's pieces of 64 bytes in turn, so that together they read a
// kilobyte of each weight row at a time, and every wave has four pieces in
// flight.  A lane's 16 bytes are its fragment of a 16 x 16 matrix instruction as
// they come from memory (rows by lane % 16, pieces of the 64 bytes by lane / 16),
// for the weights and the activations alike: nothing passes through LDS but
// the waves' sums, joined in their order.  One row of 4096 x 1024 bf16 takes 4.2 us
// (2 TB/s; half of it is the launch and the two dependent reads), where tiles of
// 128 x 64 take 8.6 and the general kernel with its join 11.
#include "aps_linear.hpp"

namespace aps {

namespace {

constexpr int DWAVES = 16, DP = 16;  // waves and p of a workgroup
constexpr int DEPTH = 4;             // pieces in flight

template <class T>
struct Few {  // 16-bit: one instruction of 32 c
    typedef T frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mma(frag p, frag q, f32x4 c) {
        if constexpr (std::is_same_v<T, __bf16>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, c, 0, 0, 0);
    }
};
template <>
struct Few<float> {  // four of 4 c
    typedef f32x4 frag;
    static __device__ __forceinline__ f32x4 mma(frag p, frag q, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], q[i], c, 0, 0, 0);
        return c;
    }
};

// QF: 16 q each.  VEC: rows are aligned to 16 bytes, the contraction a multiple of it.
template <class T, int QF, bool VEC>
__global__ __launch_bounds__(64 * DWAVES) void k_lin_decode(LinArgs a) {
    typedef typename Few<T>::frag F;
    constexpr int E = 16 / (int)sizeof(T), PIECE = 4 * E;
    __shared__ f32x4 sums[DWAVES][QF][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t p0 = (int64_t)blockIdx.x * DP;
    // rows past the end read the last one: their results are not stored
    const T* p = (const T*)a.P + min(p0 + (lane & 15), a.np - 1) * a.ldp;
    const T* q[QF];
#pragma unroll
    for (int j = 0; j < QF; ++j) q[j] = (const T*)a.Q + min((int64_t)(j * 16 + (lane & 15)), a.nq - 1) * a.ldq;
    const int nc = (int)a.nc, c0 = (wave * 4 + (lane >> 4)) * E;
    const auto read = [&](const T* row, int c) {
        F v = {};
        if constexpr (VEC) {
            if (c < nc) v = *(const F*)(row + c);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (c + i < nc) v[i] = row[c + i];
        }
        return v;
    };
    f32x4 acc[QF] = {};
    for (int c = c0; c - (lane >> 4) * E < nc; c += DEPTH * DWAVES * PIECE) {
        F fp[DEPTH], fq[DEPTH][QF];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fp[d] = read(p, c + d * DWAVES * PIECE);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
#pragma unroll
            for (int j = 0; j < QF; ++j) fq[d][j] = read(q[j], c + d * DWAVES * PIECE);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
#pragma unroll
            for (int j = 0; j < QF; ++j) acc[j] = Few<T>::mma(fp[d], fq[d][j], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < QF; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave >= QF) return;
    // lane: q = lane % 16, p = 4 (lane / 16) + i
    f32x4 s = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < DWAVES; ++w) s += sums[w][wave][lane];
    const int64_t qo = wave * 16 + (lane & 15), po = p0 + (lane >> 4) * 4, have = a.np - po;
    if (qo >= a.nq || have <= 0) return;
    float b[4];
    lin_bias4<T>(a, po, have, b);
    const float v[4] = {s[0] + b[0], s[1] + b[1], s[2] + b[2], s[3] + b[3]};
    with_act(a.act, [&](auto act) {
        LinRead<T, OP_FWD, 4> in;
        in.read(a, qo, po, have);
        lin_finish<T, OP_FWD, false, 4, act.value>(a, in, qo, po, have, v);
    });
}

}  // namespace

// A launch; then the larger of a workgroup's 4 KB of each weight row after
// another, whose latency grows with the rows of q, the workgroups' shares of the
// memory's rate, and a workgroup's start.  Element by element (off chunks) all of
// it costs more.  Fitted to graph replays of 220 products beside the other
// kernels.  In us, this kernel and the best of the others:
//                            1 row         8             32
//   4096 x 1024 bf16         4.8, 8.3      4.8, 8.2      6.1, 8.9
//   ... off chunks           12.3, 9.7     16.0, 9.9     25.1, 11.3
//   16384 x 4096 bf16, HBM   28.4, 30.6    32.8, 40.1    54.8, 41.4
//   16384 x 4096 fp32, HBM   62.4, 93.8    67.6, 93.4    113.6, 95.3
//   1024 x 4096 bf16         7.3, 8.3      8.7, 9.1      14.0, 10.4
//   16 x 16384 bf16          19.9, 10.7    25.2, 11.7    44.0, 15.0
double lin_decode_us(int64_t np, int64_t nq, int64_t nc, bool f32, bool fast) {
    static const struct {
        double launch, round, per_q, share, share_q;
    } on[] = {{3.3, 2.05, 0.095, 0.0122, 0.0004}, {3.3, 2.4, 0.1, 0.0142, 0.0004}},
      off[] = {{7.0, 11.0, 0.55, 0.067, 0.0024}, {7.0, 6.0, 0.33, 0.04, 0.0013}};
    const auto& m = (fast ? on : off)[f32];
    const double rounds = (double)nc * (f32 ? 4 : 2) / 4096, groups = (double)((np + DP - 1) / DP);
    const double work = rounds * std::max(m.round + m.per_q * nq, groups * (m.share + m.share_q * nq));
    return m.launch + std::max(work, 0.012 * (groups - 128));
}

void launch_lin_decode(int dtype, bool fast, const LinArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.np + DP - 1) / DP)), block(64 * DWAVES);
    const auto go = [&](auto t) {
        typedef decltype(t) T;
        if (a.nq <= 16) {
            if (fast) hipLaunchKernelGGL((k_lin_decode<T, 1, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((k_lin_decode<T, 1, false>), grid, block, 0, s, a);
        } else {
            if (fast) hipLaunchKernelGGL((k_lin_decode<T, 2, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((k_lin_decode<T, 2, false>), grid, block, 0, s, a);
        }
    };
    if (dtype == APS_DTYPE_BF16) go((__bf16)0.0f);
    else if (dtype == APS_DTYPE_F16) go((_Float16)0.0f);
    else go(0.0f);
}

}  // namespace aps
