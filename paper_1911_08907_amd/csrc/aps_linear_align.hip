// aps_linear_align.hip -- copies of a product's operands whose rows are no
// whole 16-byte chunks, or do not start on them, into rows that are and do,
// filled up with zeros: a read and a write of the operand, after which the tile kernel
// applies.  3.5 MB of fp32 rows of 1001 take 5 us; 700^3 bf16 went from 17.3 us to 14.2,
// the weight gradient of 1000 x 3000 x 520 from 90 to 20, 4096 x 4096 x 1024 off its
// chunks from 136 to 54.
#include "aps_linear.hpp"

namespace aps {

namespace {

// A thread writes one chunk of 16 bytes.
template <class W>
__device__ __forceinline__ void align_chunk(const LinCopy& c, int64_t k) {
    constexpr int E = 16 / (int)sizeof(W);
    typedef W vec __attribute__((ext_vector_type(E)));
    const int64_t per = c.ldd / E, r = k / per, col = k % per * E;
    const W* s = (const W*)c.src + r * c.lds + col;
    vec v = {};
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (col + i < c.cols) v[i] = s[i];
    *(vec*)((W*)c.dst + r * c.ldd + col) = v;
}

__global__ __launch_bounds__(256) void k_lin_align(LinCopy p, LinCopy q, int64_t np, int64_t nq) {
    int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool second = k >= np;
    const LinCopy& c = second ? q : p;
    if (second) k -= np;
    if (second && k >= nq) return;
    if (c.elem == 1) align_chunk<uint8_t>(c, k);
    else if (c.elem == 2) align_chunk<uint16_t>(c, k);
    else align_chunk<uint32_t>(c, k);
}

}  // namespace

// The launch and what it adds to a sequence of kernels, then the copies at 1.5 TB/s
// of what they write: in a trace 0.3 MB take 3.6 us, 2.2 MB 4.4, and of bf16 off
// its chunks 34 MB 25 us, 168 MB 114; fp32 copies up to 2.4 TB/s (336 MB 140 us).
double lin_align_us(uint64_t bytes) { return 6.0 + (double)bytes / 1.5e6; }

void launch_lin_align(const LinCopy& p, const LinCopy& q, hipStream_t s) {
    const auto chunks = [](const LinCopy& c) { return c.src ? c.rows * (c.ldd * c.elem / 16) : 0; };
    const int64_t np = chunks(p), nq = chunks(q);
    hipLaunchKernelGGL(k_lin_align, dim3((unsigned)((np + nq + 255) / 256)), dim3(256), 0, s, p, q, np, nq);
}

}  // namespace aps
