// aps_linear.hip -- the linear layer's C ABI: argument checks, the split of a
// contraction, the choice of the kernel.
#include "aps_linear.hpp"

namespace aps {

namespace {

// rows of `ld` elements of `bytes` from p, aligned for four elements at once
bool rows_of_four(const void* p, int64_t ld, int bytes) { return lin_aligned(p, 4 * bytes) && ld % 4 == 0; }

struct Dims {
    int64_t np, nq, nc;
};
Dims dims_of(int op, int64_t M, int64_t N, int64_t K) {
    if (op == OP_FWD) return {N, M, K};
    if (op == OP_DX) return {K, M, N};
    return {K, N, M};
}

int64_t part_stride(int64_t np) { return (np + 3) / 4 * 4; }

enum Kernel { GENERAL, TILE, DECODE };
struct Plan {
    Kernel kernel;
    int shape, split;
    bool copy_p, copy_q;  // operands that the tile kernel reads from aligned copies
};

// Elements of an operand's 16-byte chunk, and whether its rows are whole ones.
int chunk_p(int op, int dtype) { return op == OP_DW ? 16 : 16 / lin_elem_bytes(dtype); }
int chunk_q(int dtype) { return 16 / lin_elem_bytes(dtype); }
int64_t row_p(int op, const Dims& d) { return op == OP_FWD ? d.nc : d.np; }
int64_t row_q(int op, const Dims& d) { return op == OP_DW ? d.nq : d.nc; }
int64_t rows_p(int op, const Dims& d) { return op == OP_FWD ? d.np : d.nc; }
int64_t rows_q(int op, const Dims& d) { return op == OP_DW ? d.nc : d.nq; }

int64_t whole(int64_t n, int64_t chunk) { return (n + chunk - 1) / chunk * chunk; }
uint64_t copy_bytes(int64_t rows, int64_t row, int chunk) { return (uint64_t)(rows * whole(row, chunk)) * (16 / chunk) + 256; }

// Partial sums, then the copies.
uint64_t part_bytes(int op, const Dims& d, int split) {
    return split > 1 ? ((uint64_t)(split * d.nq * (part_stride(d.np) + (op == OP_DW ? 1 : 0))) * 4 + 255) / 256 * 256 : 0;
}

uint64_t bytes_of(int op, const Dims& d, int dtype, const Plan& p) {
    return part_bytes(op, d, p.split) + (p.copy_p ? copy_bytes(rows_p(op, d), row_p(op, d), chunk_p(op, dtype)) : 0) +
           (p.copy_q ? copy_bytes(rows_q(op, d), row_q(op, d), chunk_q(dtype)) : 0);
}

// The kernels' choices for a call's sizes, and from them what it runs.
class Planner {
  public:
    Planner(int op, const Dims& d, int dtype) : op_(op), d_(d), dtype_(dtype) {
        empty_ = d.np == 0 || d.nq == 0;
        if (empty_) return;
        const bool f32 = dtype == APS_DTYPE_F32;
        general_ = lin_general(op, d.np, d.nq, d.nc, f32);
        // a stage's offsets within a tile fit 31 bits
        tile_fits_ = row_p(op, d) < (1 << 21) && row_q(op, d) < (1 << 21);
        if (tile_fits_) tile_ = lin_tile(op, d.np, d.nq, d.nc, f32);
    }

    // The kernel that reads anything, from any workspace that a call is asked for.
    Plan any() const { return {GENERAL, 0, empty_ ? 1 : general_.split, false, false}; }

    // What the models say is fastest where the operands' rows do (on_p, on_q) or
    // do not start on 16-byte chunks; keeps: the call keeps a checkpoint of z.
    Plan plan(bool keeps, bool on_p, bool on_q) const {
        if (empty_) return any();
        const bool f32 = dtype_ == APS_DTYPE_F32, rows = d_.nc > 0;
        // operands that the tile kernel would have to read from copies
        const bool copy_p = rows && !(on_p && whole_p()), copy_q = rows && !(on_q && whole_q());
        // a copy's threads fit a launch
        const int64_t most = (int64_t)1 << 32;
        const bool tile = tile_fits_ && !(copy_p && rows_p(op_, d_) * row_p(op_, d_) > most) &&
                          !(copy_q && rows_q(op_, d_) * row_q(op_, d_) > most);
        const bool few = op_ == OP_FWD && !keeps && d_.nq <= LIN_FEW;
        // A call takes the host about 5 us and 5 for each launch: 50 x 734 x 76 fp16 in
        // one 9.9 us, copied first 14.9.
        const auto call = [](double us, int launches) { return std::max(us, 5.0 + 5.0 * launches); };
        double us = 1e300;
        Plan best = any();
        if (tile) {
            us = tile_.us;
            if (copy_p || copy_q)
                us += lin_align_us((copy_p ? copy_bytes(rows_p(op_, d_), row_p(op_, d_), chunk_p(op_, dtype_)) : 0) +
                                   (copy_q ? copy_bytes(rows_q(op_, d_), row_q(op_, d_), chunk_q(dtype_)) : 0));
            us = call(us, 1 + (tile_.split > 1) + (copy_p || copy_q));
            best = {TILE, tile_.shape, tile_.split, copy_p, copy_q};
        }
        if (copy_p || copy_q || !tile) {
            const double in_place = call(general_.us, 1 + (general_.split > 1));
            if (us >= in_place) us = in_place, best = any();
        }
        if (few) {
            // few rows leave the others no faster than the weights come from memory
            us = std::max(us, 3.0 + (double)d_.np * d_.nc * lin_elem_bytes(dtype_) / 3.6e6);
            if (call(lin_decode_us(d_.np, d_.nq, d_.nc, f32, !(copy_p || copy_q)), 1) <= us) best = {DECODE, 0, 1, false, false};
        }
        return best;
    }

    // Bytes that suffice for every call, with no copy of an operand that is merely off its chunks.
    uint64_t need() const {
        return std::max(bytes_of(op_, d_, dtype_, plan(true, true, true)), bytes_of(op_, d_, dtype_, any()));
    }

  private:
    bool whole_p() const { return row_p(op_, d_) % chunk_p(op_, dtype_) == 0; }
    bool whole_q() const { return row_q(op_, d_) % chunk_q(dtype_) == 0; }
    int op_;
    Dims d_;
    int dtype_;
    bool empty_, tile_fits_ = false;
    LinTile general_{}, tile_{};
};

// A pointer and stride on whole chunks, for an operand that is read in place.
bool on_chunks(const void* p, int64_t ld, int chunk) { return aligned16(p) && ld % chunk == 0 && ld < (1 << 21); }
bool on_chunks_p(int op, int dtype, const LinArgs& a) { return on_chunks(a.P, a.ldp, chunk_p(op, dtype)); }
bool on_chunks_q(int dtype, const LinArgs& a) { return on_chunks(a.Q, a.ldq, chunk_q(dtype)); }

int launch_product(int op, int dtype, bool e5, LinArgs& a, const Plan& plan, void* workspace, hipStream_t s) {
    const Dims d{a.np, a.nq, a.nc};
    const int cp = chunk_p(op, dtype), cq = chunk_q(dtype);
    a.split = plan.split;
    if (plan.kernel == DECODE) {
        launch_lin_decode(dtype, on_chunks_p(op, dtype, a) && on_chunks_q(dtype, a) && a.nc % cq == 0, a, s);
        return launched();
    }
    a.piece = ((a.nc + a.split - 1) / a.split + 63) / 64 * 64;
    if (a.split > 1) {
        a.ldpart = part_stride(a.np);
        a.part = (float*)workspace;
        a.part_bias = a.part + a.split * a.nq * a.ldpart;
    }
    if (plan.copy_p || plan.copy_q) {
        char* to = (char*)workspace + part_bytes(op, d, a.split);
        LinCopy p{}, q{};
        if (plan.copy_p) {
            p = {a.P, to, a.ldp, whole(row_p(op, d), cp), rows_p(op, d), row_p(op, d), 16 / cp};
            to += (copy_bytes(p.rows, p.cols, cp) + 15) / 16 * 16;
            a.P = p.dst, a.ldp = p.ldd;
        }
        if (plan.copy_q) {
            q = {a.Q, to, a.ldq, whole(row_q(op, d), cq), rows_q(op, d), row_q(op, d), 16 / cq};
            a.Q = q.dst, a.ldq = q.ldd;
        }
        launch_lin_align(p, q, s);
    }
    if (plan.kernel == TILE)
        launch_lin_tile(op, dtype, e5, plan.shape, a, s);
    else
        launch_lin_general(op, dtype, e5, a, s);
    if (a.split > 1) launch_lin_join(op, dtype, e5, a, s);
    return launched();
}

// The plan of a call that has `bytes` of workspace at w.
int choose(int op, int dtype, const LinArgs& a, const void* w, uint64_t bytes, Plan& plan) {
    const Dims d{a.np, a.nq, a.nc};
    const Planner planner(op, d, dtype);
    plan = planner.plan(a.codes != nullptr, on_chunks_p(op, dtype, a), on_chunks_q(dtype, a));
    const uint64_t wants = bytes_of(op, d, dtype, plan);
    if (!w && bytes == 0 && wants == 0) return APS_OK;
    const uint64_t need = planner.need();
    if (need > 0) {
        if (!w) return APS_ERR_NULL;
        if (bytes < need) return APS_ERR_SIZE;
        if (!aligned16(w)) return APS_ERR_ALIGN;
    }
    // operands off their chunks may be worth a copy that need() does not count
    if (wants > (w ? bytes : 0))
        plan = planner.any();
    else if (wants > 0 && !aligned16(w))
        return APS_ERR_ALIGN;
    return APS_OK;
}

}  // namespace

}  // namespace aps

using namespace aps;

extern "C" uint64_t aps_linear_workspace_bytes(int32_t op, int32_t M, int32_t N, int32_t K, int32_t dtype) {
    const bool on = op & APS_LINEAR_ON_CHUNKS, off = op & APS_LINEAR_OFF_CHUNKS, keeps = !(op & APS_LINEAR_NO_CKPT);
    op &= ~(APS_LINEAR_ON_CHUNKS | APS_LINEAR_OFF_CHUNKS | APS_LINEAR_NO_CKPT);
    if (op < OP_FWD || op > OP_DW || lin_check_dims(M, N, K, dtype) != APS_OK) return 0;
    const Dims d = dims_of(op, M, N, K);
    const Planner planner(op, d, dtype);
    if (on && bytes_of(op, d, dtype, planner.plan(keeps, true, true)) == 0) return 0;
    uint64_t bytes = planner.need();
    for (int ons = 0; off && ons < 3; ++ons)  // P, Q or both off their chunks
        bytes = std::max(bytes, bytes_of(op, d, dtype, planner.plan(keeps, ons & 1, ons & 2)));
    return bytes;
}

extern "C" int aps_linear(const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias, const void* R,
                          int64_t ldr, void* Y, int64_t ldy, int32_t M, int32_t N, int32_t K, int32_t dtype,
                          int32_t act, aps_format ckpt_fmt, uint8_t* codes, int64_t ldc, int32_t* ckpt_exp,
                          void* workspace, uint64_t workspace_bytes, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, N, K, dtype));
    if (!lin_act_known(act)) return APS_ERR_UNSUPPORTED;
    const int es = lin_elem_bytes(dtype);
    APS_LIN_TRY(lin_check_matrix(X, ldx, N ? M : 0, K, es));
    APS_LIN_TRY(lin_check_matrix(W, ldw, M ? N : 0, K, es));
    APS_LIN_TRY(lin_check_matrix(Y, ldy, M, N, es));
    if (R) APS_LIN_TRY(lin_check_matrix(R, ldr, M, N, es));
    if (bias && !lin_aligned(bias, es)) return APS_ERR_ALIGN;
    bool e5 = false;
    if (codes || ckpt_exp) APS_LIN_TRY(lin_check_checkpoint(ckpt_fmt, codes, ldc, ckpt_exp, M, N, e5));
    const Dims d = dims_of(OP_FWD, M, N, K);
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = X, a.ldq = ldx;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.bias = bias, a.R = R, a.ldr = ldr, a.out = Y, a.ldo = ldy;
    a.codes = codes, a.ldcodes = ldc, a.exps = ckpt_exp, a.act = act;
    a.vec = (rows_of_four(Y, ldy, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_CODES : 0) | (lin_aligned(bias, 4 * es) ? LV_BIAS : 0);
    Plan plan;
    APS_LIN_TRY(choose(OP_FWD, dtype, a, workspace, workspace_bytes, plan));
    if (M == 0 || N == 0) return APS_OK;
    return launch_product(OP_FWD, dtype, e5, a, plan, workspace, (hipStream_t)stream);
}

extern "C" int aps_linear_grad_input(const void* dZ, int64_t lddz, const void* W, int64_t ldw, const void* R,
                                     int64_t ldr, int32_t act, aps_format fmt, const uint8_t* codes, int64_t ldc,
                                     const int32_t* ckpt_exp, void* dX, int64_t lddx, int32_t M, int32_t N, int32_t K,
                                     int32_t dtype, void* workspace, uint64_t workspace_bytes, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, N, K, dtype));
    if (!lin_act_known(act)) return APS_ERR_UNSUPPORTED;
    const int es = lin_elem_bytes(dtype);
    APS_LIN_TRY(lin_check_matrix(dZ, lddz, K ? M : 0, N, es));
    APS_LIN_TRY(lin_check_matrix(W, ldw, M ? N : 0, K, es));
    APS_LIN_TRY(lin_check_matrix(dX, lddx, M, K, es));
    if (R) APS_LIN_TRY(lin_check_matrix(R, ldr, M, K, es));
    bool e5 = false;
    if (act != APS_ACT_NONE) APS_LIN_TRY(lin_check_checkpoint(fmt, codes, ldc, ckpt_exp, M, K, e5));
    const Dims d = dims_of(OP_DX, M, N, K);
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.R = R, a.ldr = ldr, a.out = dX, a.ldo = lddx, a.act = act;
    if (act != APS_ACT_NONE) a.zc = codes, a.ldzc = ldc, a.zexps = ckpt_exp;
    a.vec = (rows_of_four(dX, lddx, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_ZC : 0);
    Plan plan;
    APS_LIN_TRY(choose(OP_DX, dtype, a, workspace, workspace_bytes, plan));
    if (M == 0 || K == 0) return APS_OK;
    return launch_product(OP_DX, dtype, e5, a, plan, workspace, (hipStream_t)stream);
}

extern "C" int aps_linear_grad_weight(const void* dZ, int64_t lddz, aps_format fmt, const uint8_t* codes, int64_t ldc,
                                      const int32_t* ckpt_exp, float* dW, int64_t lddw, float* db, int32_t M,
                                      int32_t N, int32_t K, int32_t dtype, uint32_t flags, void* workspace,
                                      uint64_t workspace_bytes, void* stream) {
    APS_LIN_TRY(lin_check_dims(M, N, K, dtype));
    if (flags & ~APS_GRAD_ACCUMULATE) return APS_ERR_UNSUPPORTED;
    const int es = lin_elem_bytes(dtype);
    APS_LIN_TRY(lin_check_matrix(dZ, lddz, K ? M : 0, N, es));
    bool e5 = false;
    APS_LIN_TRY(lin_check_checkpoint(fmt, codes, ldc, ckpt_exp, N ? M : 0, K, e5));
    APS_LIN_TRY(lin_check_matrix(dW, lddw, N, K, 4));
    if (db && K == 0) return APS_ERR_SIZE;  // db is summed beside dW
    if (db && !lin_aligned(db, 4)) return APS_ERR_ALIGN;
    const Dims d = dims_of(OP_DW, M, N, K);
    LinArgs a{};
    a.P = codes, a.ldp = ldc, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.out = dW, a.ldo = lddw, a.zexps = ckpt_exp, a.dbias = db;
    a.accumulate = flags & APS_GRAD_ACCUMULATE;
    a.vec = rows_of_four(dW, lddw, 4) ? LV_OUT : 0;
    Plan plan;
    APS_LIN_TRY(choose(OP_DW, dtype, a, workspace, workspace_bytes, plan));
    if (N == 0 || K == 0) return APS_OK;
    return launch_product(OP_DW, dtype, e5, a, plan, workspace, (hipStream_t)stream);
}
