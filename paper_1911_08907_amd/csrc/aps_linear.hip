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

enum Kernel { GENERAL, TILE };
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

// What a call may run, by its sizes alone.
struct Plans {
    Plan aligned;  // where operands whose rows are whole chunks also start on them
    Plan any;
};

// An operand whose rows are no whole chunks is copied where the models say so:
// in us, a launch here and there, and its bytes in and out.
Plans plans_of(int op, const Dims& d, int dtype) {
    if (d.np == 0 || d.nq == 0) return {{GENERAL, 0, 1, false, false}, {GENERAL, 0, 1, false, false}};
    const bool f32 = dtype == APS_DTYPE_F32;
    const int cp = chunk_p(op, dtype), cq = chunk_q(dtype);
    const bool copy_p = d.nc > 0 && row_p(op, d) % cp != 0, copy_q = d.nc > 0 && row_q(op, d) % cq != 0;
    const LinTile g = lin_general(op, d.np, d.nq, d.nc, f32);
    const Plan any{GENERAL, 0, g.split, false, false};
    // a stage's offsets within a tile fit 31 bits, a copy's threads a launch
    const int64_t most = (int64_t)1 << 32;
    if (row_p(op, d) >= (1 << 21) || row_q(op, d) >= (1 << 21) || (copy_p && rows_p(op, d) * row_p(op, d) > most) ||
        (copy_q && rows_q(op, d) * row_q(op, d) > most))
        return {any, any};
    const LinTile t = lin_tile(op, d.np, d.nq, d.nc, f32);
    double us = t.us;
    if (copy_p || copy_q) us += 6.0;
    if (copy_p) us += (double)copy_bytes(rows_p(op, d), row_p(op, d), cp) / 1.5e6;
    if (copy_q) us += (double)copy_bytes(rows_q(op, d), row_q(op, d), cq) / 1.5e6;
    if ((copy_p || copy_q) && us >= g.us) return {any, any};
    return {{TILE, t.shape, t.split, copy_p, copy_q}, any};
}

// Partial sums, then the copies.
uint64_t part_bytes(int op, const Dims& d, int split) {
    return split > 1 ? ((uint64_t)(split * d.nq * (part_stride(d.np) + (op == OP_DW ? 1 : 0))) * 4 + 255) / 256 * 256 : 0;
}

uint64_t bytes_of(int op, const Dims& d, int dtype, const Plan& p) {
    return part_bytes(op, d, p.split) + (p.copy_p ? copy_bytes(rows_p(op, d), row_p(op, d), chunk_p(op, dtype)) : 0) +
           (p.copy_q ? copy_bytes(rows_q(op, d), row_q(op, d), chunk_q(dtype)) : 0);
}

uint64_t workspace_of(int op, const Dims& d, int dtype, const Plans& p) {
    return std::max(bytes_of(op, d, dtype, p.aligned), bytes_of(op, d, dtype, p.any));
}

// A pointer and stride on whole chunks, for an operand that is read in place.
bool on_chunks(const void* p, int64_t ld, int chunk) { return aligned16(p) && ld % chunk == 0 && ld < (1 << 21); }

int launch_product(int op, int dtype, bool e5, LinArgs& a, const Plans& plans, void* workspace, hipStream_t s) {
    const Dims d{a.np, a.nq, a.nc};
    const int cp = chunk_p(op, dtype), cq = chunk_q(dtype);
    const bool in_place_p = on_chunks(a.P, a.ldp, cp), in_place_q = on_chunks(a.Q, a.ldq, cq);
    if (op == OP_FWD && !a.codes && a.nq <= LIN_FEW) {
        a.split = 1;
        launch_lin_decode(dtype, in_place_p && in_place_q && a.nc % cq == 0, a, s);
        return launched();
    }
    const bool aligned = (in_place_p || row_p(op, d) % cp != 0) && (in_place_q || row_q(op, d) % cq != 0);
    const Plan& plan = aligned ? plans.aligned : plans.any;
    a.split = plan.split;
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

int check_workspace(int op, const Dims& d, int dtype, const Plans& p, const void* w, uint64_t bytes) {
    const uint64_t need = workspace_of(op, d, dtype, p);
    if (need == 0) return APS_OK;
    if (!w) return APS_ERR_NULL;
    if (bytes < need) return APS_ERR_SIZE;
    return aligned16(w) ? APS_OK : APS_ERR_ALIGN;
}

}  // namespace

}  // namespace aps

using namespace aps;

extern "C" uint64_t aps_linear_workspace_bytes(int32_t op, int32_t M, int32_t N, int32_t K, int32_t dtype) {
    if (op < OP_FWD || op > OP_DW || lin_check_dims(M, N, K, dtype) != APS_OK) return 0;
    const Dims d = dims_of(op, M, N, K);
    return workspace_of(op, d, dtype, plans_of(op, d, dtype));
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
    const Plans plans = plans_of(OP_FWD, d, dtype);
    APS_LIN_TRY(check_workspace(OP_FWD, d, dtype, plans, workspace, workspace_bytes));
    if (M == 0 || N == 0) return APS_OK;
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = X, a.ldq = ldx;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.bias = bias, a.R = R, a.ldr = ldr, a.out = Y, a.ldo = ldy;
    a.codes = codes, a.ldcodes = ldc, a.exps = ckpt_exp, a.act = act;
    a.vec = (rows_of_four(Y, ldy, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_CODES : 0) | (lin_aligned(bias, 4 * es) ? LV_BIAS : 0);
    return launch_product(OP_FWD, dtype, e5, a, plans, workspace, (hipStream_t)stream);
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
    const Plans plans = plans_of(OP_DX, d, dtype);
    APS_LIN_TRY(check_workspace(OP_DX, d, dtype, plans, workspace, workspace_bytes));
    if (M == 0 || K == 0) return APS_OK;
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.R = R, a.ldr = ldr, a.out = dX, a.ldo = lddx, a.act = act;
    if (act != APS_ACT_NONE) a.zc = codes, a.ldzc = ldc, a.zexps = ckpt_exp;
    a.vec = (rows_of_four(dX, lddx, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_ZC : 0);
    return launch_product(OP_DX, dtype, e5, a, plans, workspace, (hipStream_t)stream);
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
    const Plans plans = plans_of(OP_DW, d, dtype);
    APS_LIN_TRY(check_workspace(OP_DW, d, dtype, plans, workspace, workspace_bytes));
    if (N == 0 || K == 0) return APS_OK;
    LinArgs a{};
    a.P = codes, a.ldp = ldc, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.out = dW, a.ldo = lddw, a.zexps = ckpt_exp, a.dbias = db;
    a.accumulate = flags & APS_GRAD_ACCUMULATE;
    a.vec = rows_of_four(dW, lddw, 4) ? LV_OUT : 0;
    return launch_product(OP_DW, dtype, e5, a, plans, workspace, (hipStream_t)stream);
}
