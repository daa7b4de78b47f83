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
};

// `fast`: the operands' rows are aligned for the tile kernel; `plain`: no
// checkpoint is written.
Plan plan_of(int op, const Dims& d, int dtype, bool fast, bool plain) {
    if (d.np == 0 || d.nq == 0) return {GENERAL, 0, 1};
    if (op == OP_FWD && plain && d.nq <= LIN_FEW) return {DECODE, 0, 1};
    if (fast) {
        const LinTile t = lin_tile(op, d.np, d.nq, d.nc, dtype == APS_DTYPE_F32);
        return {TILE, t.shape, t.split};
    }
    return {GENERAL, 0, lin_split(op, d.np, d.nq, d.nc, dtype)};
}

uint64_t workspace_of(int op, const Dims& d, int dtype) {
    const int64_t s = std::max(plan_of(op, d, dtype, false, false).split, plan_of(op, d, dtype, true, false).split);
    return s > 1 ? (uint64_t)(s * d.nq * (part_stride(d.np) + (op == OP_DW ? 1 : 0))) * 4 : 0;
}

int launch_product(int op, int dtype, bool e5, LinArgs& a, void* workspace, hipStream_t s) {
    // rows of whole 16-byte chunks, and offsets within a tile that fit 31 bits
    const int e = 16 / lin_elem_bytes(dtype), pe = op == OP_DW ? 16 : e;
    const bool fast = aligned16(a.P) && aligned16(a.Q) && a.ldp % pe == 0 && a.ldq % e == 0 && a.ldp < (1 << 22) &&
                      a.ldq < (1 << 22) && (op == OP_FWD ? a.nc : a.np) % pe == 0 && (op == OP_DW ? a.nq : a.nc) % e == 0;
    const Plan plan = plan_of(op, {a.np, a.nq, a.nc}, dtype, fast, !a.codes);
    a.split = plan.split;
    a.piece = ((a.nc + a.split - 1) / a.split + 63) / 64 * 64;
    if (a.split > 1) {
        a.ldpart = part_stride(a.np);
        a.part = (float*)workspace;
        a.part_bias = a.part + a.split * a.nq * a.ldpart;
    }
    if (plan.kernel == DECODE)
        launch_lin_decode(dtype, fast, a, s);
    else if (plan.kernel == TILE)
        launch_lin_tile(op, dtype, e5, plan.shape, a, s);
    else
        launch_lin_general(op, dtype, e5, a, s);
    if (a.split > 1) launch_lin_join(op, dtype, e5, a, s);
    return launched();
}

int check_workspace(int op, const Dims& d, int dtype, const void* w, uint64_t bytes) {
    const uint64_t need = workspace_of(op, d, dtype);
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
    return workspace_of(op, dims_of(op, M, N, K), dtype);
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
    APS_LIN_TRY(check_workspace(OP_FWD, d, dtype, workspace, workspace_bytes));
    if (M == 0 || N == 0) return APS_OK;
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = X, a.ldq = ldx;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.bias = bias, a.R = R, a.ldr = ldr, a.out = Y, a.ldo = ldy;
    a.codes = codes, a.ldcodes = ldc, a.exps = ckpt_exp, a.act = act;
    a.vec = (rows_of_four(Y, ldy, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_CODES : 0) | (lin_aligned(bias, 4 * es) ? LV_BIAS : 0);
    return launch_product(OP_FWD, dtype, e5, a, workspace, (hipStream_t)stream);
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
    APS_LIN_TRY(check_workspace(OP_DX, d, dtype, workspace, workspace_bytes));
    if (M == 0 || K == 0) return APS_OK;
    LinArgs a{};
    a.P = W, a.ldp = ldw, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.R = R, a.ldr = ldr, a.out = dX, a.ldo = lddx, a.act = act;
    if (act != APS_ACT_NONE) a.zc = codes, a.ldzc = ldc, a.zexps = ckpt_exp;
    a.vec = (rows_of_four(dX, lddx, es) ? LV_OUT : 0) | (rows_of_four(R, ldr, es) ? LV_R : 0) |
            (rows_of_four(codes, ldc, 1) ? LV_ZC : 0);
    return launch_product(OP_DX, dtype, e5, a, workspace, (hipStream_t)stream);
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
    APS_LIN_TRY(check_workspace(OP_DW, d, dtype, workspace, workspace_bytes));
    if (N == 0 || K == 0) return APS_OK;
    LinArgs a{};
    a.P = codes, a.ldp = ldc, a.Q = dZ, a.ldq = lddz;
    a.np = d.np, a.nq = d.nq, a.nc = d.nc;
    a.out = dW, a.ldo = lddw, a.zexps = ckpt_exp, a.dbias = db;
    a.accumulate = flags & APS_GRAD_ACCUMULATE;
    a.vec = rows_of_four(dW, lddw, 4) ? LV_OUT : 0;
    return launch_product(OP_DW, dtype, e5, a, workspace, (hipStream_t)stream);
}
