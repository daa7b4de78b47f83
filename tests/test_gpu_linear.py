"""The linear layer's operators against float64: checkpoints to the last bit,
products and gradients within bounds counted from their roundings."""
import math

import pytest
import torch

from paper_1911_08907_amd import aps as A
from tests import linear_ref as R
from tests._util import log

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
FMT = {"1-5-2": A.Format(5, 2), "1-4-3": A.Format(4, 3)}
ACT = {"none": A.APS_ACT_NONE, "relu": A.APS_ACT_RELU, "gelu": A.APS_ACT_GELU, "silu": A.APS_ACT_SILU}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    A.lib()
    return torch.device("cuda:0")


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _place(x, dev, layout, fill=math.nan):
    """x on the GPU as a matrix of the given layout, surrounded by `fill`:
    "dense" rows, "padded" rows (16-byte aligned, wider than the matrix), or
    "odd" (rows that start anywhere)."""
    M, C = x.shape
    if layout == "dense":
        return x.to(dev).contiguous()
    per16 = 16 // x.element_size()
    if layout == "padded":
        ld, off = -(-(C + 1) // per16) * per16 + per16, per16
    else:
        ld, off = C + 3, 1
    buf = torch.full((M * ld + off + ld,), fill, dtype=x.dtype) if x.dtype.is_floating_point else torch.full(
        (M * ld + off + ld,), 0xA5, dtype=x.dtype)
    buf = buf.to(dev)
    v = buf[off:off + M * ld].view(M, ld)[:, :C]
    v.copy_(x.to(dev))
    return v


def _blank(M, C, dtype, dev, layout):
    """An output of the given layout and a check that nothing around it changed."""
    per16 = 16 // torch.empty(0, dtype=dtype).element_size()
    ld, off = {"dense": (C, 0), "padded": (-(-(C + 1) // per16) * per16 + per16, per16), "odd": (C + 3, 1)}[layout]
    mark = 77
    buf = torch.full((M * ld + off + ld,), mark, dtype=dtype, device=dev)
    v = buf[off:off + M * ld].view(M, ld)[:, :C]

    def clean():
        b = buf.clone()
        b[off:off + M * ld].view(M, ld)[:, :C] = mark
        return bool((b == mark).all())
    return v, clean


def _mixed(g, M, C, T):
    """Values over many binades, zeros, and the type's extremes."""
    x = torch.randn(M, C, generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-12, 6, (M, C), generator=g).double())
    x[torch.rand(M, C, generator=g) < 0.1] = 0.0
    return x.to(T)


def _same(a, b):
    """Equal values, NaN equal to NaN."""
    return bool(((a == b) | ((a != a) & (b != b))).all())


# ------------------------------------------------------------- checkpoints

CK_SHAPES = [(1, 1), (1, 128), (32, 128), (33, 129), (31, 250), (70, 1001), (96, 512), (5, 3)]


@pytest.mark.parametrize("layout", ["dense", "padded", "odd"])
@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("t", list(TYPES))
def test_save_and_load(dev, t, fmt, layout):
    T = TYPES[t]
    for M, C in CK_SHAPES:
        log("save", t, fmt, layout, M, C)
        x = _mixed(_gen(M * 1000 + C), M, C, T)
        X = _place(x, dev, layout)
        codes, clean = _blank(M, C, torch.uint8, dev, layout)
        words = torch.full((-(-M // 32) + 1, -(-C // 128)), -5, dtype=torch.int32, device=dev)
        A.aps_checkpoint_save(X, FMT[fmt], codes, words[:-1])
        rc, rw = R.save(x.double(), fmt, T)
        assert torch.equal(codes.cpu(), rc)
        assert torch.equal(words[:-1].cpu(), rw) and bool((words[-1] == -5).all())
        assert clean()
        out, clean = _blank(M, C, T, dev, layout)
        A.aps_checkpoint_load(codes, words[:-1].contiguous(), FMT[fmt], X=out)
        assert _same(out.cpu().double(), R.load(rc, rw, fmt)) and clean()


@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("t", list(TYPES))
def test_save_special_values(dev, t, fmt):
    """A block of zeros; one of the smallest values; the largest finite value;
    INF and NaN, which cost only their own elements; a max on and next to a
    power of two; ties."""
    T, fi = TYPES[t], torch.finfo(TYPES[t])
    x = torch.zeros(32, 128 * 8, dtype=T)
    b = [x[:, 128 * i:128 * (i + 1)] for i in range(8)]
    b[1][:] = fi.smallest_normal * fi.eps  # the smallest subnormal
    b[1][3, 5] = -fi.smallest_normal
    b[2][7, 7], b[2][8, 8], b[2][9, 9] = fi.max, -fi.max / 2, 1.0
    b[3][:] = 0.75
    b[3][0, 0], b[3][1, 1], b[3][2, 2], b[3][31, 127] = math.inf, -math.inf, math.nan, -0.0
    b[4][:] = math.nan
    b[5][:] = 1.0 + fi.eps
    b[5][:, :64] = -1.0
    b[6][:] = torch.arange(128, dtype=torch.float64).to(T) / 16 - 4
    b[7][:] = -math.inf
    codes, words = A.aps_checkpoint_save(x.to(dev), FMT[fmt])
    rc, rw = R.save(x.double(), fmt, T)
    nan = torch.isnan(x)
    got = codes.cpu()
    assert torch.equal(got[~nan], rc[~nan]) and torch.equal(got[nan] & 127, rc[nan] & 127)
    assert torch.equal(words.cpu(), rw)
    out = A.aps_checkpoint_load(codes, words, FMT[fmt], dtype=T).cpu()
    assert _same(out.double(), R.load(rc, rw, fmt))
    assert bool(torch.isfinite(out[torch.isfinite(x)]).all())  # a finite value never becomes INF


@pytest.mark.parametrize("act", list(ACT))
@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("t", list(TYPES))
def test_load_and_gradient_of_every_code(dev, t, fmt, act):
    T = TYPES[t]
    M, C = 64, 256
    codes = torch.arange(256, dtype=torch.uint8).repeat(M, 1)
    words = torch.tensor([[3, (-4 & 0xFFFF)], [0, 12]], dtype=torch.int32) | (1 << 16)
    z = R.load(codes, words, fmt)
    Z = A.aps_checkpoint_load(codes.to(dev), words.to(dev), FMT[fmt], ACT[act], dtype=T).cpu()
    ref = R.act(z, act)
    big = ref.abs() >= torch.finfo(T).max  # half: beyond its range
    err = (Z.double() - ref).abs()
    tol = R.half_step(T) * ref.abs() + R.ACT_ULPS * z.abs() + R.tiny(T)
    fine = torch.isfinite(ref) & ~big
    assert bool((err[fine] <= tol[fine]).all())
    assert _same(Z[~fine & ~big].double(), ref[~fine & ~big])
    dY = torch.randn(M, C, generator=_gen(5)).to(T)
    dZ = A.aps_activation_grad(dY.to(dev), codes.to(dev), words.to(dev), FMT[fmt], ACT[act]).cpu()
    s = R.slope(z, act)
    ref = dY.double() * s
    fine = torch.isfinite(ref)
    # the slope's own error: of sums of terms up to |z| phi(z) <= 0.25 and 1
    tol = R.half_step(T) * ref.abs() + dY.double().abs() * 1.5 * R.ACT_ULPS * (1 if act in ("gelu", "silu") else 0) + R.tiny(T)
    assert bool(((dZ.double() - ref).abs()[fine] <= tol[fine]).all())
    assert bool(torch.isnan(dZ[~fine]).all())


@pytest.mark.parametrize("layout", ["dense", "padded", "odd"])
@pytest.mark.parametrize("t", list(TYPES))
def test_activation_grad_layouts(dev, t, layout):
    T = TYPES[t]
    for M, C in CK_SHAPES:
        log("act_grad", t, layout, M, C)
        g = _gen(C)
        rc, rw = R.save(torch.randn(M, C, generator=g).to(T).double(), "1-4-3", T)
        dY = torch.randn(M, C, generator=g).to(T)
        D = _place(dY, dev, layout)
        codes = _place(rc, dev, layout)
        out, clean = _blank(M, C, T, dev, layout)
        A.aps_activation_grad(D, codes, rw.to(dev), FMT["1-4-3"], ACT["gelu"], out)
        ref = dY.double() * R.slope(R.load(rc, rw, "1-4-3"), "gelu")
        tol = R.half_step(T) * ref.abs() + dY.double().abs() * 1.5 * R.ACT_ULPS + R.tiny(T)
        assert bool(((out.cpu().double() - ref).abs() <= tol).all()) and clean()
        A.aps_activation_grad(D, codes, rw.to(dev), FMT["1-4-3"], ACT["gelu"], D)  # in place
        assert torch.equal(D, out)


# ---------------------------------------------------------------- products

# (M, N, K): single elements, single rows, partial tiles on every side, whole
# tiles of every size, long contractions that are split, odd lengths
SHAPES = [(1, 1, 1), (1, 64, 48), (2, 130, 257), (7, 777, 101), (16, 256, 512), (17, 264, 1032), (33, 128, 64),
          (64, 512, 2048), (100, 96, 31), (128, 128, 128), (129, 136, 72), (256, 256, 64), (250, 1000, 512),
          (260, 520, 136), (300, 77, 4099), (512, 768, 320)]


def _problem(t, M, N, K, seed):
    T, g = TYPES[t], _gen(seed)
    X = (torch.randn(M, K, generator=g) * torch.where(torch.rand(K, generator=g) < 0.02, 20.0, 1.0)).to(T)
    W = (torch.randn(N, K, generator=g) / math.sqrt(K)).to(T)
    b = torch.randn(N, generator=g).to(T)
    r = torch.randn(M, N, generator=g).to(T)
    return X, W, b, r


def _check_zhat(codes, words, fmt, T, z, ez):
    """The checkpoint of a z known within ez: each block's exponent is that of
    a maximum within ez of z's, each value within half a step."""
    e, m, bias = R.FORMATS[fmt]
    emax, emin = (1 << e) - 2 - bias, 1 - bias
    lim = R.limit(fmt, T)
    lo, _ = R.block_exponents(torch.sign(z) * (z.abs() + ez).clamp(max=lim), fmt, T)
    hi, _ = R.block_exponents(torch.sign(z) * (z.abs() - ez).clamp(min=0), fmt, T)
    ft = ((words.cpu().long() & 0xFFFF) ^ 0x8000) - 0x8000
    lo, hi = torch.tensor(lo), torch.tensor(hi)
    assert bool(((ft >= lo) & (ft <= torch.where(hi == 0, ft, hi))).all())
    assert not bool((words.cpu() >> 16).any())
    zc = z.clamp(-lim, lim)
    f = torch.exp2(-R.spread(ft.double(), *z.shape))
    half = torch.maximum((z.abs() + ez) * 2.0 ** -(m + 1), f * 2.0 ** (emin - m - 1))
    assert bool(((R.load(codes.cpu(), words.cpu(), fmt) - zc).abs() <= half + ez).all())


@pytest.mark.parametrize("layout", ["dense", "padded", "odd"])
@pytest.mark.parametrize("t", list(TYPES))
def test_linear(dev, t, layout):
    T = TYPES[t]
    acts, fmts = list(ACT), list(FMT)
    for i, (M, N, K) in enumerate(SHAPES):
        act, fmt = acts[i % 4], fmts[i % 2]
        log("linear", t, layout, M, N, K, act, fmt)
        X, W, b, r = _problem(t, M, N, K, i)
        z = X.double() @ W.double().t() + b.double()
        ez = R.sums_bound(W.double().abs().t(), X.double().abs(), b.double().abs())
        ref = R.act(z, act) + r.double()
        ey = R.LIPSCHITZ * ez + R.ACT_ULPS * z.abs() + 2.0 ** -24 * ref.abs()
        tol = ey + R.half_step(T) * (ref.abs() + ey) + R.tiny(T)
        Y, clean_y = _blank(M, N, T, dev, layout)
        codes, clean_c = _blank(M, N, torch.uint8, dev, layout)
        args = [_place(v, dev, layout) for v in (X, W)]
        R_ = _place(r, dev, layout)
        bias = torch.cat([torch.zeros(1, dtype=T), b]).to(dev)[1:] if layout == "odd" else b.to(dev)
        _, codes, words = A.aps_linear(*args, bias, R_, ACT[act], Y, FMT[fmt], codes)
        assert bool(((Y.cpu().double() - ref).abs() <= tol).all()), float(((Y.cpu().double() - ref).abs() / tol).max())
        assert clean_y() and clean_c()
        _check_zhat(codes, words, fmt, T, z, ez)
        # without bias, residual and checkpoint, in place of the residual
        A.aps_linear(*args, None, R_, ACT["none"], R_)
        ref = X.double() @ W.double().t() + r.double()
        tol = ez + R.half_step(T) * (ref.abs() + ez) + 2.0 ** -24 * ref.abs() + R.tiny(T)
        assert bool(((R_.cpu().double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("layout", ["dense", "padded", "odd"])
@pytest.mark.parametrize("t", list(TYPES))
def test_linear_grad_input(dev, t, layout):
    T = TYPES[t]
    acts, fmts = list(ACT), list(FMT)
    for i, (M, N, K) in enumerate(SHAPES):
        act, fmt = acts[i % 4], fmts[i % 2]
        log("grad_input", t, layout, M, N, K, act, fmt)
        g = _gen(100 + i)
        dZ = torch.randn(M, N, generator=g).to(T)
        W = (torch.randn(N, K, generator=g) / math.sqrt(N)).to(T)
        r = torch.randn(M, K, generator=g).to(T)
        rc, rw = R.save(torch.randn(M, K, generator=g).to(T).double(), fmt, T)
        s = R.slope(R.load(rc, rw, fmt), act)
        d = dZ.double() @ W.double()
        ed = R.sums_bound(W.double().abs(), dZ.double().abs())
        ref = d * s + r.double()
        e = R.LIPSCHITZ * ed + d.abs() * 2 * R.ACT_ULPS + 2.0 ** -23 * ref.abs()
        tol = e + R.half_step(T) * (ref.abs() + e) + R.tiny(T)
        out, clean = _blank(M, K, T, dev, layout)
        args = [_place(v, dev, layout) for v in (dZ, W, r)]
        ck = () if act == "none" else (_place(rc, dev, layout), rw.to(dev), FMT[fmt])
        A.aps_linear_grad_input(*args, ACT[act], *ck, dX=out)
        err = (out.cpu().double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        assert clean()


@pytest.mark.parametrize("layout", ["dense", "padded", "odd"])
@pytest.mark.parametrize("t", list(TYPES))
def test_linear_grad_weight(dev, t, layout):
    T = TYPES[t]
    fmts = list(FMT)
    for i, (M, N, K) in enumerate(SHAPES + [(4100, 130, 72), (2048, 256, 256)]):
        fmt = fmts[i % 2]
        log("grad_weight", t, layout, M, N, K, fmt)
        g = _gen(200 + i)
        dZ = (torch.randn(M, N, generator=g) * 0.01).to(T)
        rc, rw = R.save((torch.randn(M, K, generator=g) * torch.exp2(torch.randn(M, 1, generator=g) * 3)).to(T).double(),
                        fmt, T)
        x = R.load(rc, rw, fmt)
        ref = dZ.double().t() @ x
        e = R.sums_bound(x.abs(), dZ.double().abs().t()) + 2.0 ** -24 * ref.abs()
        dW, clean = _blank(N, K, torch.float32, dev, layout)
        D, C = _place(dZ, dev, layout), _place(rc, dev, layout)
        db = torch.full((N + 1,), 7.0, device=dev)
        A.aps_linear_grad_weight(D, C, rw.to(dev), FMT[fmt], dW, db[:N])
        err = (dW.cpu().double() - ref).abs()
        assert bool((err <= e + R.tiny(torch.float32)).all()), float((err / e).max())
        refb = dZ.double().sum(0)
        eb = (M + 2) * 2.0 ** -23 * dZ.double().abs().sum(0)
        assert bool(((db[:N].cpu().double() - refb).abs() <= eb).all())
        assert clean() and float(db[N]) == 7.0
        first, firstb = dW.clone(), db.clone()
        A.aps_linear_grad_weight(D, C, rw.to(dev), FMT[fmt], dW, db[:N], accumulate=True)
        assert torch.equal(dW, first + first) and torch.equal(db[:N], firstb[:N] + firstb[:N]) and clean()
        dW2 = A.aps_linear_grad_weight(D, C, rw.to(dev), FMT[fmt])  # without db: the same dW
        assert torch.equal(dW2, first)


@pytest.mark.parametrize("t", list(TYPES))
def test_empty_dimensions(dev, t):
    T = TYPES[t]
    z = lambda *s: torch.zeros(*s, dtype=T, device=dev)  # noqa: E731
    b = torch.arange(9, dtype=T, device=dev)
    assert A.aps_linear(z(0, 5), z(9, 5), b).shape == (0, 9)
    assert A.aps_linear(z(4, 5), z(0, 5)).shape == (4, 0)
    Y, codes, words = A.aps_linear(z(40, 0), z(9, 0), b, None, ACT["none"], ckpt_fmt=FMT["1-5-2"])  # K = 0: z = b
    assert torch.equal(Y, b.expand(40, 9))
    assert _same(A.aps_checkpoint_load(codes, words, FMT["1-5-2"], dtype=T).float(), torch.tensor(
        [0., 1, 2, 3, 4, 5, 6, 7, 8], device=dev).expand(40, 9))
    assert torch.equal(A.aps_linear_grad_input(z(4, 0), z(0, 6), torch.ones(4, 6, dtype=T, device=dev)),
                       torch.ones(4, 6, dtype=T, device=dev))
    none = torch.zeros(0, 6, dtype=torch.uint8, device=dev), torch.zeros(0, 1, dtype=torch.int32, device=dev)
    db = torch.full((3,), 5.0, device=dev)
    dW = A.aps_linear_grad_weight(z(0, 3), *none, FMT["1-4-3"], torch.full((3, 6), 2.0, device=dev), db)
    assert not bool(dW.any()) and not bool(db.any())
    dW = A.aps_linear_grad_weight(z(0, 3), *none, FMT["1-4-3"], torch.full((3, 6), 2.0, device=dev), db, True)
    assert bool((dW == 2).all())
    codes, words = A.aps_checkpoint_save(z(0, 6), FMT["1-4-3"])
    assert A.aps_checkpoint_load(codes, words, FMT["1-4-3"], dtype=T).shape == (0, 6)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("rows", [1000, 1001])
def test_empty_contractions_of_odd_rows(dev, t, rows):
    """No row to contract over, and operand rows that would have been copied."""
    T = TYPES[t]
    z = lambda *s: torch.zeros(*s, dtype=T, device=dev)  # noqa: E731
    none = torch.zeros(0, 520, dtype=torch.uint8, device=dev), torch.zeros(0, 5, dtype=torch.int32, device=dev)
    db = torch.full((rows,), 5.0, device=dev)
    dW = A.aps_linear_grad_weight(z(0, rows), *none, FMT["1-4-3"], torch.full((rows, 520), 2.0, device=dev), db)
    assert not bool(dW.any()) and not bool(db.any())
    r = torch.ones(333, rows, dtype=T, device=dev)
    assert torch.equal(A.aps_linear_grad_input(z(333, 0), z(0, rows), r), r)
    assert not bool(A.aps_linear(z(333, 0), z(rows, 0)).any())


@pytest.mark.parametrize("M,N,K", [(5, 70, 40), (40, 256, 128), (300, 256, 128), (300, 130, 101)])
@pytest.mark.parametrize("t", list(TYPES))
def test_bad_tokens_stay_their_own(dev, t, M, N, K):
    """NaN, INF and the type's lowest value in some tokens (padding that was
    never cleared): the other tokens' outputs and checkpoints hold no trace."""
    T = TYPES[t]
    X, W, b, _ = _problem(t, M, N, K, 3)
    bad = torch.zeros(M, dtype=torch.bool)
    bad[::4] = True
    Xb = X.clone()
    Xb[::12], Xb[4::12], Xb[8::12] = math.nan, math.inf, -torch.finfo(T).max
    run = lambda x: A.aps_linear(x.to(dev), W.to(dev), b.to(dev), None, ACT["gelu"], ckpt_fmt=FMT["1-4-3"])  # noqa: E731
    Y0 = run(X)[0]
    Y1, codes, words = run(Xb)
    assert torch.equal(Y0[~bad], Y1[~bad])
    assert bool(torch.isnan(Y1[::12]).all())
    zhat = A.aps_checkpoint_load(codes, words, FMT["1-4-3"], dtype=torch.float32)
    assert bool(torch.isfinite(zhat[~bad]).all()) and bool(torch.isnan(zhat[::12]).all())
    # their gradients, zero: dW is the other tokens'
    dZ = torch.randn(M, N, generator=_gen(8)).to(T)
    dZ[bad] = 0
    Xf = X.clone()
    Xf[bad] = -torch.finfo(T).max
    big, bw = A.aps_checkpoint_save(Xf.to(dev), FMT["1-5-2"])
    dW = A.aps_linear_grad_weight(dZ.to(dev), big, bw, FMT["1-5-2"])
    assert bool(torch.isfinite(dW).all())
    # an INF in the checkpoint reaches its own column of dW only
    Xi = X.clone()
    Xi[1, 7 % K] = math.inf
    for fmt in FMT:
        ci, wi = A.aps_checkpoint_save(Xi.to(dev), FMT[fmt])
        dW = A.aps_linear_grad_weight(dZ.to(dev), ci, wi, FMT[fmt])
        ok = torch.ones(K, dtype=torch.bool)
        ok[7 % K] = False
        assert bool(torch.isfinite(dW[:, ok]).all()) and not bool(torch.isfinite(dW[:, ~ok]).any())
        d = A.aps_linear_grad_input(torch.ones(M, N, dtype=T, device=dev), W.to(dev), None, ACT["silu"], ci, wi, FMT[fmt])
        assert bool(torch.isfinite(d).all())


def test_refusals_on_gpu_tensors(dev):
    z = lambda *s, T=torch.bfloat16: torch.zeros(*s, dtype=T, device=dev)  # noqa: E731
    X, W = z(8, 16), z(4, 16)
    codes, words = A.aps_checkpoint_save(X, FMT["1-4-3"])
    F = FMT["1-4-3"]
    bad = {
        "X int": lambda: A.aps_linear(X.int(), W),
        "types differ": lambda: A.aps_linear(X, W.half()),
        "bias type": lambda: A.aps_linear(X, W, z(4, T=torch.float32)),
        "bias short": lambda: A.aps_linear(X, W, z(3)),
        "inner": lambda: A.aps_linear(X, z(4, 15)),
        "1-D": lambda: A.aps_linear(X[0], W),
        "CPU": lambda: A.aps_linear(X.cpu(), W),
        "transposed": lambda: A.aps_linear(z(16, 8).t(), W),
        "overlapping rows": lambda: A.aps_linear(z(1, 16).expand(8, 16), W),
        "residual shape": lambda: A.aps_linear(X, W, None, z(8, 5)),
        "Y shape": lambda: A.aps_linear(X, W, Y=z(8, 5)),
        "codes without a format": lambda: A.aps_linear(X, W, codes=codes),
        "workspace type": lambda: A.aps_linear(X, W, workspace=z(64)),
        "words": lambda: A.aps_checkpoint_load(codes, words.repeat(2, 1), F, dtype=torch.float16),
        "words type": lambda: A.aps_checkpoint_load(codes, words.long(), F, dtype=torch.float16),
        "load type": lambda: A.aps_checkpoint_load(codes, words, F, dtype=torch.float64),
        "load no type": lambda: A.aps_checkpoint_load(codes, words, F),
        "grad without checkpoint": lambda: A.aps_linear_grad_input(z(8, 4), W, None, ACT["relu"]),
        "grad with a checkpoint unread": lambda: A.aps_linear_grad_input(z(8, 4), W, None, ACT["none"], codes, words, F),
        "rows": lambda: A.aps_linear_grad_weight(z(9, 4), codes, words, F),
        "dW type": lambda: A.aps_linear_grad_weight(z(8, 4), codes, words, F, z(4, 16)),
        "accumulate into nothing": lambda: A.aps_linear_grad_weight(z(8, 4), codes, words, F, accumulate=True),
        "act_grad shape": lambda: A.aps_activation_grad(z(8, 15), codes, words, F, ACT["relu"]),
    }
    for name, call in bad.items():
        with pytest.raises(ValueError):
            call()
            print(name)
    for st, call in {
        A.APS_ERR_UNSUPPORTED: lambda: A.aps_checkpoint_save(X, A.Format(3, 4)),
        A.APS_ERR_FORMAT: lambda: A.aps_checkpoint_save(X, A.Format(9, 4)),
    }.items():
        with pytest.raises(A.ApsError) as e:
            call()
        assert e.value.status == st
    with pytest.raises(A.ApsError):
        A.aps_linear(X, W, act=7)
    torch.cuda.synchronize()


# ------------------------------------------------------------ as they are used

class _Mlp:
    """Y = X + gelu(X W1^T + b1) W2^T + b2, the inputs of both layers and the
    pre-activation kept in 8 bits, the gradients in a worker's row of G."""

    def __init__(self, dev, t, M, H, F, fmt, seed=1, exact=False):
        T, g = TYPES[t], _gen(seed)
        self.T, self.fmt, self.dims = T, FMT[fmt], (M, H, F)
        draw = (lambda *s: torch.randint(-4, 5, s, generator=g) / 4) if exact else (  # noqa: E731
            lambda *s: torch.randn(*s, generator=g))
        self.X = draw(M, H).to(T).to(dev)
        self.W1, self.b1 = (draw(F, H) / 8).to(T).to(dev), (draw(F) / 8).to(T).to(dev)
        self.W2, self.b2 = (draw(H, F) / 8).to(T).to(dev), (draw(H) / 8).to(T).to(dev)
        self.dY = (draw(M, H) / 64).to(T).to(dev)
        self.sizes = [F * H, F, H * F, H]

    def forward(self, out=None):
        cx, wx = A.aps_checkpoint_save(self.X, self.fmt)
        Hid, cz, wz = A.aps_linear(self.X, self.W1, self.b1, None, A.APS_ACT_GELU, ckpt_fmt=self.fmt)
        ch, wh = A.aps_checkpoint_save(Hid, self.fmt)
        Y = A.aps_linear(Hid, self.W2, self.b2, self.X, Y=out)
        return Y, (cx, wx, cz, wz, ch, wh)

    def backward(self, saved, row, accumulate=False):
        M, H, F = self.dims
        cx, wx, cz, wz, ch, wh = saved
        o = [0]
        for s in self.sizes:
            o.append(o[-1] + s)
        A.aps_linear_grad_weight(self.dY, ch, wh, self.fmt, row[o[2]:o[3]].view(H, F), row[o[3]:o[4]], accumulate)
        dz = A.aps_linear_grad_input(self.dY, self.W2, None, A.APS_ACT_GELU, cz, wz, self.fmt)
        A.aps_linear_grad_weight(dz, cx, wx, self.fmt, row[o[0]:o[1]].view(F, H), row[o[1]:o[2]], accumulate)
        return A.aps_linear_grad_input(dz, self.W1, self.dY)

    def loss64(self, X, W1, b1, W2, b2):
        return ((X + R.act(X @ W1.t() + b1, "gelu") @ W2.t() + b2) * self.dY.cpu().double()).sum()


@pytest.mark.parametrize("t,M,H,F", [("bf16", 96, 128, 256), ("fp16", 50, 72, 130), ("fp32", 70, 67, 101)])
def test_gradients_of_a_block_and_their_synchronisation(dev, t, M, H, F):
    """Forward, backward and aps_sync of W = 2 workers.  The gradients are
    within what 4-bit significands of the checkpoints and the type's roundings
    allow of autograd's in float64; then the sum is the oracle's."""
    import numpy as np
    import oracle as O
    from tests._util import ofmt, same_f32

    n = 2 * F * H + F + H
    ld = -(-n // 64) * 64
    G = torch.zeros(2, ld, device=dev)
    for w in range(2):
        m = _Mlp(dev, t, M, H, F, "1-4-3", seed=w + 1)
        Y, saved = m.forward()
        dX = m.backward(saved, G[w])
        v = [p.cpu().double().requires_grad_() for p in (m.X, m.W1, m.b1, m.W2, m.b2)]
        z = v[0] @ v[1].t() + v[2]
        h = torch.nn.functional.gelu(z)
        y = v[0] + h @ v[3].t() + v[4]
        y.backward(m.dY.cpu().double())
        with torch.no_grad():
            norm = lambda a: float(a.norm())  # noqa: E731
            assert norm(Y.cpu().double() - y) <= 0.02 * norm(y)
            refs = [v[1].grad, v[2].grad, v[3].grad, v[4].grad]
            o = 0
            for s, ref in zip(m.sizes, refs):
                got = G[w, o:o + s].cpu().double().view(ref.shape)
                # each factor of each term is off by at most 2^-4 (a code of
                # x or h; the slope, which moves by at most 0.8 * 2^-4 |z|),
                # independently of the others: so the sums, by norm
                assert norm(got - ref) <= 2 * 2.0 ** -4 * norm(ref)
                o += s
            assert norm(dX.cpu().double() - v[0].grad) <= 0.12 * norm(v[0].grad)
    offs = np.concatenate([[0], np.cumsum(m.sizes)]).astype(np.int64)
    out, se, _, _ = A.aps_sync(G, n, torch.from_numpy(offs).to(dev), [A.Format(5, 2)])
    Gh = G.cpu().numpy()
    o_se = O.layer_scales(O.layer_maxabs(Gh, n, offs), 2, [ofmt(A.Format(5, 2))])
    assert same_f32(out.cpu().numpy(), O.sim_reduce(Gh, n, offs, o_se, [ofmt(A.Format(5, 2))]))


def test_gradients_against_differences(dev):
    """fp32 with inputs that the checkpoints hold exactly (quarters up to 1 in
    1-5-2): the weight and input gradients are those of central differences of
    the float64 loss, to the accuracy of the checkpoint of z and h."""
    M, N, K = 40, 24, 16
    g = _gen(4)
    X = torch.randint(-4, 5, (M, K), generator=g) / 4.0
    W = torch.randn(N, K, generator=g) / 4
    dY = torch.randn(M, N, generator=g)
    codes, words = A.aps_checkpoint_save(X.to(dev), FMT["1-5-2"])
    assert torch.equal(A.aps_checkpoint_load(codes, words, FMT["1-5-2"], dtype=torch.float32).cpu(), X)
    # z on values that 1-4-3 holds: the slope is taken at z itself
    zq = torch.randint(-12, 13, (M, N), generator=g) / 8.0
    cz, wz = A.aps_checkpoint_save(zq.to(dev), FMT["1-4-3"])
    assert torch.equal(A.aps_checkpoint_load(cz, wz, FMT["1-4-3"], dtype=torch.float32).cpu(), zq)
    h = 1e-5
    for act in ("gelu", "silu"):
        dZ = A.aps_activation_grad(dY.to(dev), cz, wz, FMT["1-4-3"], ACT[act])
        num = dY.double() * (R.act(zq.double() + h, act) - R.act(zq.double() - h, act)) / (2 * h)
        assert float((dZ.cpu().double() - num).abs().max()) <= 1e-6 * float(dY.abs().max())
        # through the product: d sum(dY * act(z + X' W^T)) / dX' at 0 is dZ W
        dX = A.aps_linear_grad_input(dZ, W.to(dev))
        D = torch.randn(M, K, generator=g).double()
        f = lambda e: (dY.double() * R.act(zq.double() + e * D @ W.double().t(), act)).sum()  # noqa: E731
        assert abs(float((dX.cpu().double() * D).sum()) - float((f(h) - f(-h)) / (2 * h))) <= 1e-4
        # and the weights': d sum(dY * act(z + X W'^T)) / dW' at 0 is dZ^T X
        db = torch.empty(N, device=dev)
        dW = A.aps_linear_grad_weight(dZ, codes, words, FMT["1-5-2"], dbias=db)
        D = torch.randn(N, K, generator=g).double()
        f = lambda e: (dY.double() * R.act(zq.double() + e * X.double() @ D.t(), act)).sum()  # noqa: E731
        assert abs(float((dW.cpu().double() * D).sum()) - float((f(h) - f(-h)) / (2 * h))) <= 1e-4
        assert float((db.cpu().double() - dZ.cpu().double().sum(0)).abs().max()) <= 1e-4


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_captured_and_replayed(dev, t):
    """A step captured in a HIP graph, replayed on changing inputs with eager
    work in between: every replay is the eager result, to the last bit."""
    M, H, F = 64, 128, 512
    n = 2 * F * H + F + H
    m = _Mlp(dev, t, M, H, F, "1-4-3")
    row = torch.zeros(n, device=dev)

    def step(r):
        Y, saved = m.forward()
        return Y, m.backward(saved, r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(row)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, dX = step(row)
    for k in range(4):
        m.X.copy_(torch.randn(M, H, generator=_gen(50 + k)).to(m.T))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (Y, dX, row)]
        eager = torch.zeros_like(row)
        Ye, dXe = step(eager)
        for a, b in zip(got, (Ye, dXe, eager)):
            assert torch.equal(a, b)


def test_streams_and_workspaces(dev):
    """Two streams at once, each with a workspace of its own; a workspace's
    contents do not matter, a short one is refused."""
    M, N, K = 48, 256, 4096
    X, W, b, r = (v.to(dev) for v in _problem("bf16", M, N, K, 9))
    need = A.aps_linear_workspace_bytes(A.APS_LINEAR_FORWARD, M, N, K, torch.bfloat16)
    ref = A.aps_linear(X, W, b, r)
    assert need > 0
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            ws = torch.full((need,), 255, dtype=torch.uint8, device=dev)
            outs.append(A.aps_linear(X, W, b, r, workspace=ws))
    out = torch.empty_like(ref)
    torch.cuda.synchronize()
    A.aps_linear(X, W, b, r, Y=out, stream=streams[0])
    outs += [A.aps_linear(X, W, b, r, stream=streams[1]), A.aps_linear(X, W, b, r, stream=streams[1].cuda_stream),
             A.aps_linear(X, W, b, r, stream=0)]
    torch.cuda.synchronize()
    for o in outs + [out]:
        assert torch.equal(o, ref)
    with pytest.raises(A.ApsError) as e:
        A.aps_linear(X, W, b, r, workspace=torch.empty(need - 1, dtype=torch.uint8, device=dev))
    assert e.value.status == A.APS_ERR_SIZE


# Products for every shape of the tile kernel (256 x 256, 128 x 128 and 128 x 64
# tiles), split and whole, the few rows of a decoding step, and odd rows that
# are copied; in float64 on the GPU.
LARGE = [(700, 700, 700), (333, 1000, 520), (2304, 2048, 320), (4096, 4096, 128), (40, 4096, 512), (1, 4096, 1024),
         (32, 1000, 4100), (20, 333, 77), (512, 520, 4096), (4096, 264, 520), (130, 2000, 1000)]


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("t", list(TYPES))
def test_larger_products(dev, t, M, N, K):
    T = TYPES[t]
    g = torch.Generator(device=dev)
    g.manual_seed(M + N + K)
    rnd = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    X, W = rnd(M, K).to(T), (rnd(N, K) / math.sqrt(K)).to(T)
    b, r, dZ = rnd(N).to(T), rnd(M, N).to(T), (rnd(M, N) / 16).to(T)
    X64, W64, b64, r64, dZ64 = (v.double() for v in (X, W, b, r, dZ))
    fmt = "1-4-3" if (M + N) % 2 else "1-5-2"
    # forward, with and without a checkpoint
    z = X64 @ W64.t() + b64
    ez = R.sums_bound(W64.abs().t(), X64.abs(), b64.abs())
    ref = R.act(z, "gelu") + r64
    e = R.LIPSCHITZ * ez + R.ACT_ULPS * z.abs() + 2.0 ** -24 * ref.abs()
    tol = e + R.half_step(T) * (ref.abs() + e) + R.tiny(T)
    Y = A.aps_linear(X, W, b, r, ACT["gelu"])
    assert bool(((Y.double() - ref).abs() <= tol).all())
    Y, codes, words = A.aps_linear(X, W, b, r, ACT["gelu"], ckpt_fmt=FMT[fmt])
    assert bool(((Y.double() - ref).abs() <= tol).all())
    _check_zhat(codes, words, fmt, T, z.cpu(), ez.cpu())
    # the input gradient at this checkpoint's shape: the layer below has N out features
    s = R.slope(R.load(codes, words, fmt), "silu")
    up = (rnd(M, K) / 16).to(T)          # the gradient of a layer with K out and N in features
    W2 = (rnd(K, N) / math.sqrt(K)).to(T)
    d = up.double() @ W2.double()
    ref = d * s + r64
    ed = R.sums_bound(W2.double().abs(), up.double().abs())
    e = R.LIPSCHITZ * ed + d.abs() * 2 * R.ACT_ULPS + 2.0 ** -23 * ref.abs()
    tol = e + R.half_step(T) * (ref.abs() + e) + R.tiny(T)
    dX = A.aps_linear_grad_input(up, W2, r, ACT["silu"], codes, words, FMT[fmt])
    assert bool(((dX.double() - ref).abs() <= tol).all())
    # the weight gradient
    cx, wx = A.aps_checkpoint_save(X, FMT[fmt])
    x = R.load(cx, wx, fmt)
    db = torch.empty(N, device=dev)
    dW = A.aps_linear_grad_weight(dZ, cx, wx, FMT[fmt], dbias=db)
    ref = dZ64.t() @ x
    tol = R.sums_bound(x.abs(), dZ64.abs().t()) + 2.0 ** -24 * ref.abs()
    assert bool(((dW.double() - ref).abs() <= tol).all())
    assert bool(((db.double() - dZ64.sum(0)).abs() <= (M + 2) * 2.0 ** -23 * dZ64.abs().sum(0)).all())


@pytest.mark.parametrize("t", ["bf16", "fp16"])
def test_subnormal_operands_count(dev, t):
    """The matrix instructions take the type's subnormals as they are."""
    T = TYPES[t]
    tiny = torch.finfo(T).smallest_normal
    X = torch.full((40, 64), tiny / 4, dtype=T, device=dev)
    W = torch.full((128, 64), 2.0, dtype=T, device=dev)
    want = torch.full((40, 128), 64 * 2 * tiny / 4, dtype=T, device=dev)
    assert torch.equal(A.aps_linear(X, W), want) and torch.equal(A.aps_linear(X[:3], W), want[:3])
    assert torch.equal(A.aps_linear_grad_input(X, W.t().contiguous()), want)


def test_rows_in_a_long_buffer(dev):
    """Operands and outputs whose rows lie beyond 2^31 elements of each other's
    start: strides of 2^20 and 2100 rows."""
    ld, M, N, K = 1 << 20, 2100, 96, 64
    buf = torch.zeros(M * ld, dtype=torch.bfloat16, device=dev)
    X = buf.view(M, ld)[:, :K]
    Y = buf.view(M, ld)[:, 1024:1024 + N]
    X.copy_(torch.randn(M, K, generator=_gen(1)))
    W = torch.randn(N, K, generator=_gen(2)).to(dev).bfloat16()
    A.aps_linear(X, W, Y=Y)
    assert torch.equal(Y, A.aps_linear(X.contiguous(), W))
    codes = buf.view(torch.uint8).view(M, 2 * ld)[:, 8192:8192 + K]
    words = torch.empty(66, 1, dtype=torch.int32, device=dev)
    A.aps_checkpoint_save(X, FMT["1-4-3"], codes, words)
    rc, rw = A.aps_checkpoint_save(X.contiguous(), FMT["1-4-3"])
    assert torch.equal(codes, rc) and torch.equal(words, rw)
    # strides choose the kernel, and with it the sums' order: within the sums' bound
    dW = A.aps_linear_grad_weight(Y, codes, words, FMT["1-4-3"])
    x, y = R.load(rc, rw, "1-4-3"), Y.double()
    ref = y.t() @ x
    assert bool(((dW.double() - ref).abs() <= R.sums_bound(x.abs(), y.abs().t()) + 2.0 ** -24 * ref.abs()).all())
    del buf, X, Y, codes
    torch.cuda.empty_cache()
