"""Host-side checks of the linear layer's calls and the pins of their float64
reference (no GPU: every call of the library here is refused or empty)."""
import ctypes
import math
import os

import pytest
import torch

import oracle as O
from paper_1911_08907_amd import aps as A
from paper_1911_08907_amd import build as B
from tests import linear_ref as R
from tests.test_abi import GOOD, HEADER, MIS, no_gpu

F43, F52 = A.Format(4, 3).c(), A.Format(5, 2).c()
BF16, F32 = A.APS_DTYPE_BF16, A.APS_DTYPE_F32
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(A.LIB_PATH):
        B.build()
    return A.lib()


def test_the_header_is_the_binding(lib):
    import re
    txt = open(os.path.join(os.path.dirname(HEADER), "aps_linear.h")).read()
    names = set(re.findall(r"\b(aps_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", txt, flags=re.S)))
    assert names == set(A.LINEAR_EXPORTS)
    for name in names:
        assert hasattr(lib, name)


def _linear(lib, **kw):
    a = dict(X=GOOD, ldx=64, W=GOOD, ldw=64, bias=None, R=None, ldr=0, Y=GOOD, ldy=64, M=8, N=64, K=64, dtype=BF16,
             act=0, fmt=F43, codes=None, ldc=0, exps=None, ws=None, wb=1 << 40, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.aps_linear(*a.values())


@no_gpu
def test_linear_refusals(lib):
    bad = [({"M": -1}, "SIZE"), ({"N": (1 << 22) + 1}, "SIZE"), ({"dtype": 3}, "UNSUPPORTED"), ({"act": 4}, "UNSUPPORTED"),
           ({"act": -1}, "UNSUPPORTED"), ({"X": None}, "NULL"), ({"W": None}, "NULL"), ({"Y": None}, "NULL"),
           ({"ldx": 63}, "SIZE"), ({"ldw": 63}, "SIZE"), ({"ldy": 63}, "SIZE"), ({"ldx": 1 << 31}, "SIZE"),
           ({"X": ODD}, "ALIGN"), ({"dtype": F32, "W": ctypes.c_void_p(4098)}, "ALIGN"), ({"R": GOOD, "ldr": 5}, "SIZE"),
           ({"bias": ODD}, "ALIGN"), ({"codes": GOOD, "ldc": 64}, "NULL"), ({"exps": GOOD}, "NULL"),
           ({"codes": GOOD, "ldc": 63, "exps": GOOD}, "SIZE"), ({"codes": GOOD, "ldc": 64, "exps": ODD}, "ALIGN"),
           ({"codes": GOOD, "ldc": 64, "exps": GOOD, "fmt": A.Format(5, 10).c()}, "UNSUPPORTED"),
           ({"codes": GOOD, "ldc": 64, "exps": GOOD, "fmt": A.Format(4, 3, 8).c()}, "UNSUPPORTED"),
           ({"codes": GOOD, "ldc": 64, "exps": GOOD, "fmt": A.Format(1, 3).c()}, "FORMAT"),
           ({"M": 1 << 22, "N": 1 << 22, "ldy": 1 << 22}, "SIZE"),
           ({"K": 4096, "ldx": 4096, "ldw": 4096}, "NULL"),                        # the workspace
           ({"K": 4096, "ldx": 4096, "ldw": 4096, "ws": GOOD, "wb": 16}, "SIZE"),
           ({"K": 4096, "ldx": 4096, "ldw": 4096, "ws": MIS}, "ALIGN")]
    for kw, name in bad:
        assert _linear(lib, **kw) == getattr(A, "APS_ERR_" + name), kw
    # nothing to do: nothing is asked of the arrays
    assert _linear(lib, M=0, X=None, Y=None, W=None) == A.APS_OK
    assert _linear(lib, N=0, X=None, Y=None, W=None) == A.APS_OK


@no_gpu
def test_gradient_refusals(lib):
    def gi(**kw):
        a = dict(dZ=GOOD, lddz=64, W=GOOD, ldw=64, R=None, ldr=0, act=2, fmt=F43, codes=GOOD, ldc=64, exps=GOOD, dX=GOOD,
                 lddx=64, M=8, N=64, K=64, dtype=BF16, ws=None, wb=0, stream=None)
        a.update(kw)
        return lib.aps_linear_grad_input(*a.values())

    def gw(**kw):
        a = dict(dZ=GOOD, lddz=64, fmt=F43, codes=GOOD, ldc=64, exps=GOOD, dW=GOOD, lddw=64, db=None, M=8, N=64, K=64,
                 dtype=BF16, flags=0, ws=None, wb=0, stream=None)
        a.update(kw)
        return lib.aps_linear_grad_weight(*a.values())

    for kw, name in [({"K": -1}, "SIZE"), ({"act": 9}, "UNSUPPORTED"), ({"codes": None}, "NULL"), ({"exps": None}, "NULL"),
                     ({"fmt": A.Format(5, 3).c()}, "UNSUPPORTED"), ({"dZ": None}, "NULL"), ({"dX": None}, "NULL"),
                     ({"lddx": 3}, "SIZE"), ({"R": ODD, "ldr": 64}, "ALIGN"),
                     ({"N": 8192, "lddz": 8192}, "NULL")]:
        assert gi(**kw) == getattr(A, "APS_ERR_" + name), kw
    for kw, name in [({"flags": 2}, "UNSUPPORTED"), ({"codes": None}, "NULL"), ({"exps": None}, "NULL"), ({"dW": None}, "NULL"),
                     ({"dW": ctypes.c_void_p(4098)}, "ALIGN"), ({"db": ctypes.c_void_p(4098)}, "ALIGN"),
                     ({"lddw": 63}, "SIZE"), ({"lddz": 63}, "SIZE"), ({"ldc": 63}, "SIZE"),
                     ({"K": 0, "db": GOOD}, "SIZE"), ({"M": 8192}, "NULL")]:
        assert gw(**kw) == getattr(A, "APS_ERR_" + name), kw
    assert gi(M=0, dZ=None, dX=None, codes=None, exps=None) == A.APS_OK
    assert gw(N=0, dZ=None, dW=None, codes=None, exps=None) == A.APS_OK


@no_gpu
def test_checkpoint_refusals(lib):
    f = lib.aps_checkpoint_save
    assert f(None, 64, 8, 64, BF16, F43, GOOD, 64, GOOD, None) == A.APS_ERR_NULL
    assert f(GOOD, 64, 8, 64, BF16, F43, None, 64, GOOD, None) == A.APS_ERR_NULL
    assert f(GOOD, 64, 8, 64, BF16, F43, GOOD, 64, None, None) == A.APS_ERR_NULL
    assert f(GOOD, 63, 8, 64, BF16, F43, GOOD, 64, GOOD, None) == A.APS_ERR_SIZE
    assert f(ODD, 64, 8, 64, BF16, F43, GOOD, 64, GOOD, None) == A.APS_ERR_ALIGN
    assert f(GOOD, 64, 8, 64, 5, F43, GOOD, 64, GOOD, None) == A.APS_ERR_UNSUPPORTED
    assert f(None, 64, 0, 64, BF16, F43, None, 64, None, None) == A.APS_OK
    f = lib.aps_checkpoint_load
    assert f(None, 64, GOOD, 8, 64, F43, 0, GOOD, 64, BF16, None) == A.APS_ERR_NULL
    assert f(GOOD, 64, GOOD, 8, 64, F43, 5, GOOD, 64, BF16, None) == A.APS_ERR_UNSUPPORTED
    assert f(GOOD, 64, GOOD, 8, 64, F43, 0, GOOD, 63, BF16, None) == A.APS_ERR_SIZE
    f = lib.aps_activation_grad
    assert f(None, 64, 1, F43, GOOD, 64, GOOD, GOOD, 64, 8, 64, BF16, None) == A.APS_ERR_NULL
    assert f(GOOD, 64, 1, F43, GOOD, 64, GOOD, None, 64, 8, 64, BF16, None) == A.APS_ERR_NULL
    assert f(GOOD, 64, -1, F43, GOOD, 64, GOOD, GOOD, 64, 8, 64, BF16, None) == A.APS_ERR_UNSUPPORTED


def test_workspace_bytes(lib):
    w = lib.aps_linear_workspace_bytes
    assert w(0, 1 << 22, 1 << 22, 8, BF16) == 0 and w(3, 8, 8, 8, BF16) == 0 and w(0, 8, 8, 8, 9) == 0
    assert w(0, 0, 64, 64, BF16) == 0
    for op in range(3):
        for dims in ((1, 1, 1), (16, 4096, 1024), (1, 64, 65536), (4096, 4096, 4096), (65536, 64, 64), (100000, 3, 5)):
            for dt in range(3):
                assert w(op, *dims, dt) < 1 << 31


def test_tile_kernels_keep_their_sums_in_registers():
    """No instance of the tile kernel takes scratch: accumulators that spilled
    in the stage loop ran six times slower."""
    from tests import test_kernel_resources as TR
    msgpack = pytest.importorskip("msgpack")
    if not os.path.exists(A.LIB_PATH):
        pytest.skip("libaps.so is not built")
    blob = open(A.LIB_PATH, "rb").read()
    scratch = {k[".name"]: k[".private_segment_fixed_size"]
               for elf in TR._code_objects(blob) for k in TR._kernels(elf, msgpack)}
    tile = {n: v for n, v in scratch.items() if "k_lin_tile" in n}
    assert len(tile) == 2 * 3 * 2 * 3 + 3 * 2 * 2 and not any(tile.values()), tile


def test_workspace_bytes_needs_a_known_type():
    with pytest.raises(ValueError):
        A.aps_linear_workspace_bytes(0, 8, 8, 8, torch.float64)


def test_binding_refuses_cpu_tensors():
    X, W = torch.zeros(4, 8), torch.zeros(3, 8)
    c, e = torch.zeros(4, 8, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32)
    for call in (lambda: A.aps_linear(X, W), lambda: A.aps_linear_grad_input(X, W),
                 lambda: A.aps_linear_grad_weight(X, c, e, A.Format(4, 3)), lambda: A.aps_checkpoint_save(X, A.Format(4, 3)),
                 lambda: A.aps_checkpoint_load(c, e, A.Format(4, 3), dtype=torch.float32),
                 lambda: A.aps_activation_grad(X, c, e, A.Format(4, 3), 1), lambda: A.aps_linear(None, W)):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------- the reference's own pins

def test_reference_table_is_the_formats():
    """1-5-2 is OCP E5M2; 1-4-3 is E4M3 below 248."""
    c = torch.arange(256, dtype=torch.uint8)
    a, b = R.table("1-5-2"), c.view(torch.float8_e5m2).double()
    assert bool(((a == b) | (a.isnan() & b.isnan())).all())
    a, b = R.table("1-4-3"), c.view(torch.float8_e4m3fn).double()
    low = (c & 127) < 0x78
    assert torch.equal(a[low], b[low])


@pytest.mark.parametrize("fmt", list(R.FORMATS))
def test_reference_codes_are_the_oracles(fmt):
    """A block's codes are the oracle's cast of the block as one layer with the
    same exponent, which is the oracle's own for N = 1 where it is not held."""
    import numpy as np
    e, m, _ = R.FORMATS[fmt]
    g = torch.Generator().manual_seed(3)
    x = torch.randn(32, 128, generator=g) * torch.exp2(torch.randint(-9, 9, (32, 128), generator=g).float())
    codes, words = R.save(x.double(), fmt, torch.float32)
    flat = x.numpy().reshape(1, -1).copy()
    offs = np.array([0, flat.size], np.int64)
    of = O.Format(e, m)
    se = O.layer_scales(O.layer_maxabs(flat, flat.size, offs), 1, of)
    assert int(words[0, 0]) == int(se[0]) & 0xFFFF
    q = torch.from_numpy(O.quantize(flat, flat.size, offs, se, of)).double().view(32, 128)
    assert torch.equal(R.table(fmt)[codes.long()], q) and torch.equal(torch.signbit(q), codes >= 128)


def test_reference_round_trip_and_activations():
    g = torch.Generator().manual_seed(4)
    x = torch.randn(40, 200, generator=g).double()
    for fmt, (e, m, _) in R.FORMATS.items():
        v = R.load(*R.save(x, fmt, torch.float32), fmt)
        assert bool(((v - x).abs() <= x.abs() * 2.0 ** -(m + 1) + 2.0 ** -6).all())
        again = R.save(v, fmt, torch.float32)
        assert torch.equal(R.load(*again, fmt), v)
    z = torch.linspace(-8, 8, 401, dtype=torch.float64, requires_grad=True)
    for name, f in (("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu), ("relu", torch.relu)):
        y = f(z)
        assert float((y - R.act(z, name)).detach().abs().max()) < 1e-12
        d, = torch.autograd.grad(y.sum(), z)
        assert float((d - R.slope(z, name)).detach().abs().max()) < 1e-12
    inf = torch.tensor([math.inf, -math.inf, math.nan], dtype=torch.float64)
    for name in ("gelu", "silu", "relu"):
        assert R.act(inf, name)[:2].tolist() == [math.inf, 0.0]
        assert float((R.slope(inf, name)[:2] - torch.tensor([1.0, 0.0])).abs().max()) < 1e-300
        assert bool(R.act(inf, name)[2].isnan()) and bool(R.slope(inf, name)[2].isnan())
