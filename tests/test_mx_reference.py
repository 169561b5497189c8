"""The definition the kernels are tested against, pinned by hand, and the library's refusals (host only)."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_1912_04822_amd import molgrid  # noqa: E402
from mx_reference import FORMATS, pack, unpack, values  # noqa: E402


def test_levels():
    assert len(FORMATS["int8"].levels) == 128 and FORMATS["int8"].levels[-1] == 127
    assert len(FORMATS["e4m3"].levels) == 127 and FORMATS["e4m3"].levels[-1] == 448
    got = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, np.array(FORMATS["e4m3"].levels))
    for f in FORMATS.values():
        assert all(a < b for a, b in zip(f.levels, f.levels[1:]))


@pytest.mark.parametrize("fmt,x,scale,want", [
    # amax 1: k = 0; int8 steps of 2^-6
    ("int8", [1.0, 0.0078125, -0.0234375], 121, [1.0, 0.0, -0.03125]),
    # 1.99 < 255/128 keeps k = 0, 1.9921875 does not
    ("int8", [1.99, 0.01], 121, [1.984375, 0.015625]),
    ("int8", [1.9921875, 0.01], 122, [2.0, 0.0]),
    ("e4m3", [448.0, 1.0625, 0.001], 127, [448.0, 1.0, 0.001953125]),
    ("e4m3", [463.9, 17.0], 127, [448.0, 16.0]),
    # 464 / 2 = 232 lies halfway between 224 and 240; the even one is 224
    ("e4m3", [464.0, 17.0], 128, [448.0, 16.0]),
    ("e2m1", [6.9, 0.25, 0.75, 2.5, 5.0], 127, [6.0, 0.0, 1.0, 2.0, 4.0]),
    ("e2m1", [7.0, 0.5], 128, [8.0, 0.0]),
])
def test_blocks_by_hand(fmt, x, scale, want):
    codes, scales = pack(np.array([x]), fmt)
    assert scales[0, 0] == scale and not scales[0, 1:].any()
    assert np.array_equal(values(np.array([x]), fmt)[0], want)
    assert codes.shape == (1, 16 if fmt == "e2m1" else 32)


def test_bounds_of_the_rounding():
    """Half a step: int8 2^(k-7); e4m3 2^-4 and e2m1 2^-2 of the number, or half the smallest step."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 320)) * np.exp(2 * rng.standard_normal((200, 320)))
    for fmt, f in FORMATS.items():
        _, s = pack(x, fmt)
        p = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, axis=1)[:, :320]
        err = np.abs(values(x, fmt) - x)
        rel = {"int8": 0.0, "e4m3": 2.0 ** -4, "e2m1": 2.0 ** -2}[fmt]
        assert (err <= np.maximum(rel * np.abs(x), p * (f.levels[1] - f.levels[0]) / 2)).all()


def test_a_block_that_is_not_finite():
    x = np.ones((2, 96))
    x[0, 40], x[1, 0] = np.inf, np.nan
    for fmt in FORMATS:
        codes, scales = pack(x, fmt)
        assert scales[0, 1] == 255 and scales[1, 0] == 255
        v = unpack(codes, scales, 96, fmt)
        assert np.isnan(v[0, 32:64]).all() and np.isnan(v[1, :32]).all()
        assert (v[0, :32] == 1).all() and (v[0, 64:] == 1).all() and (v[1, 32:] == 1).all()


# ---- refusals: on the host, before anything is enqueued ----

OK, ENULL, ESHAPE, EPARAM, EWORKSPACE, EALIGN = 0, -1, -2, -3, -4, -7
P = 1 << 20                                         # an address no call touches: every call below is refused


@pytest.fixture(scope="module")
def L():
    return molgrid.lib()


def test_pack_and_unpack_refuse(L):
    def pack_(fmt=0, dtype=0, rows=2, cols=40, x=P, stride=40, codes=P, scales=P):
        return L.mg_mx_pack(fmt, dtype, rows, cols, x, stride, codes, scales, None)

    def unpack_(fmt=0, dtype=0, rows=2, cols=40, x=P, stride=40, codes=P, scales=P):
        return L.mg_mx_unpack(fmt, dtype, rows, cols, codes, scales, x, stride, None)

    for f in (pack_, unpack_):
        for k in ("x", "codes", "scales"):
            assert f(**{k: None}) == ENULL
        assert f(fmt=3) == f(fmt=-1) == f(dtype=3) == f(dtype=-1) == EPARAM
        assert f(rows=0) == f(cols=0) == f(rows=-1) == f(stride=39) == ESHAPE
        assert f(rows=1 << 31) == f(rows=1, cols=1 << 37) == f(rows=1 << 30, cols=500, stride=500) == ESHAPE
        assert f(x=P + 2) == f(dtype=1, x=P + 1) == f(codes=P + 8) == f(scales=P + 2) == EALIGN


def test_weight_gradient_refuses(L):
    need = ctypes.c_size_t()
    assert L.mg_mx8_weight_gradient_workspace(50, 2040, 28, 256, ctypes.byref(need)) == OK and need.value > 0

    def call(fmt=0, dtype=0, B=50, N=2040, T=28, E=256, grad=P, stride=28, codes=P, scales=P, natoms=None, dw=P,
             db=None, ws=P, size=need.value):
        return L.mg_mx8_weight_gradient(fmt, dtype, B, N, T, E, grad, stride, codes, scales, natoms, dw, db, ws,
                                        size, None)

    for k in ("grad", "codes", "scales", "dw"):
        assert call(**{k: None}) == ENULL
    assert call(fmt=2) == call(fmt=-1) == call(dtype=7) == EPARAM
    for k in ("B", "N", "T", "E"):
        assert call(**{k: 0}) == ESHAPE
    assert call(T=65536, stride=65536) == call(E=(1 << 20) + 1) == call(stride=27) == ESHAPE
    assert call(B=1 << 16, N=1 << 15) == ESHAPE
    assert call(grad=P + 2) == call(codes=P + 4) == call(scales=P + 1) == call(natoms=P + 2) == EALIGN
    assert call(dw=P + 2) == call(db=P + 1) == EALIGN
    assert call(ws=None) == call(ws=P + 16) == call(size=need.value - 1) == EWORKSPACE
    assert L.mg_mx8_weight_gradient_workspace(1, 1, 1, 1, None) == ENULL
    assert L.mg_mx8_weight_gradient_workspace(0, 1, 1, 1, ctypes.byref(need)) == ESHAPE


def test_products_refuse(L):
    def product(dtype=0, M=300, N=300, K=100, a=P, asc=P, b=P, bsc=P, bias=None, out=P, stride=300):
        return L.mg_mx4_product(dtype, M, N, K, a, asc, b, bsc, bias, out, stride, None)

    for k in ("a", "asc", "b", "bsc", "out"):
        assert product(**{k: None}) == ENULL
    assert product(dtype=3) == EPARAM
    assert product(M=0) == product(N=0) == product(K=0) == product(stride=299) == ESHAPE
    assert product(M=(1 << 30) + 1) == product(N=1 << 20, stride=1 << 20) == product(K=(1 << 24) + 1) == ESHAPE
    assert product(a=P + 8) == product(bsc=P + 2) == product(bias=P + 2) == product(out=P + 2) == EALIGN

    need = ctypes.c_size_t()
    assert L.mg_mx4_linear_workspace(3000, 3000, 1000, ctypes.byref(need)) == OK and need.value >= 3000 * (16 * 32 + 32)
    size = need.value
    assert L.mg_mx4_linear_workspace(300, 28, 100, ctypes.byref(need)) == OK and need.value == 0
    assert L.mg_mx4_linear_workspace(300, 0, 100, ctypes.byref(need)) == ESHAPE
    assert L.mg_mx4_linear_workspace(300, 300, 100, None) == ENULL

    def linear(dtype=0, M=3000, N=3000, K=1000, x=P, xs=1000, w=P, wsc=P, bias=None, out=P, stride=3000, ws=P, size=size):
        return L.mg_mx4_linear(dtype, M, N, K, x, xs, w, wsc, bias, out, stride, ws, size, None)

    for k in ("x", "w", "wsc", "out"):
        assert linear(**{k: None}) == ENULL
    assert linear(dtype=-1) == EPARAM
    assert linear(M=0) == linear(xs=999) == linear(stride=2999) == ESHAPE
    assert linear(x=P + 1) == linear(w=P + 8) == linear(wsc=P + 1) == linear(out=P + 3) == EALIGN
    assert linear(ws=None) == linear(ws=P + 8) == linear(size=size - 1) == EWORKSPACE


def test_binding_refuses():
    x = torch.zeros((4, 40))
    with pytest.raises(ValueError):
        molgrid.mg_mx_pack(x)                       # not on the device
    with pytest.raises(ValueError):
        molgrid.mg_mx_pack(x, "e5m2")
    with pytest.raises(ValueError):
        molgrid.mg_mx_pack(torch.zeros(()), "int8")
    with pytest.raises(TypeError):
        molgrid.mg_mx_pack(x.double())
    with pytest.raises(TypeError):
        molgrid.mg_mx4_linear(x, x)
    t = molgrid.MXTensor(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8), (4, 40), "int8")
    assert t.rows == 4
    with pytest.raises(ValueError):
        molgrid.mg_mx4_linear(x, t)                 # eight bits where four are wanted
    with pytest.raises(ValueError):
        molgrid.mg_mx_unpack(t)                     # codes not on the device


def test_the_native_side_leaves_other_calls_alone():
    """Calls that are not of the common form are handed back (None) before anything is touched."""
    molgrid.lib()
    b = molgrid._binding
    x, codes, scales = torch.zeros((4, 40)), torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8)
    assert b.pack(x, 0, 0, 0) is None and b.pack(None, 0, 0, 0) is None and b.pack(x) is None
    assert b.pack(x, "int8", 0, 0) is None and b.pack(x, 0, 1 << 70, 0) is None
    assert b.unpack(codes, scales, (4, 40), 0, 0, 0, 0) is None
    assert b.unpack(codes, scales, [4, 40], 0, 0, 0, 0) is None
    assert b.gradient(x, codes, scales, (4, 40), 0, None, 0, 0) is None
    assert b.product(codes, scales, (4, 40), codes, scales, (4, 40), None, 0, 0, 0) is None
    assert b.linear(x, codes, scales, (4, 40), None, 0, 0) is None
    with pytest.raises(TypeError):
        b.bind(1)


def test_sizes_past_an_int_are_refused():
    molgrid._fits("mg_mx4_product", 1, 0x7fffffff)
    with pytest.raises(molgrid.MolgridError) as e:
        molgrid._fits("mg_mx4_product", 5, 1 << 32)
    assert e.value.code == ESHAPE


def test_plain_tensors_in_place_of_packed_ones_are_refused():
    x = torch.zeros((4, 32))
    packed = molgrid.MXTensor(x.to(torch.uint8), x.to(torch.uint8), (4, 32), "e2m1")
    for call in (lambda: molgrid.mg_mx_unpack(x), lambda: molgrid.mg_mx4_product(x, packed),
                 lambda: molgrid.mg_mx4_product(packed, x), lambda: molgrid.mg_mx4_linear(x, x),
                 lambda: molgrid.mg_mx8_weight_gradient(x, x)):
        with pytest.raises(TypeError):
            call()
