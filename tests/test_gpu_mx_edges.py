"""Microscaled formats where codes, counts and gradients are unusual: codes that no pack makes, gradients that
are not finite, counts at the ends of their type."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1912_04822_amd import molgrid as mgd  # noqa: E402
from paper_1912_04822_amd.autograd import AtomTyper, saved_in_8_bits  # noqa: E402

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def same(a, b):
    """Equal to the bit as numbers; NaN equals NaN."""
    a, b = a.double().cpu(), b.double().cpu()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0, 100, 127, 254])
def test_every_e4m3_code(dtype, scale):
    """All 256 codes, whoever made them: 0x7f and 0xff are the type's NaN."""
    t = DTYPES[dtype]
    codes = torch.arange(256, dtype=torch.uint8).view(8, 32)
    scales = torch.full((8, 4), scale, dtype=torch.uint8)
    packed = mgd.MXTensor(codes.cuda(), scales.cuda(), (8, 32), "e4m3")
    top = torch.finfo(t).max
    want = (codes.view(torch.float8_e4m3fn).double() * 2.0 ** (scale - 127)).clamp(-top, top).to(t)
    assert want.isnan().sum() == 2
    for got in (mgd.mg_mx_unpack(packed, dtype=t), mgd.mg_mx_unpack(packed, out=torch.empty((8, 32), dtype=t, device="cuda"))):
        assert same(got, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [3, 20])
def test_a_block_of_scale_255_is_nan_whatever_its_codes(fmt, dtype, T):
    codes = torch.randint(1, 120, (40, 64), generator=torch.Generator().manual_seed(1)).to(torch.uint8)
    scales = torch.full((40, 4), 120, dtype=torch.uint8)
    scales[7, 1] = 255
    packed = mgd.MXTensor(codes.cuda(), scales.cuda(), (40, 64), fmt)
    assert mgd.mg_mx_unpack(packed)[7, 32:].isnan().all()
    dw, db = mgd.mg_mx8_weight_gradient(torch.ones((40, T), device="cuda", dtype=DTYPES[dtype]), packed)
    assert dw[:, 32:].isnan().all() and dw[:, :32].isfinite().all() and (db == 40).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T,E", [(3, 20), (5, 100), (20, 100)])
def test_infinite_gradients(fmt, dtype, T, E):
    """An infinity in the gradient is one in the sums it belongs to: of its sign times the number's, NaN where the
    number is 0, where both signs meet or where a NaN stands beside it."""
    t, inf = DTYPES[dtype], float("inf")
    gen = torch.Generator().manual_seed(T)
    x = torch.randn((1, 70, E), generator=gen)
    x[0, 5, 4] = 0.0
    x[0, 5, 6] = x[0, 9, 6]
    x[0, 5, 7], x[0, 9, 7] = x[0, 9, 7].abs(), -x[0, 9, 7].abs()
    g = torch.randn((1, 70, T), generator=gen).to(t)
    g[0, 5, 0], g[0, 9, 1], g[0, 5, 2], g[0, 9, 2] = inf, -inf, inf, -inf
    if T > 3:
        g[0, 69, 3], g[0, 5, 4], g[0, 33, 4] = torch.finfo(t).max / 4, inf, float("nan")
    packed = mgd.mg_mx_pack(x.cuda(), fmt)
    xv = mgd.mg_mx_unpack(packed).double().cpu()[0]
    want = (g[0].double().t()[:, None, :] * xv.t()[None]).sum(2)
    dw, db = (v.double().cpu() for v in mgd.mg_mx8_weight_gradient(g.cuda(), packed))
    odd = ~want.isfinite()
    assert odd[:3].all() and want[0].isinf().any() and want[2].isnan().any()
    assert same(dw[odd], want[odd])
    bound = 3 * 70 * 2.0 ** -24 * (g[0].double().t().abs() @ xv.abs())     # three pieces, three sums
    assert ((dw - want).abs()[~odd] <= bound[~odd]).all()
    assert same(db[:3], torch.tensor([inf, -inf, float("nan")]))


def test_gradient_bits_that_only_the_low_half_of_a_float_holds():
    """A NaN of low payload bits alone stays one."""
    g = torch.ones((1, 40, 3))
    g.view(torch.int32)[0, 3, 1] = 0x7f800001
    dw, db = mgd.mg_mx8_weight_gradient(g.cuda(), mgd.mg_mx_pack(torch.ones((1, 40, 33), device="cuda")))
    assert dw[1].isnan().all() and db[1].isnan() and (dw[[0, 2]] == 40).all() and (db[[0, 2]] == 40).all()


@pytest.mark.parametrize("N", [1, 31, 100, 1000])
def test_counts_at_the_ends_of_their_type(N):
    """Counts below 0 are 0 and counts above N are N, also where steps of rows start inside an example."""
    low, high = -1 << 31, (1 << 31) - 1
    x = mgd.mg_mx_pack(torch.randn((5, N, 70), device="cuda", generator=torch.Generator("cuda").manual_seed(N)))
    g = torch.randn((5, N, 6), device="cuda", generator=torch.Generator("cuda").manual_seed(N + 1))
    count = lambda *n: torch.tensor(n, dtype=torch.int32, device="cuda")
    got = mgd.mg_mx8_weight_gradient(g, x, natoms=count(low, high, low + 5, N // 2, high - 1))
    want = mgd.mg_mx8_weight_gradient(g, x, natoms=count(0, N, 0, N // 2, N))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for out in mgd.mg_mx8_weight_gradient(g, x, natoms=count(*[low] * 5)):
        assert not out.any()


def test_calls_without_the_binding(monkeypatch):
    """Where the C++ side is missing the same kernels give the same bits."""
    x = torch.randn((3, 50, 70), device="cuda")
    w = torch.randn((30, 70), device="cuda")
    g = torch.randn((3, 50, 6), device="cuda")

    def work():
        packed, four = mgd.mg_mx_pack(x), mgd.mg_mx_pack(w, "e2m1")
        return (packed.codes, packed.scales, mgd.mg_mx_unpack(packed), *mgd.mg_mx8_weight_gradient(g, packed),
                mgd.mg_mx4_linear(x, four), mgd.mg_mx4_product(mgd.mg_mx_pack(x, "e2m1"), four))

    want = work()
    assert mgd._binding is not None
    monkeypatch.setattr(mgd, "_binding", None)
    for a, b in zip(work(), want):
        assert torch.equal(a, b)


def test_as_many_rows_as_the_scales_allow():
    """2^31 - 4 bytes of scales: floats of one column, whose lanes past the last row are counted past 2^32."""
    rows = (1 << 29) - 1
    x = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(251).sub_(120).float().view(rows, 1)
    got = mgd.mg_mx_pack(x, "int8")
    for k in (0, 12345678, rows - 4096):
        want = mgd.mg_mx_pack(x[k:k + 4096].clone(), "int8")
        assert torch.equal(got.codes[k:k + 4096], want.codes) and torch.equal(got.scales[k:k + 4096], want.scales)
    del x
    back = mgd.mg_mx_unpack(got)
    bad = 0
    for k in range(0, rows, 1 << 26):       # up to 127 numbers come back as they were; from 128 on in steps of
        want = torch.arange(k, min(rows, k + (1 << 26)), dtype=torch.int32, device="cuda").remainder_(251).sub_(120)
        want[want == 129] = 128             # two, 129 lies halfway and goes to 128 (64 is even)
        bad += int((back[k:k + (1 << 26), 0] != want.float()).sum())
    assert bad == 0


@pytest.mark.parametrize("exponent", [-100, -110, -118, -124, -130, -140])
def test_gradients_near_the_end_of_the_range(exponent):
    """Float gradients with 24 significant bits: what lies above 2^-133 counts, also below the normal range."""
    gen = torch.Generator().manual_seed(7)
    g = (torch.randn((1, 64, 20), generator=gen, dtype=torch.float64) * 2.0 ** exponent).float()
    x = torch.randint(-127, 128, (1, 64, 40), generator=gen).float() * 2.0 ** 60
    packed = mgd.mg_mx_pack(x.cuda())
    xv = mgd.mg_mx_unpack(packed).double().cpu()[0]
    gv = g.double()[0]
    dw, db = (v.double().cpu() for v in mgd.mg_mx8_weight_gradient(g.cuda(), packed))
    # three sums of 64 exact products, and less than 2^-133 of every gradient
    bound = 3 * 64 * 2.0 ** -24 * (gv.abs().t() @ xv.abs()) + 2.0 ** -133 * xv.abs().sum(0)
    assert ((dw - gv.t() @ xv).abs() <= bound).all()
    assert ((db - gv.sum(0)).abs() <= 64 * 2.0 ** -24 * gv.abs().sum(0) + 2.0 ** -149).all()


def test_codes_near_the_end_of_the_range():
    """e4m3 blocks of the lowest scales: every code above 2^-133 counts."""
    codes = torch.arange(256, dtype=torch.uint8).view(8, 32)[[0, 1, 2, 4, 5, 6]].contiguous()
    for scale in (0, 1, 2, 9):
        scales = torch.full((6, 4), scale, dtype=torch.uint8)
        packed = mgd.MXTensor(codes.cuda(), scales.cuda(), (6, 32), "e4m3")
        xv = codes.view(torch.float8_e4m3fn).double() * 2.0 ** (scale - 127)
        dw, _ = mgd.mg_mx8_weight_gradient(torch.full((6, 2), 2.0 ** 60, device="cuda"), packed)
        want = xv.sum(0) * 2.0 ** 60
        bound = 6 * 2.0 ** -24 * xv.abs().sum(0) * 2.0 ** 60 + 6 * 2.0 ** (60 - 133)
        assert ((dw.double().cpu() - want).abs() <= bound).all()


def test_views_that_negate():
    for rows in (1, 4):
        x = torch.full((1, rows, 1), 1.0 + 2.0j, device="cuda").conj().imag
        w = mgd.mg_mx_pack(torch.ones((3, 1), device="cuda"), "e2m1")
        packed = mgd.mg_mx_pack(torch.ones((1, rows, 5), device="cuda"))
        for call in (lambda: mgd.mg_mx_pack(x), lambda: mgd.mg_mx4_linear(x, w),
                     lambda: mgd.mg_mx8_weight_gradient(x, packed), lambda: mgd.mg_mx_unpack(mgd.mg_mx_pack(x.clone()), out=x)):
            with pytest.raises(ValueError, match="resolve_neg"):
                call()
        assert (mgd.mg_mx4_linear(x.resolve_neg(), w) == -2).all()
        typer = AtomTyper(1, 3).cuda()
        assert torch.equal(typer.in_4_bits()(x), typer.in_4_bits()(x.resolve_neg()))
        typer(x).sum().backward()
        assert (typer.weight.grad == -2 * rows).all()
    x = torch.full((1,), 1.0 + 2.0j, device="cuda", requires_grad=True)
    with saved_in_8_bits(min_elements=1):
        y = x.conj().imag.square()
    y.backward()
    assert x.grad == 4.0j                               # d (imag x)^2


@pytest.mark.parametrize("K", [6100, 6220, 6400, 6505])
def test_product_where_large_tiles_win_by_a_tenth(K):
    """4090 x 4070 in tiles of 256 x 256, well past the k from which they are the faster ones; ends of k in each of
    four steps, edges of C both ways.  Against the product in double of what the codes stand for."""
    torch.manual_seed(K)
    M, N = 4090, 4070
    a, b = (mgd.mg_mx_pack(torch.randn((rows, K), device="cuda"), "e2m1") for rows in (M, N))
    bias = torch.randn(N, device="cuda")
    x, y = mgd.mg_mx_unpack(a).double(), mgd.mg_mx_unpack(b).double().t().contiguous()
    want, bound = x @ y, K * 2.0 ** -24 * (x.abs() @ y.abs())
    for use in (None, bias):
        if use is not None:
            want, bound = want + bias, bound + 2.0 ** -23 * (want.abs() + bias.abs())
        for dtype in DTYPES.values():
            half = torch.finfo(dtype).eps / 2
            tiny = float(torch.finfo(dtype).smallest_normal) * half if dtype == torch.float16 else 0.0
            got = mgd.mg_mx4_product(a, b, bias=use, dtype=dtype).double()
            assert ((got - want).abs() <= bound + half * (want.abs() + bound) + tiny).all(), dtype


def test_every_block_of_a_row_longer_than_the_offsets_of_32_bits():
    """2.1e9 half numbers whose blocks differ in size: each is off by at most half a step of its own block (at most
    2^-7 of 256/255 of its largest: a largest number from 255/128 of a power of two on takes the next one), and by
    half a step of its type."""
    n = (1 << 31) + 12345
    x = torch.empty((1, n), dtype=torch.float16, device="cuda").normal_()
    for part in x[0, :n // 32 * 32].view(-1, 32).split(1 << 20):
        part *= torch.randint(0, 6, (part.shape[0], 1), device="cuda").float().mul_(2).exp2_().div_(256.0)
    back = mgd.mg_mx_unpack(mgd.mg_mx_pack(x, "int8"))
    bad = 0
    for a, b in zip(x[0, :n // 32 * 32].view(-1, 32).split(1 << 22), back[0, :n // 32 * 32].view(-1, 32).split(1 << 22)):
        a, b = a.float(), b.float()
        off = a.abs().amax(1, keepdim=True) * (2.0 ** -7 * 256 / 255) + b.abs() * 2.0 ** -11 + 2.0 ** -25
        bad += int(((a - b).abs() > off).sum())
    assert bad == 0


def test_calls_on_tensors_record_no_history():
    x = torch.randn((4, 40), device="cuda", requires_grad=True)
    packed, w = mgd.mg_mx_pack(x), mgd.mg_mx_pack(x, "e2m1")
    for y in (packed.codes, mgd.mg_mx_unpack(packed), mgd.mg_mx4_linear(x, w), *mgd.mg_mx8_weight_gradient(x, packed)):
        assert not y.requires_grad


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [7, 28, 100])
def test_infinite_gradients_among_many_rows(dtype, T):
    """Over many workgroups: channels without one keep the bits they have without any, rows past the counts none."""
    t, inf = DTYPES[dtype], float("inf")
    gen = torch.Generator("cuda").manual_seed(T)
    B, N, E = 6, 2040, 256
    x = torch.randn((B, N, E), device="cuda", generator=gen).abs() + 0.5
    g = torch.randn((B, N, T), device="cuda", generator=gen).to(t)
    natoms = torch.tensor([2040, 1000, 0, 33, 2040, 7], dtype=torch.int32, device="cuda")
    packed = mgd.mg_mx_pack(x)
    clean = mgd.mg_mx8_weight_gradient(g, packed, natoms=natoms)
    g[1, 1000:], g[2], g[5, 7] = inf, float("nan"), -inf            # of no atom
    for a, b in zip(mgd.mg_mx8_weight_gradient(g, packed, natoms=natoms), clean):
        assert torch.equal(a, b)
    g[0, 2039, 3], g[4, 5, 3], g[1, 999, 5], g[4, 0, 6], g[3, 32, 6] = inf, inf, -inf, inf, -inf
    dw, db = mgd.mg_mx8_weight_gradient(g, packed, natoms=natoms)
    assert (dw[3] == inf).all() and (dw[5] == -inf).all() and dw[6].isnan().all()
    assert db[3] == inf and db[5] == -inf and db[6].isnan()
    rest = [k for k in range(T) if k not in (3, 5, 6)]
    assert torch.equal(dw[rest], clean[0][rest]) and torch.equal(db[rest], clean[1][rest])
