"""Learned types and tensors saved in 8 bits, the parts that run without a device."""
import pytest

torch = pytest.importorskip("torch")

from paper_1912_04822_amd.autograd import AtomTyper, GridLayer, _LiveMap, _is_parameter  # noqa: E402


@pytest.mark.parametrize("bias", [False, True])
def test_plain_typer_leaves_out_what_lies_past_the_counts(bias):
    """With ``keep=None``: the live rows' gradients, also where the others' features and gradients are NaN, and the
    same forward values with gradients and without."""
    torch.manual_seed(1)
    B, N, E, T = 4, 6, 5, 3
    typer = AtomTyper(E, T, bias=bias, keep=None)
    natoms = torch.tensor([6, 2, 0, 1], dtype=torch.int32)
    live = torch.arange(N)[None] < natoms[:, None]
    x, G = torch.randn((B, N, E)), torch.randn((B, N, T))
    for dead in (1.0, float("nan")):
        x[~live], G[~live] = dead, dead
        leaf = x.clone().requires_grad_()
        typer.zero_grad()
        y = typer(leaf, natoms)
        y.backward(G)
        with torch.no_grad():
            assert torch.equal(torch.nan_to_num(y, 7.0), torch.nan_to_num(typer(x, natoms), 7.0))
        g, xs = G[live].double(), x[live].double()
        eps = 2.0 ** -24 * live.sum()
        assert ((typer.weight.grad - g.t() @ xs).abs() <= eps * (g.abs().t() @ xs.abs())).all()
        if bias:
            assert ((typer.bias.grad - g.sum(0)).abs() <= eps * g.abs().sum(0)).all()
        w = typer.weight.detach().double()
        assert (leaf.grad[~live] == 0).all()
        assert ((leaf.grad[live] - g @ w).abs() <= T * 2.0 ** -24 * (g.abs() @ w.abs())).all()


def test_plain_typer_is_differentiated_like_any_map():
    """Gradients and their gradients against differences, forward mode, and over a batch of parameters."""
    torch.manual_seed(2)
    x, w, b = (torch.randn(s, dtype=torch.float64, requires_grad=True) for s in ((3, 4, 5), (2, 5), (2,)))
    natoms = torch.tensor([4, 0, 2], dtype=torch.int32)
    live = (torch.arange(4)[None] < natoms[:, None])[:, :, None]
    only_live = lambda x, w, b: torch.where(live, _LiveMap.apply(x, w, b, natoms), 0.0)     # rows past it have no gradient
    assert torch.autograd.gradcheck(only_live, (x, w, b), check_forward_ad=True)
    assert torch.autograd.gradgradcheck(only_live, (x, w, b))
    assert torch.autograd.gradcheck(lambda x, w: torch.where(live, _LiveMap.apply(x, w, None, natoms), 0.0), (x, w))
    ws = torch.randn((6, 2, 5), dtype=torch.float64)
    got = torch.func.vmap(lambda v: torch.func.grad(lambda u: _LiveMap.apply(x.detach(), u, b.detach(), natoms).sum())(v))(ws)
    assert torch.allclose(got, torch.where(live, x.detach(), 0.0).sum((0, 1)).expand(6, 2, 5))


def test_plain_typer_under_autocast():
    torch.manual_seed(3)
    typer = AtomTyper(8, 4, keep=None)
    x = torch.randn((2, 5, 8), requires_grad=True)
    natoms = torch.tensor([5, 2], dtype=torch.int32)
    with torch.autocast("cpu", dtype=torch.bfloat16):
        y = typer(x, natoms)
    assert y.dtype == torch.float32
    y.sum().backward()
    assert x.grad.dtype == typer.weight.grad.dtype == typer.bias.grad.dtype == torch.float32
    assert (typer.bias.grad == 7).all() and (x.grad[1, 2:] == 0).all()


def taken_for_parameters(run):
    """What autograd saves while ``run`` runs: (shape, whether it counts as a parameter or a view of one)."""
    seen = []

    def look(x):
        seen.append((tuple(x.shape), _is_parameter(x) or (x._base is not None and _is_parameter(x._base))))
        return x

    with torch.autograd.graph.saved_tensors_hooks(look, lambda x: x):
        run()
    return seen


@pytest.mark.parametrize("frozen", [False, True])
def test_weights_are_told_from_activations(frozen):
    x = torch.randn((7, 9), requires_grad=True) * 1.0
    linear = torch.nn.Linear(9, 5).requires_grad_(not frozen)
    seen = dict(taken_for_parameters(lambda: linear(x)))
    assert seen[(9, 5) if (9, 5) in seen else (5, 9)] and not seen.get((7, 9), False)
    x = torch.randn((2, 3, 6, 6), requires_grad=True) * 1.0
    seen = dict(taken_for_parameters(lambda: torch.nn.Conv2d(3, 4, 3).requires_grad_(not frozen)(x)))
    assert seen[(4, 3, 3, 3)] and not seen[(2, 3, 6, 6)]


def test_copies_of_weights_are_told_from_activations():
    x = torch.randn((7, 9), requires_grad=True) * 1.0
    image = torch.randn((2, 3, 6, 6), requires_grad=True) * 1.0
    linear, conv = torch.nn.Linear(9, 5), torch.nn.Conv2d(3, 4, 3)
    with torch.autocast("cpu", dtype=torch.bfloat16):
        seen = dict(taken_for_parameters(lambda: linear(x)))
        assert seen[(9, 5) if (9, 5) in seen else (5, 9)] and not seen.get((7, 9), False)
        seen = dict(taken_for_parameters(lambda: conv(image)))
        assert seen[(4, 3, 3, 3)] and not seen[(2, 3, 6, 6)]
    twice = (x * x).to(torch.bfloat16)                  # copies of activations are activations
    seen = dict(taken_for_parameters(lambda: twice * twice))
    assert not seen[(7, 9)]


@pytest.mark.parametrize("E,T", [(1, 65536), ((1 << 20) + 1, 1)])
def test_sizes_the_backward_pass_has_no_gradient_for_are_refused_at_the_call(E, T):
    typer = AtomTyper(E, T)
    with pytest.raises(ValueError, match="keep=None"):
        typer(torch.zeros((1, 2, E)))
    assert AtomTyper(E, T, keep=None)(torch.zeros((1, 2, E))).shape == (1, 2, T)
    with torch.no_grad():
        assert typer(torch.zeros((1, 2, E))).shape == (1, 2, T)


@pytest.mark.parametrize("shape", [(2, 4, 3), (2, 6, 3), (1, 5, 3), (3, 5, 3), (2, 5)])
@pytest.mark.parametrize("learned", [False, True])
def test_weights_of_other_atoms_than_the_coordinates_are_refused(shape, learned):
    """Before anything reaches the device: with gradients, tables are built for the coordinates' atoms."""
    coords, radii = torch.zeros((2, 5, 3), requires_grad=True), torch.ones(3)
    layer = GridLayer(typer=AtomTyper(8, 3, keep=None))
    if learned and len(shape) == 3:
        given = dict(features=torch.zeros(shape[:2] + (8,)))
    else:
        given = dict(weights=torch.zeros(shape))
    with pytest.raises(ValueError, match="weights must have shape"):
        layer(coords, radii, **given)
