"""Refusals of the layers on microscaled formats, and what they do without a device (host only)."""
import pytest

torch = pytest.importorskip("torch")

from paper_1912_04822_amd.autograd import AtomTyper, GridLayer, saved_in_8_bits  # noqa: E402


def test_refusals():
    for bad in ("e2m1", "int4", 8):
        with pytest.raises(ValueError):
            AtomTyper(8, 4, keep=bad)
        with pytest.raises(ValueError):
            saved_in_8_bits(bad)
    with pytest.raises(ValueError):
        AtomTyper(0, 4)
    with pytest.raises(ValueError):
        saved_in_8_bits(min_elements=0)
    typer = AtomTyper(8, 4)
    with pytest.raises(ValueError):
        typer(torch.zeros((2, 3, 7)))
    with pytest.raises(ValueError):
        typer(torch.zeros((3, 8)))
    with pytest.raises(ValueError):
        typer(torch.zeros((2, 3, 8)))               # 8 bits are kept on the device
    with pytest.raises(ValueError):
        typer.in_4_bits()
    coords, radii = torch.zeros((1, 2, 3)), torch.ones(4)
    with pytest.raises(ValueError):
        GridLayer()(coords, radii, features=torch.zeros((1, 2, 8)))
    with pytest.raises(ValueError):
        GridLayer(typer=typer)(coords, radii, features=torch.zeros((1, 2, 8)), weights=torch.zeros((1, 2, 4)))
    with pytest.raises(ValueError):
        GridLayer(typer=typer)(coords, radii)


def test_parameters_reach_the_layer():
    layer = GridLayer(typer=AtomTyper(8, 4))
    assert [n for n, _ in layer.named_parameters()] == ["typer.weight", "typer.bias"]
    assert list(GridLayer().parameters()) == []
    assert AtomTyper(8, 4, bias=False).bias is None


def test_plain_typer_is_a_linear_map():
    torch.manual_seed(0)
    typer = AtomTyper(8, 4, keep=None)
    x = torch.randn((2, 5, 8), requires_grad=True)
    n = torch.tensor([5, 2], dtype=torch.int32)
    y = typer(x, n)
    y.sum().backward()
    assert torch.allclose(y[0], x[0] @ typer.weight.t() + typer.bias, atol=1e-6)
    assert torch.allclose(typer.weight.grad, (x[0].sum(0) + x[1, :2].sum(0)).expand(4, 8).detach(), atol=1e-5)
    assert (x.grad[1, 2:] == 0).all()


def test_host_tensors_are_saved_as_they_are():
    x = torch.randn((300, 300), requires_grad=True)
    with saved_in_8_bits(min_elements=1):
        y = (x * x).sum()
    y.backward()
    assert torch.equal(x.grad, 2 * x.detach())


def test_natoms_are_checked():
    for keep in (None, "int8"):
        typer = AtomTyper(8, 4, keep=keep)
        for bad in (torch.tensor([1, 2]), torch.ones(3, dtype=torch.int32), torch.ones((2, 1), dtype=torch.int32)):
            with pytest.raises(ValueError):
                typer(torch.zeros((2, 3, 8)), bad)


def test_rows_of_a_tensor():
    from paper_1912_04822_amd.molgrid import row_stride
    x = torch.zeros((4, 6, 10))
    assert row_stride(x) == 10 and row_stride(x[:, :, 2:5]) == 10 and row_stride(x[:, :, :1]) == 10
    assert row_stride(x[:, 1:3]) is None and row_stride(x[1:2, 1:3]) == 10 and row_stride(x[:, 1]) == 60
    assert row_stride(x.transpose(0, 1)) is None and row_stride(x[:, :, ::2]) is None
    assert row_stride(x[:1, :1].expand(4, 6, 10)) is None and row_stride(x[:1].expand(4, 6, 10)) is None
    assert row_stride(torch.zeros(7)) == 7 and row_stride(torch.zeros((5, 1))) == 1
    assert row_stride(torch.zeros(20).as_strided((3, 8), (4, 1))) is None
