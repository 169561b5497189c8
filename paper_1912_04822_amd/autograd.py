"""``torch.autograd`` glue over the C-ABI binding (GridMaker section: the grid is generated
in place on a Torch tensor, and ``backward`` turns a gradient on the grid into atomic gradients,
so coordinates -- and, with vector types, type weights -- can be optimised through the grid).

No arithmetic of the method happens here: ``forward`` calls ``mg_forward_*`` and ``backward``
calls ``mg_backward_*``; this module only tells autograd which call belongs to which.  When a
gradient will be asked for, forward builds the tables once (``mg_prepare``) in a workspace of its
own and both passes run on them (the ``*_prepared`` calls): the backward pass then starts without
a prep kernel.
A binary GridMaker has no gradient (the indicator is piecewise constant); asking for one raises.

Two things beside it, on the microscaled formats of the binding (blocks of 32 numbers that share a
power of two): ``AtomTyper`` learns types from atom features -- the weights a vector-typed grid takes
are a linear map of them -- and keeps its input in 8 bits for the weight gradient, or runs in 4 bits
where no gradient is wanted; ``saved_in_8_bits`` keeps what a whole network saves for its backward
pass in 8 bits.
"""
from __future__ import annotations

import threading
from typing import Optional

import torch

from . import molgrid

_exact = threading.local()          # set while a layer of this module saves what has to stay exact


class _IndexGrid(torch.autograd.Function):
    @staticmethod
    def forward(ctx, coords, gm, types, radii, T, natoms, centers, quats, translations):
        ctx.gm, ctx.T, ctx.ws = gm, T, None
        ctx.save_for_backward(coords, types, radii, natoms, centers, quats, translations)
        if ctx.needs_input_grad[0] and not gm.binary:
            B, N, _ = coords.shape
            ctx.ws = gm.mg_prepare(coords.detach(), types, radii, T, natoms=natoms, centers=centers,
                                   quats=quats, translations=translations)
            return gm.mg_forward_index_prepared(B, N, T, ctx.ws)
        return gm.mg_forward_index(coords.detach(), types, radii, T, natoms=natoms, centers=centers,
                                   quats=quats, translations=translations)

    @staticmethod
    def backward(ctx, grad_out):
        if ctx.gm.binary:
            raise RuntimeError("a binary GridMaker has no gradient")
        coords, types, radii, natoms, centers, quats, translations = ctx.saved_tensors
        if ctx.ws is not None and grad_out.dtype == torch.float32:
            B, N, _ = coords.shape
            g = ctx.gm.mg_backward_index_prepared(B, N, ctx.T, grad_out.contiguous(), ctx.ws)
            return (g,) + (None,) * 8
        g = ctx.gm.mg_backward_index(coords.detach(), types, radii, ctx.T, grad_out.contiguous(),
                                     natoms=natoms, centers=centers, quats=quats,
                                     translations=translations)
        return (g,) + (None,) * 8


class _VectorGrid(torch.autograd.Function):
    @staticmethod
    def forward(ctx, coords, weights, gm, radii, natoms, centers, quats, translations):
        if weights.dim() != 3 or weights.shape[:2] != coords.shape[:2]:     # tables of other atoms than the weights'
            raise ValueError("weights must have shape [%d,%d,T], got %s" % (*coords.shape[:2], tuple(weights.shape)))
        ctx.gm, ctx.ws = gm, None
        ctx.save_for_backward(coords, weights, radii, natoms, centers, quats, translations)
        if (ctx.needs_input_grad[0] or ctx.needs_input_grad[1]) and not gm.binary:
            ctx.ws = gm.mg_prepare(coords.detach(), None, radii, weights.shape[2], natoms=natoms,
                                   centers=centers, quats=quats, translations=translations)
            return gm.mg_forward_vector_prepared(weights.detach(), radii, ctx.ws)
        return gm.mg_forward_vector(coords.detach(), weights.detach(), radii, natoms=natoms,
                                    centers=centers, quats=quats, translations=translations)

    @staticmethod
    def backward(ctx, grad_out):
        if ctx.gm.binary:
            raise RuntimeError("a binary GridMaker has no gradient")
        coords, weights, radii, natoms, centers, quats, translations = ctx.saved_tensors
        want_c, want_w = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        if ctx.ws is not None and grad_out.dtype == torch.float32:
            gc, gw = ctx.gm.mg_backward_vector_prepared(
                weights.detach(), radii, grad_out.contiguous(), ctx.ws, want_coords=True,
                want_weights=bool(want_w))
            return (gc if want_c else None, gw if want_w else None) + (None,) * 6
        gc, gw = ctx.gm.mg_backward_vector(
            coords.detach(), weights.detach(), radii, grad_out.contiguous(), natoms=natoms,
            centers=centers, quats=quats, translations=translations,
            want_coords=True, want_weights=bool(want_w))
        return (gc if want_c else None, gw if want_w else None) + (None,) * 6


class _Exact:
    """What is saved inside stays as it is, also within ``saved_in_8_bits``."""

    def __enter__(self):
        self.before = getattr(_exact, "on", False)
        _exact.on = True

    def __exit__(self, *_):
        _exact.on = self.before


class saved_in_8_bits(torch.autograd.graph.saved_tensors_hooks):
    """Within ``with saved_in_8_bits():`` what autograd saves for the backward pass is kept in 8 bits
    (blocks of 32 neighbouring numbers in memory that share a power of two) and restored when it is
    needed.  Every save takes 33/32 bytes a number.  What several operations save (a ReLU's result is
    the next convolution's input) is kept once for each of them, where torch holds it once: four
    convolutions followed by ReLU take 0.41 of their float32 memory and 0.83 of bfloat16's, by softplus,
    where nothing is saved twice, 0.26 and 0.52.  For the network behind a grid, whose activations are
    as large as the grid:

        with saved_in_8_bits():
            loss = net(layer(coords, radii, types=types, T=T))
        loss.backward()

    Kept so: float32, float16 and bfloat16 device tensors of at least ``min_elements`` numbers that
    lie without gaps in memory, but for parameters (frozen ones too), other leaves that require a
    gradient, and views of either, which exist anyway, and the copies autocast makes of them in
    another type.  (Its copies of frozen weights cannot be told from data: have a frozen layer in the
    type it runs in.)  Everything else, nested tensors and subclasses of tensors among it, and what
    this module's own layers save, stays exact.

    ``format`` "int8" is off by at most 2^-7 of the block's largest number (256/255 of that where the
    largest is just below a power of two), "e4m3" by at most 2^-4 of each (or 1.2 times 2^-18 of the
    largest, where that is more).  Gradients change accordingly; small positive numbers of a block may
    become zero (and with them the gradient of a ReLU there), and a block that holds an infinity or a
    NaN becomes NaN."""

    def __init__(self, format="int8", min_elements=1 << 16):
        if format not in ("int8", "e4m3"):
            raise ValueError("format must be int8 or e4m3, got %r" % (format,))
        if min_elements < 1:
            raise ValueError("min_elements must be at least 1")
        self.format, self.min_elements = format, int(min_elements)
        super().__init__(self._pack, self._unpack)

    def _pack(self, x):
        if (getattr(_exact, "on", False) or type(x) is not torch.Tensor or x.is_nested or not x.is_cuda
                or x.dtype not in molgrid.NUMBERS
                or x.numel() < self.min_elements or x.layout is not torch.strided or x.is_neg()
                or _is_parameter(x) or (x._base is not None and _is_parameter(x._base))):
            return x
        flat = _in_memory_order(x.detach())
        if flat is None:
            return x
        return molgrid.mg_mx_pack(flat, self.format), x.shape, x.stride()

    @staticmethod
    def _unpack(kept):
        if isinstance(kept, torch.Tensor):
            return kept
        packed, shape, stride = kept
        flat = molgrid.mg_mx_unpack(packed)
        return flat.as_strided(shape, stride)


def _is_parameter(x):
    if isinstance(x, torch.nn.Parameter) or (x.is_leaf and x.requires_grad):
        return True
    if x.grad_fn is None or x.grad_fn.name() != "ToCopyBackward0":
        return False
    return hasattr(x.grad_fn.next_functions[0][0], "variable")     # a copy of a leaf in another type


def _in_memory_order(x):
    """``x`` as one row [1, numel], or None where its memory has gaps or is used twice."""
    if not x.is_contiguous():
        x = x.permute(sorted(range(x.dim()), key=lambda d: (-x.stride(d), -x.shape[d])))
        if not x.is_contiguous():
            return None
    return x.view(1, -1)


class _TypeWeights(torch.autograd.Function):
    @staticmethod
    def forward(ctx, features, weight, bias, natoms, keep):
        y = torch.nn.functional.linear(features, weight, bias)
        packed = molgrid.mg_mx_pack(_even_rows(features), keep) if ctx.needs_input_grad[1] else None
        ctx.keep = keep
        ctx.shape, ctx.dtypes = features.shape, (features.dtype, weight.dtype, None if bias is None else bias.dtype)
        ctx.save_for_backward(weight, natoms, *((packed.codes, packed.scales) if packed is not None else (None, None)))
        return y.float()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        weight, natoms, codes, scales = ctx.saved_tensors
        gx = gw = gb = None
        grad = grad.contiguous()
        if ctx.needs_input_grad[0]:
            if natoms is not None:
                grad = _live_rows(grad, natoms)
            gx = torch.matmul(grad.view(-1, grad.shape[2]), weight.float()).view(ctx.shape).to(ctx.dtypes[0])
        if ctx.needs_input_grad[1]:
            packed = molgrid.MXTensor(codes, scales, ctx.shape, ctx.keep)
            gw, gb = molgrid.mg_mx8_weight_gradient(grad, packed, natoms=natoms)
            gw = gw.to(ctx.dtypes[1])
        if ctx.dtypes[2] is None or not ctx.needs_input_grad[2]:
            gb = None
        else:
            if gb is None:                          # a bias alone
                gb = _sum_of_rows(grad, natoms)
            gb = gb.to(ctx.dtypes[2])
        return gx, gw, gb, None, None


class _LiveMap(torch.autograd.Function):
    """A linear map of [B,N,E] whose gradients leave out the rows past ``natoms``, whatever features and gradients
    hold there, from torch's operations alone."""

    generate_vmap_rule = True

    @staticmethod
    def forward(features, weight, bias, natoms):
        return torch.nn.functional.linear(features, weight, bias)

    @staticmethod
    def setup_context(ctx, inputs, output):
        ctx.save_for_backward(*inputs)
        ctx.save_for_forward(*inputs)

    @staticmethod
    def backward(ctx, grad):
        features, weight, bias, natoms = ctx.saved_tensors
        gx = gw = gb = None
        grad = _live_rows(grad, natoms)
        flat = grad.flatten(0, 1)
        if ctx.needs_input_grad[0]:
            gx = torch.matmul(grad, weight.to(grad.dtype)).to(features.dtype)
        if ctx.needs_input_grad[1]:
            live = _live_rows(features, natoms).flatten(0, 1)
            gw = torch.matmul(flat.t(), live.to(grad.dtype)).to(weight.dtype)
        if bias is not None and ctx.needs_input_grad[2]:
            gb = flat.sum(0).to(bias.dtype)
        return gx, gw, gb, None

    @staticmethod
    def jvp(ctx, features_t, weight_t, bias_t, _):
        features, weight, bias, natoms = ctx.saved_tensors
        y = torch.zeros((), dtype=features.dtype, device=features.device)
        if features_t is not None:
            y = y + torch.nn.functional.linear(_live_rows(features_t, natoms), weight)
        if weight_t is not None:
            y = y + torch.nn.functional.linear(_live_rows(features, natoms), weight_t)
        if bias_t is not None:
            y = y + bias_t
        return _live_rows(y.expand(*features.shape[:2], weight.shape[0]), natoms)


def _even_rows(x):
    """``x``, or a copy where its rows are not equally far apart (expanded, transposed)."""
    x = x.resolve_neg()
    return x if molgrid.row_stride(x) is not None else x.contiguous()


def _check_natoms(natoms, features):
    if natoms is not None and (natoms.dtype is not torch.int32 or tuple(natoms.shape) != (features.shape[0],)):
        raise ValueError("natoms must be int32 of shape (%d,), got %s of %s"
                         % (features.shape[0], natoms.dtype, tuple(natoms.shape)))
    if natoms is not None and natoms.device != features.device and torch.is_grad_enabled():
        raise ValueError("natoms is on %s, features are on %s" % (natoms.device, features.device))


def _live_rows(x, natoms):
    """``x`` [B,N,...] with zeros past every example's ``natoms``."""
    live = torch.arange(x.shape[1], device=x.device)[None, :] < natoms[:, None]
    return torch.where(live[:, :, None], x, torch.zeros((), dtype=x.dtype, device=x.device))


def _sum_of_rows(grad, natoms):
    """Sum of the live rows of ``grad`` [B,N,T]: the bias that goes with weights of one feature, whose codes are
    zeros.  (torch's sum over many rows gives wrong numbers when a graph it was captured in is replayed.)"""
    B, N, _ = grad.shape
    codes, scales = (torch.zeros((B * N, k), dtype=torch.uint8, device=grad.device) for k in (32, 4))
    return molgrid.mg_mx8_weight_gradient(grad, molgrid.MXTensor(codes, scales, (B, N, 1), "int8"), natoms=natoms)[1]


class AtomTyper(torch.nn.Module):
    """Learned vector types: ``typer(features)`` maps per-atom features [B,N,E] (float32, float16 or
    bfloat16) linearly to type weights [B,N,T] in float32, which a vector-typed grid takes
    (``GridLayer(..., typer=AtomTyper(E, T))`` and ``layer(coords, radii, features=features)``).

    What the weight gradient needs of the features is kept in 8 bits (``keep`` "int8" or "e4m3") and
    the gradient formed from the codes, once: no second derivatives, forward mode or ``vmap``.  The map
    itself and the features' gradient are torch's products; ``keep=None`` leaves all of it to torch.
    With ``natoms`` [B] (int32) atoms past an example's count have no part in any gradient, whatever
    their rows hold.

    A training step can be captured in a graph; as for every leaf in torch, no graph of the same
    parameters that was recorded outside may be alive at the capture (drop losses and outputs first).
    With ``keep=None`` the bias's gradient is torch's sum, which over many atoms is wrong when replayed."""

    def __init__(self, features, channels, bias=True, keep="int8", device=None, dtype=None):
        super().__init__()
        if keep not in (None, "int8", "e4m3"):
            raise ValueError("keep must be int8, e4m3 or None, got %r" % (keep,))
        if features < 1 or channels < 1:
            raise ValueError("features and channels must be at least 1")
        self.keep = keep
        self.weight = torch.nn.Parameter(torch.empty((channels, features), device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.empty((channels,), device=device, dtype=dtype)) if bias else None
        bound = features ** -0.5
        torch.nn.init.uniform_(self.weight, -bound, bound)
        if bias:
            torch.nn.init.uniform_(self.bias, -bound, bound)

    def forward(self, features, natoms=None):
        if features.dim() != 3 or features.shape[2] != self.weight.shape[1]:
            raise ValueError("features must have shape [B,N,%d], got %s"
                             % (self.weight.shape[1], tuple(features.shape)))
        _check_natoms(natoms, features)
        with _Exact():
            if not torch.is_grad_enabled() or (self.keep is None and natoms is None) or features.numel() == 0:
                return torch.nn.functional.linear(features, self.weight, self.bias).float()
            if self.keep is None:
                return _LiveMap.apply(features, self.weight, self.bias, natoms).float()
            T, E = self.weight.shape
            if (T > 65535 or E > 1 << 20) and any(p.requires_grad for p in self.parameters()):
                raise ValueError("the gradient from 8 bits takes up to 2^20 features and 65535 channels, got %d and %d:"
                                 " use keep=None" % (E, T))
            natoms = None if natoms is None else natoms.contiguous()
            return _TypeWeights.apply(features, self.weight, self.bias, natoms, self.keep)

    def in_4_bits(self):
        """A copy for use without gradients (screening), its weights laid out in 4 bits once."""
        return AtomTyper4(self.weight, self.bias)


class AtomTyper4(torch.nn.Module):
    """``AtomTyper`` where no gradient is wanted: features and weights enter the product in 4 bits
    (e2m1, a power of two for every 32 features), sums are float.  Made by ``AtomTyper.in_4_bits``
    from the weights of that moment; ``state_dict`` holds the codes."""

    def __init__(self, weight, bias=None):
        super().__init__()
        packed = molgrid.mg_mx_pack(weight.detach().contiguous(), "e2m1")
        self.features = weight.shape[1]
        self.register_buffer("codes", packed.codes)
        self.register_buffer("scales", packed.scales)
        self.register_buffer("bias", None if bias is None else bias.detach().float().clone())

    def forward(self, features, natoms=None):
        """``natoms`` is taken for the sake of ``AtomTyper``'s signature: every row is mapped."""
        if torch.is_grad_enabled() and features.requires_grad:
            raise RuntimeError("a typer in 4 bits has no gradient")
        if features.dim() != 3 or features.shape[2] != self.features:
            raise ValueError("features must have shape [B,N,%d], got %s" % (self.features, tuple(features.shape)))
        if features.numel() == 0:
            return features.new_empty(features.shape[:2] + (self.codes.shape[0],), dtype=torch.float32)
        weight = molgrid.MXTensor(self.codes, self.scales, (self.codes.shape[0], self.features), "e2m1")
        bias = None if self.bias is None else self.bias.float()
        return molgrid.mg_mx4_linear(_even_rows(features), weight, bias).float()


class GridLayer(torch.nn.Module):
    """A GridMaker as a differentiable layer: ``layer(coords, types=... | weights=..., ...)``
    returns the ``[B,T,D,D,D]`` grid (``[B,S,S,S,T,D,D,D]`` with ``subgrids_per_side`` = S > 1);
    gradients flow to ``coords`` (and ``weights``).  With a ``typer`` (``AtomTyper`` or
    ``AtomTyper4``) it also takes ``features`` [B,N,E], whose type weights the typer computes.

    ``random_rotation`` / ``random_translation`` (GridMaker.forward's optional augmentation): a
    fresh per-example rotation and a translation of at most that many Angstrom per axis are
    drawn on the device for every call (``mg_draw_transforms``, counter-based: ``seed`` and the
    number of the call fix them) and kept in ``last_quats`` / ``last_translations``, so the
    applied transformation can be retained; gradients come back in the caller's frame."""

    def __init__(self, resolution=0.5, dimension=23.5, binary=False, radius_type_indexed=True,
                 radius_scale=1.0, gaussian_radius_multiple=1.0, subgrids_per_side=1, typer=None):
        super().__init__()
        self.typer = typer
        self.gm = molgrid.GridMaker(resolution, dimension, binary=binary,
                                    radius_type_indexed=radius_type_indexed,
                                    radius_scale=radius_scale,
                                    gaussian_radius_multiple=gaussian_radius_multiple,
                                    subgrids_per_side=subgrids_per_side)
        self.seed, self.draws = 0, 0
        self.last_quats = self.last_translations = None

    def forward(self, coords, radii, *, types: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None, T: Optional[int] = None, natoms=None,
                centers=None, quats=None, translations=None, random_rotation=False,
                random_translation=0.0, features: Optional[torch.Tensor] = None):
        if features is not None:
            if self.typer is None:
                raise ValueError("features need a typer (GridLayer(..., typer=AtomTyper(E, T)))")
            if types is not None or weights is not None:
                raise ValueError("give features, types or weights, not two of them")
            weights = self.typer(features, natoms)
        if (types is None) == (weights is None):
            raise ValueError("give exactly one of types (index) or weights (vector)")
        if random_rotation or random_translation > 0.0:
            if quats is not None or translations is not None:
                raise ValueError("give explicit transforms or ask for random ones, not both")
            quats, translations = molgrid.mg_draw_transforms(
                self.seed, self.draws, coords.shape[0], random_rotation=bool(random_rotation),
                max_translation=float(random_translation), device=coords.device)
            self.draws += 1
            self.last_quats, self.last_translations = quats, translations
        if types is not None:
            if T is None:
                raise ValueError("index types need the number of channels T")
            with _Exact():
                return _IndexGrid.apply(coords, self.gm, types, radii, T, natoms, centers, quats,
                                        translations)
        with _Exact():
            return _VectorGrid.apply(coords, weights, self.gm, radii, natoms, centers, quats,
                                     translations)
