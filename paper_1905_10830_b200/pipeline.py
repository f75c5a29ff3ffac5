"""Layer-by-layer calibration and chained coding of several layers' feature maps.

Section 3.1 ("Linear transform"): the covariance of a layer is estimated on a calibration batch
*with the layers before it already quantised*, so that every encoder sees, at calibration time,
the inputs it will see at inference.  Fig. 2 puts the codec between the layers: the feature map
a layer produces is encoded, stored, decoded, passed through the layer's non-linearity and
consumed by the next convolution.

The network itself is the caller's: a stage is any callable that maps the (reconstructed,
activated) feature map of the stage before to this stage's pre-activation feature map -- a
convolution and batch normalisation in the paper, any torch function here.  This module only
orders the calls of the C-ABI library (fit, statistics, codebook, encode, decode); every step
of the coding path runs in the library's kernels."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Callable, Sequence

import torch

from . import binding as tc


@dataclass
class CodedLayer:
    """What calibration leaves behind for one layer: its transform / quantiser and its code table."""
    model: tc.Model
    codebook: tc.Codebook
    bits: int
    relu: bool

    def close(self) -> None:
        self.model.close()
        self.codebook.close()


def code_layer(ctx: tc.Context, layer: CodedLayer, z: torch.Tensor):
    """Encode `z`, decode it again (with the layer's non-linearity when it has one) and return
    (reconstruction, coded bits): what the next stage reads from memory."""
    enc = tc.tc_encode(ctx, layer.model, layer.codebook, z)
    xhat = tc.tc_decode(ctx, layer.model, layer.codebook, enc, z.shape, z.dtype, relu=layer.relu)
    return xhat, enc.total_bits()


def calibrate_layer_by_layer(ctx: tc.Context, stages: Sequence[Callable[[torch.Tensor], torch.Tensor]],
                             calib_input: torch.Tensor, bits: Sequence[int], relu: Sequence[bool], *,
                             per_channel_codebook: bool = False, k: Sequence[int] | None = None) -> list[CodedLayer]:
    """Fit one CodedLayer per stage on `calib_input`.  Stage l's feature maps are computed from the
    *reconstruction* of stage l - 1 (encode, decode, non-linearity), never from its clean output, so
    the statistics each fit sees include the quantisation noise of everything upstream."""
    layers: list[CodedLayer] = []
    cur = calib_input
    for l, stage in enumerate(stages):
        z = stage(cur).contiguous()
        model = tc.tc_fit_pca(ctx, z, bits=bits[l], k=0 if k is None else k[l])
        groups = (k[l] if k is not None and k[l] else z.shape[1]) if per_channel_codebook else 1
        st = tc.tc_stats(ctx, model, None, z, groups=groups)
        cb = tc.tc_build_codebook(ctx, model, st.hist, groups=groups)
        layer = CodedLayer(model, cb, bits[l], bool(relu[l]))
        layers.append(layer)
        cur, _ = code_layer(ctx, layer, z)
    return layers


def run_chain(ctx: tc.Context, stages: Sequence[Callable[[torch.Tensor], torch.Tensor]], layers: Sequence[CodedLayer],
              x: torch.Tensor):
    """Inference through the chain: every stage's feature map goes through its encoder and decoder
    before the next stage reads it.  Returns (feature maps as coded, reconstructions, bits per layer)."""
    maps, recons, bits = [], [], []
    cur = x
    for stage, layer in zip(stages, layers):
        z = stage(cur).contiguous()
        cur, nbits = code_layer(ctx, layer, z)
        maps.append(z)
        recons.append(cur)
        bits.append(nbits)
    return maps, recons, bits


class ResidualBlock:
    """A residual block on the pixels' vectors, to stand between two coded maps (a stage of the functions above) or to be
    trained: s = h + scale * gate * norm(W norm(h) before) after, the 1 x 1 convolution W [C][C] as a product of 8-bit blocks.
    Vectors are float32 CUDA tensors [C] (`scale`: one value); `gate` and `scale` may be None.  Nothing is recorded for autograd: a
    training step takes its gradients from `gradients`."""

    def __init__(self, ctx: tc.Context, weight: torch.Tensor, *, before: torch.Tensor, after: torch.Tensor,
                 gate: torch.Tensor | None = None, scale: torch.Tensor | None = None, eps: float = 1e-6):
        if weight.dim() != 2 or weight.shape[0] != weight.shape[1]:
            raise ValueError("weight: expected [C][C]")
        self.ctx, self.eps, self.before = ctx, eps, before
        self.around = dict(after=after, gate=gate, scale=scale)
        self.set_weight(weight)

    def set_weight(self, weight: torch.Tensor) -> None:
        """New values of W: its codes, by rows for the product and by columns for the gradient to its input."""
        self.rows, self.columns = tc.tc_quantize_blocks(self.ctx, weight[:, :, None, None].contiguous(), rows="both", square=True)

    def __call__(self, h: torch.Tensor) -> torch.Tensor:
        n, _, hh, ww = h.shape
        _, codes = tc.tc_residual_norms(self.ctx, h, before=self.before, eps=self.eps, blocks=True)
        y = tc.tc_matmul_blocks(self.ctx, codes, self.rows, shape=(n, hh, ww), dtype=h.dtype)
        return tc.tc_residual_norms(self.ctx, h, y, eps=self.eps, **self.around)[0]

    def gradients(self, h: torch.Tensor, ds: torch.Tensor) -> dict:
        """Gradients to `h`, the weight (float32) and the vectors, from the gradient `ds` of the block's output; the forward
        pass is computed again (the same bits), the products' operands in both directions are 8-bit blocks."""
        n, c, hh, ww = h.shape
        _, (x, x_pixels) = tc.tc_residual_norms(self.ctx, h, before=self.before, eps=self.eps, blocks="both")
        x_channels = tc.tc_quantize_blocks(self.ctx, x, rows="channels")
        y = tc.tc_matmul_blocks(self.ctx, x_pixels, self.rows, shape=(n, hh, ww), dtype=h.dtype)
        s = tc.tc_residual_norms(self.ctx, h, y, eps=self.eps, **self.around)[0]
        outer = tc.tc_residual_norms_backward(self.ctx, s, y, None, ds, eps=self.eps, **self.around)
        dy_pixels, dy_channels = tc.tc_quantize_blocks(self.ctx, outer.y, rows="both")
        dx = tc.tc_matmul_blocks(self.ctx, dy_pixels, self.columns, shape=(n, hh, ww), dtype=h.dtype)
        dw = tc.tc_matmul_blocks(self.ctx, dy_channels, x_channels, dtype=torch.float32)
        inner = tc.tc_residual_norms_backward(self.ctx, h, None, dx, outer.h, before=self.before, eps=self.eps)
        return dict(h=inner.h, weight=dw.reshape(c, c), before=inner.before, after=outer.after, gate=outer.gate, scale=outer.scale)


def _pixels(x: torch.Tensor) -> torch.Tensor:
    """A channels_last tensor's pixels as a list of tokens, (N H W, C, 1, 1): a view."""
    return x.permute(0, 2, 3, 1).reshape(-1, x.shape[1], 1, 1)


class IntegerBlock:
    """A residual block on 8-bit integers, as the paper's networks run their layers, to stand between two coded maps or to be trained:
    s = h + W act(group_norm(h)), the 1 x 1 convolution W [C][C] as a product of integers with a scale for each pixel and each row of W.  Maps go in and
    come out in the same order, contiguous (as the codec's are; the block's own are channels_last, which costs one copy) or channels_last.
    Vectors are float32 CUDA tensors [C] or None.  Nothing is recorded for autograd: a training step takes its gradients from `gradients`."""

    def __init__(self, ctx: tc.Context, weight: torch.Tensor, *, groups: int, norm_weight: torch.Tensor | None = None, norm_bias: torch.Tensor | None = None,
                 eps: float = 1e-5, activation: str | None = "relu"):
        if weight.dim() != 2 or weight.shape[0] != weight.shape[1]:
            raise ValueError("weight: expected [C][C]")
        self.ctx, self.groups, self.eps = ctx, groups, eps
        self.norm = dict(weight=norm_weight, bias=norm_bias, activation=activation)
        self.set_weight(weight)

    def set_weight(self, weight: torch.Tensor) -> None:
        """New values of W: its codes, by rows for the product and by columns for the gradient to its input."""
        self.rows, self.columns = tc.tc_quantize_rows(self.ctx, weight[:, :, None, None].contiguous(), rows="both")

    def _sum(self, a: torch.Tensor, b: torch.Tensor) -> torch.Tensor:
        if a.is_contiguous():
            return tc.tc_residual_norms(self.ctx, a, b.contiguous())[0]
        n, c, h, w = a.shape
        return tc.tc_residual_norms(self.ctx, _pixels(a), _pixels(b))[0].view(n, h, w, c).permute(0, 3, 1, 2)

    def __call__(self, h: torch.Tensor) -> torch.Tensor:
        n, _, hh, ww = h.shape
        x = h.contiguous(memory_format=torch.channels_last)
        codes, _ = tc.tc_group_norm(self.ctx, x, self.groups, eps=self.eps, codes=True, **self.norm)
        y = tc.tc_matmul_rows(self.ctx, codes, self.rows, shape=(n, hh, ww), dtype=h.dtype, channels_last=not h.is_contiguous())
        return self._sum(h if h.is_contiguous() else x, y)

    def gradients(self, h: torch.Tensor, ds: torch.Tensor) -> dict:
        """Gradients to `h`, the weight (float32) and the vectors, from the gradient `ds` of the block's output; the norm is computed again, the
        products' operands in both directions are 8-bit integers."""
        n, c, hh, ww = h.shape
        x, d = (t.contiguous(memory_format=torch.channels_last) for t in (h, ds))
        xn, stats = tc.tc_group_norm(self.ctx, x, self.groups, eps=self.eps, **self.norm)
        d_pixels, d_channels = tc.tc_quantize_rows(self.ctx, d, rows="both")
        dxn = tc.tc_matmul_rows(self.ctx, d_pixels, self.columns, shape=(n, hh, ww), dtype=h.dtype, channels_last=True)
        dw = tc.tc_matmul_rows(self.ctx, d_channels, tc.tc_quantize_rows(self.ctx, xn, rows="channels"), dtype=torch.float32)
        inner = tc.tc_group_norm_backward(self.ctx, x, dxn, stats, **self.norm)
        return dict(h=self._sum(ds if ds.is_contiguous() else d, inner.x), weight=dw.reshape(c, c), norm_weight=inner.weight, norm_bias=inner.bias)


def chain_gradients(ctx: tc.Context, blocks: Sequence, h: torch.Tensor, ds: torch.Tensor, max_norm: float):
    """A training step's gradients through blocks that follow one another (ResidualBlock, IntegerBlock): each block's by its names and without its
    input's, all of them clipped to `max_norm` together, and their norm before that (float32 [1])."""
    inputs = [h]
    for block in blocks[:-1]:
        inputs.append(block(inputs[-1]))
    grads = []
    for block, x in zip(reversed(blocks), reversed(inputs)):
        g = block.gradients(x, ds)
        ds = g.pop("h")
        grads.insert(0, g)
    norm = tc.tc_clip_gradients(ctx, [v for g in grads for v in g.values() if v is not None], max_norm)
    return grads, norm
