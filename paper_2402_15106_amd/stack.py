"""A deep pre-norm stack of message-passing layers, trained with its
activations kept in 8 bits; composed from library calls (call order and buffers
only, no arithmetic happens here).

    s_0 = x;  for each layer l:  u_l = act(norm_l(s_l)),  s_{l+1} = s_l + K_l(u_l)
    y = norm_L(s_L)

The residual stream s is float32.  The addition of a layer's output is part of
the next norm's forward call, and its gradient, which passes by the norm, part of
the norm's backward call.

With ``checkpoints`` what stays between the forward and the backward pass is
each s_l in 8 bits and its norms' statistics.  One `saved` buffer serves all
layers: the backward pass rebuilds each layer's operand u_l from the checkpoint
(dsmp_group_norm_restore) and runs the layer's forward again before its
backward.  Without them every layer keeps its own `saved` buffer, u_l and s_l.
"""

from dataclasses import dataclass
from typing import Sequence, Tuple

import torch

from . import _lib as L


@dataclass
class StackShapes:
    n: int            # nodes (all destinations)
    dim: int          # spatial dimension; node attributes have dim + 1 components
    d: int            # width of the stream and of every layer
    h1: int
    h2: int
    dtype: int        # F32 or BF16: the layers' operands u
    layers: int
    groups: int       # of the norms
    act: int = L.ACT_SILU
    eps: float = 1e-5


class CheckpointedStack:
    """Buffers for one graph; ``forward`` gives y, ``backward`` the gradients of
    the forward pass that came last.

    segments: the packed sub-graphs that the norms' statistics are taken over, as
    in ``Dsmp.dsmp_group_norm_forward`` (None: the whole graph)."""

    def __init__(self, lib: "L.Dsmp", graph: "L.Graph", s: StackShapes, segments=None, checkpoints: bool = True):
        if s.layers < 1:
            raise L.DsmpError(L.INVALID_ARG, "a stack has at least one layer")
        if graph.n_dst != s.n or graph.n_src != s.n:
            raise L.DsmpError(L.INVALID_ARG, "every node of the graph is a destination")
        self.lib, self.g, self.s, self.segments, self.checkpoints = lib, graph, s, segments, checkpoints
        n, d, dev = s.n, s.d, lib.device
        f32 = dict(dtype=torch.float32, device=dev)
        self.conv = L.layer_desc(s.dim, d, s.h1, s.h2, s.dtype, L.ACT_IDENTITY, 0, L.ATTR_CONCAT)
        self.norm = L.norm_desc(d, s.groups, L.F32, s.dtype, s.act, s.eps)
        self.last = L.norm_desc(d, s.groups, L.F32, L.F32, L.ACT_IDENTITY, s.eps)
        tdt = torch.bfloat16 if s.dtype == L.BF16 else torch.float32
        one = checkpoints
        sb, fb, bb = lib.dsmp_nnconv_workspace(self.conv, graph)
        self.saved = [torch.empty(max(sb, 256), dtype=torch.uint8, device=dev) for _ in range(1 if one else s.layers)]
        self.u = [torch.empty(n, d, dtype=tdt, device=dev) for _ in range(1 if one else s.layers)]
        self.stream = [torch.empty(n, d, **f32) for _ in range(1 if one else s.layers)]
        self.kept = [L.Checkpoint.empty(n, d, dev) if one else None for _ in range(s.layers + 1)]
        n_seg = 1 if segments is None else segments.numel() - 1 if isinstance(segments, torch.Tensor) else int(segments)
        self.stats = [torch.empty(n_seg, s.groups, 2, **f32) for _ in range(s.layers + 1)]
        self.f = torch.empty(n, d, **f32)
        self.y = torch.empty(n, d, **f32)
        self.gu = torch.empty(n, d, **f32)
        self.fws = torch.empty(max(fb, 256), dtype=torch.uint8, device=dev)
        self.bws = torch.empty(max(bb, 256), dtype=torch.uint8, device=dev)
        self._whole = False     # a forward pass has ended
        self._holds = None      # with checkpoints: the layer whose operand and `saved` the buffers hold

    def kept_bytes(self) -> int:
        """Bytes held from the forward to the backward pass."""
        held = self.saved + self.u + self.stats
        held += [t for c in self.kept if c is not None for t in (c.q, c.scale)]
        held += [] if self.checkpoints else self.stream
        return sum(t.numel() * t.element_size() for t in held)

    def _at(self, buffers, l):
        return buffers[0 if self.checkpoints else l]

    def forward(self, packed: Sequence[torch.Tensor], norms: Sequence[Tuple[torch.Tensor, torch.Tensor]],
                attr: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
        """y [n, d] of the stack on x (float32 [n, d], left as it is).  packed: each
        layer's parameters (dsmp_nnconv_pack); norms: layers + 1 pairs (gamma, beta)."""
        lib, s = self.lib, self.s
        self._whole, self._holds = False, None
        self.attr, self.packed, self.norms, self.x = attr, packed, norms, x
        for l in range(s.layers + 1):
            end = l == s.layers
            add = dict(addend=self.f, sum_out=self._at(self.stream, l - 1)) if l else {}
            before = x if l < 2 else self._at(self.stream, l - 2)
            lib.dsmp_group_norm_forward(self.last if end else self.norm, before, *norms[l], segments=self.segments,
                                        y=self.y if end else self._at(self.u, l), stats=self.stats[l],
                                        checkpoint=self.kept[l], **add)
            if not end:
                lib.dsmp_nnconv_forward(self.conv, packed[l], self.g, attr, self._at(self.u, l), h_out=self.f,
                                        saved=self._at(self.saved, l), ws=self.fws)
                self._holds = l
        self._whole = True
        return self.y

    def backward(self, grad_y: torch.Tensor):
        """(grad_x, layer gradients, norm gradients) of sum(grad_y * y) for the
        forward pass that came last, with its arguments as they were.  It may be called
        again, with another grad_y; with checkpoints the last layer's operand, which the
        first call still has as it was, then comes from its checkpoint, as the others' do."""
        if not self._whole:
            raise L.DsmpError(L.INVALID_ARG, "no forward pass that came to its end")
        lib, s, seg = self.lib, self.s, self.segments

        def source(l):
            return self.kept[l] if self.checkpoints else self.x if l == 0 else self.stream[l - 1]

        conv_g, norm_g = [None] * s.layers, [None] * (s.layers + 1)
        G, norm_g[s.layers] = lib.dsmp_group_norm_backward(self.last, source(s.layers), self.stats[s.layers],
                                                           *self.norms[s.layers], grad_y, segments=seg)
        for l in reversed(range(s.layers)):
            u, saved = self._at(self.u, l), self._at(self.saved, l)
            # after the forward pass the last layer's operand and what it saved are still there
            if self.checkpoints and l != self._holds:
                self._holds = None
                lib.dsmp_group_norm_restore(self.norm, self.kept[l], self.stats[l], *self.norms[l], segments=seg, y=u)
                lib.dsmp_nnconv_forward(self.conv, self.packed[l], self.g, self.attr, u, h_out=self.f, saved=saved,
                                        ws=self.fws)
                self._holds = l
            _, conv_g[l] = lib.dsmp_nnconv_backward(self.conv, self.packed[l], self.g, self.attr, u, saved, G,
                                                    grad_h=self.gu, ws=self.bws)
            _, norm_g[l] = lib.dsmp_group_norm_backward(self.norm, source(l), self.stats[l], *self.norms[l], self.gu,
                                                        segments=seg, grad_addend=G, grad_x=G)
        return G, conv_g, norm_g
