"""Attention within packed sub-graphs as a layer, composed from library calls (call
order and buffers only; the projections are plain matrix products of torch).

    [q k v] = u Wqkv^T, q and k normed for each head and rotated by the nodes' coordinates
    out = softmax(c(q.k / sqrt(head_dim)) - slope |p_i - p_j|) v  over the nodes of a sub-graph
    f = out Wo^T

Message passing reaches the neighbours within the radius; here every node of a sub-graph
sees every other one.  u is what a norm hands to a layer (dsmp_group_norm_forward), f is
float32, the addend of the next norm, as a message-passing layer's output is; f, the
gradient of u and those of the weights are float32 sums in either type, while q, k, v and
what grad_f hands back to them are operands of the next products and have the layer's type.
"""

from dataclasses import dataclass

import torch

from . import _lib as L


@dataclass
class AttentionShapes:
    n: int                 # nodes
    d: int                 # width of u and f
    heads: int
    kv_heads: int          # divides heads
    head_dim: int          # a multiple of 8, at most 128
    dtype: int             # F32 or BF16: u and the weights
    dim: int               # coordinates (1..3): of the rotation and of the distance
    rot: int = 0           # rotated values of each head
    layout: int = L.ROTATE_HALF
    norm: bool = True      # queries and keys normed
    cap: float = 0.0
    distance: bool = True  # whether scores fall with the distance
    eps: float = 1e-6


def _sums(a, b):
    """a @ b as float32 sums, whatever the operands' type (rounded to bfloat16 and back they would keep 8 bits)."""
    return torch.mm(a, b) if a.dtype == torch.float32 else torch.mm(a, b, out_dtype=torch.float32)


class AttentionLayer:
    """Buffers for n nodes; ``forward`` gives f, ``backward`` the gradients of the forward
    call that came last, with its arguments as they were.  ``read`` is for evaluation: few points
    that read the field of many nodes.

    params: Wqkv [(heads + 2 kv_heads) head_dim, d], Wo [d, heads head_dim] (of the layer's type),
    gamma_q, gamma_k (float32 [head_dim], with norm), freq (float32 [rot / 2], with rot),
    slopes (float32 [heads], with distance)."""

    def __init__(self, lib: "L.Dsmp", s: AttentionShapes):
        self.lib, self.s = lib, s
        self.rotate = L.rotate_desc(s.heads, s.kv_heads, s.head_dim, s.dtype, s.rot, axes=s.dim, layout=s.layout,
                                    norm=s.norm, eps=s.eps)
        self.attend = L.attention_desc(s.heads, s.kv_heads, s.head_dim, s.dtype, dim=s.dim if s.distance else 0, cap=s.cap)
        self.wq, self.wk = s.heads * s.head_dim, s.kv_heads * s.head_dim
        self._kept = None

    def _checked(self, u, what):
        if u.dim() != 2 or u.shape[1] != self.s.d or u.dtype is not L._TORCH.get(self.s.dtype):
            raise L.DsmpError(L.INVALID_ARG, "%s: a %s matrix of %d columns is needed" % (what, L._TORCH.get(self.s.dtype), self.s.d))
        return u

    @staticmethod
    def _buffer(like, segments):
        """Rows of no segment stay as they are: zero."""
        return torch.zeros_like(like) if isinstance(segments, torch.Tensor) else torch.empty_like(like)

    def _room(self, segments):
        """Which rows belong to no segment, [n, 1], by the bounds on the device (None: there are none)."""
        self.lib._segments(self.s.n, segments)   # refused here, or they are bounds on the device
        if not isinstance(segments, torch.Tensor):
            return None
        rows = torch.arange(self.s.n, dtype=torch.int32, device=segments.device)[:, None]   # on the call's own stream
        below = rows < segments[::segments.numel() - 1]   # the first bound and the last one
        return below[:, :1] == below[:, 1:]

    @staticmethod
    def _cleared(t, room):
        """t without what it holds in those rows (what is no matrix is refused by the calls that take it)."""
        return t if room is None or t is None or t.dim() != 2 else torch.where(room, 0.0, t)

    def _attention(self, p, q, k, v, pos, k_pos, segments, k_segments):
        place = dict(pos=pos, k_pos=k_pos, slopes=p["slopes"]) if self.s.distance else {}
        return place, self.lib.dsmp_attention_forward(self.attend, q, k, v, segments=segments, k_segments=k_segments,
                                                      out=self._buffer(q, segments), **place)

    def forward(self, params: dict, u: torch.Tensor, pos: torch.Tensor, segments=None) -> torch.Tensor:
        """f [n, d] (float32) of u [n, d] at pos (float32 [n, dim]); segments as for dsmp_attention_forward: whatever
        u, pos and later grad_f hold in rows in front of the first bound and behind the last one (room
        for further sub-graphs), f and the gradient of u are 0 there, and the other gradients know nothing of them."""
        lib, p, wq, wk = self.lib, params, self.wq, self.wk
        self._kept = None
        if self._checked(u, "u").shape[0] != self.s.n:
            raise L.DsmpError(L.INVALID_ARG, "u: %d rows are needed" % self.s.n)
        room = self._room(segments)
        u, pos = self._cleared(u, room), self._cleared(pos, room)
        qkv = torch.mm(u, p["Wqkv"].t())
        if room is not None and self.s.norm and self.s.eps == 0.0:
            qkv.masked_fill_(room, 1.0)   # rows of zeros have no norm without eps; their gradients are 0 times what there is
        q, k, v = qkv[:, :wq], qkv[:, wq:wq + wk], qkv[:, wq + wk:]
        qr, kr = lib.dsmp_qk_rotate_forward(self.rotate, q, k, p.get("gamma_q"), p.get("gamma_k"), pos, p.get("freq"))
        place, (out, lse) = self._attention(p, qr, kr, v, pos, None, segments, None)
        f = _sums(out, p["Wo"].t())
        self._kept = (p, u, pos, segments, room, place, qkv, qr, kr, out, lse)
        return f

    def backward(self, grad_f: torch.Tensor):
        """(grad_u float32, {"dWqkv", "dWo"[, "dgamma_q", "dgamma_k"]}) of sum(grad_f * f)."""
        if self._kept is None:
            raise L.DsmpError(L.INVALID_ARG, "no forward call that came to its end")
        lib, wq, wk = self.lib, self.wq, self.wk
        p, u, pos, segments, room, place, qkv, qr, kr, out, lse = self._kept
        q, k, v = qkv[:, :wq], qkv[:, wq:wq + wk], qkv[:, wq + wk:]
        if grad_f.shape != (self.s.n, self.s.d):
            raise L.DsmpError(L.INVALID_ARG, "grad_f: a matrix of %d rows and %d columns is needed" % (self.s.n, self.s.d))
        g = self._cleared(grad_f.to(u.dtype), room)
        dqkv = self._buffer(qkv, segments)
        dq, dk, dv = dqkv[:, :wq], dqkv[:, wq:wq + wk], dqkv[:, wq + wk:]
        lib.dsmp_attention_backward(self.attend, qr, kr, v, out, lse, torch.mm(g, p["Wo"]), segments=segments,
                                    grad_q=dq, grad_k=dk, grad_v=dv, **place)
        _, _, grads = lib.dsmp_qk_rotate_backward(self.rotate, q, k, p.get("gamma_q"), p.get("gamma_k"), pos, p.get("freq"),
                                                  dq, dk, grad_q=dq, grad_k=dk)
        grads["dWqkv"], grads["dWo"] = _sums(dqkv.t(), u), _sums(g.t(), out)
        return _sums(dqkv, p["Wqkv"]), grads

    def read(self, params: dict, u, pos, u_keys, pos_keys, segments=None, k_segments=None) -> torch.Tensor:
        """f [m, d] (float32) at m points with features u and coordinates pos, from the nodes u_keys,
        pos_keys of the same segments.  Nothing is kept."""
        lib, p, wq, wk = self.lib, params, self.wq, self.wk
        q = torch.mm(self._checked(u, "u"), p["Wqkv"][:wq].t())
        kv = torch.mm(self._checked(u_keys, "u_keys"), p["Wqkv"][wq:].t())
        lib.dsmp_qk_rotate_forward(self.rotate, q, None, p.get("gamma_q"), None, pos, p.get("freq"), q_out=q)
        k = kv[:, :wk]
        lib.dsmp_qk_rotate_forward(self.rotate, None, k, None, p.get("gamma_k"), pos_keys, p.get("freq"), k_out=k)
        _, (out, _) = self._attention(p, q, k, kv[:, wk:], pos, pos_keys, segments, k_segments)
        return _sums(out, p["Wo"].t())
