"""Order of the calls of the stack with checkpoints, on a stand-in for the library that
works on the CPU: each buffer holds the number of the layer that it was written for."""

import pytest

torch = pytest.importorskip("torch")

import paper_2402_15106_amd as dm  # noqa: E402

N, D, LAYERS = 4, 8, 4


class StandIn:
    """The norms' parameters and the layers' packed parameters are the layer's number."""
    device = torch.device("cpu")

    def __init__(self):
        self.seen = []      # of each layer's backward: (layer, whose operand, whose saved)

    def dsmp_nnconv_workspace(self, desc, graph):
        return N, 1, 1

    def dsmp_group_norm_forward(self, desc, x, gamma, beta, segments=None, addend=None, sum_out=None, y=None, stats=None,
                                checkpoint=None):
        y.fill_(gamma)
        stats.fill_(gamma)
        if checkpoint is not None:
            checkpoint.q.fill_(gamma)
        return y, stats

    def dsmp_group_norm_restore(self, desc, checkpoint, stats, gamma, beta, segments=None, y=None):
        assert (checkpoint.q == gamma).all() and (stats == gamma).all()
        return y.fill_(gamma)

    def dsmp_group_norm_backward(self, desc, source, stats, gamma, beta, grad_y, segments=None, grad_addend=None,
                                 grad_x=None):
        assert (stats == gamma).all()
        return torch.zeros(N, D) if grad_x is None else grad_x, {}

    def dsmp_nnconv_forward(self, desc, packed, graph, attr, u, h_out=None, saved=None, ws=None):
        assert (u == packed).all()
        saved.fill_(packed)

    def dsmp_nnconv_backward(self, desc, packed, graph, attr, u, saved, grad_out, grad_h=None, ws=None):
        self.seen.append((packed, float(u[0, 0]), int(saved[0])))
        return grad_h, {}


class Square:
    n_dst = n_src = N


def stack(checkpoints, layers=LAYERS):
    lib = StandIn()
    s = dm.CheckpointedStack(lib, Square, dm.StackShapes(N, 2, D, 8, 8, dm.F32, layers, 1), checkpoints=checkpoints)
    args = (list(range(layers)), [(l, l) for l in range(layers + 1)], None, torch.zeros(N, D))
    return lib, s, args


@pytest.mark.parametrize("checkpoints", [True, False])
@pytest.mark.parametrize("layers", [1, 2, LAYERS])
def test_every_backward_runs_on_its_own_layers_operand(checkpoints, layers):
    lib, s, args = stack(checkpoints, layers)
    want = [(l, l, l) for l in reversed(range(layers))]
    for _ in range(2):
        s.forward(*args)
        for _ in range(3):
            lib.seen.clear()
            s.backward(torch.zeros(N, D))
            assert lib.seen == want


@pytest.mark.parametrize("checkpoints", [True, False])
def test_no_backward_of_a_forward_that_did_not_end(checkpoints):
    """Before any forward pass, and after one that raised on its way over an earlier one's buffers."""
    lib, s, args = stack(checkpoints)
    with pytest.raises(dm.DsmpError) as e:
        s.backward(torch.zeros(N, D))
    assert e.value.status == dm.INVALID_ARG
    s.forward(*args)
    s.backward(torch.zeros(N, D))
    with pytest.raises(IndexError):
        s.forward(args[0][:2], *args[1:])
    lib.seen.clear()
    with pytest.raises(dm.DsmpError):
        s.backward(torch.zeros(N, D))
    assert not lib.seen
    s.forward(*args)
    s.backward(torch.zeros(N, D))
    assert len(lib.seen) == LAYERS
