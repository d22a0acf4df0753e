"""Which stream's memory the buffers of paper_2507_03220_amd/head.py are (see test_block_streams.py).  The calls and torch's allocator are stood in for; no GPU is touched."""
import pytest
import torch

from paper_2507_03220_amd import binding as sb
from paper_2507_03220_amd import head as hd
from test_block_streams import HERE, _check, world  # noqa: F401


@pytest.fixture
def head(world, monkeypatch):  # noqa: F811
    monkeypatch.setattr(hd, "_on", __import__("paper_2507_03220_amd.block", fromlist=["_on"])._on)

    def call(name, stream_at):
        return lambda *a: world.calls.append((name, a[stream_at], [x.data_ptr() for x in a if isinstance(x, torch.Tensor)]))
    for name, at in (("symb_cross_entropy", 9), ("symb_distillation", 10)):
        monkeypatch.setattr(sb, name, call(name, at))
    monkeypatch.setattr(sb, "symb_norm_bwd", call("symb_norm_bwd", 7))
    W = torch.zeros(24, 16, dtype=torch.bfloat16)
    return hd.LossHead(None, W, [3, 2], [sb.Norm(), sb.Norm()], [sb.Loss(), sb.Loss()])


# (held: no address of theirs is a buffer's later)
X, LABELS, IDS, LOGITS = torch.zeros(5, 16, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32), torch.zeros(5, 40, dtype=torch.int32), torch.zeros(5, 40)
MANY = torch.zeros(5, 900, dtype=torch.int32), torch.zeros(5, 900)


@pytest.mark.parametrize("order", [(HERE,), (9,), (0,), (9, HERE, 9), (9, 11, HERE)])
def test_steps_on_any_stream(world, head, order):  # noqa: F811
    for s in order:
        loss, dX = head.cross_entropy(X, LABELS, stream=s)
        assert loss is head.loss and dX is head.dX
        assert head.cross_entropy(X, LABELS, gradient=False, stream=s)[1] is None
        head.distillation(X, IDS, LOGITS, stream=s)
    _check(world)


def test_buffers_stay_while_the_stream_does(world, head):  # noqa: F811
    loss, dX = head.cross_entropy(X, LABELS, stream=9)
    ws = head.ws
    again = head.cross_entropy(X, LABELS, stream=9)
    assert again[0] is loss and again[1] is dX and head.ws is ws
    head.distillation(X, *MANY, stream=9)        # (needs more room)
    assert head.ws is not ws and head.ws.numel() >= sb.symb_loss_workspace_bytes(head.batch, 900, True)


def test_one_norm_and_one_loss_for_each_client():
    W = torch.zeros(24, 16, dtype=torch.bfloat16)
    for norms, losses in ((1, 2), (2, 1), (3, 2)):
        with pytest.raises(ValueError):
            hd.LossHead(None, W, [3, 2], [sb.Norm()] * norms, [sb.Loss()] * losses)
