"""check=True of a call whose tensors are on another device than the current one: it is that device's stream that is waited for, and its workspace that is looked at (no GPU needed: the
binding and the streams are stand-ins)."""
import contextlib

import pytest
import torch

from paper_2508_12594_b200 import flare


class Workspace:
    device = torch.device("cuda", 1)


class Native:
    """What the binding returns, workspace last."""

    def token_loss(self, *a):
        return "result", Workspace()

    token_loss_backward = token_loss


@pytest.mark.parametrize("call", [lambda s: flare.token_loss(0, 0, 0, stream=s, check=True), lambda s: flare.token_loss_backward(0, 0, 0, 0, stream=s, check=True)], ids=["loss", "gradients"])
@pytest.mark.parametrize("given", [False, True])
def test_the_stream_that_is_waited_for(monkeypatch, call, given):
    seen, now = [], ["cuda:0"]

    class Stream:
        def __init__(self, name):
            self.name = name

        def synchronize(self):
            seen.append(("waited", self.name))

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], str(d)
        yield
        now[0] = before

    monkeypatch.setattr(flare, "_native", Native())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream("of " + str(d or now[0])))
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(flare, "flare_check", lambda ws, stream=None: seen.append(("checked", now[0], stream and stream.name)))
    mine = Stream("mine") if given else None
    assert call(mine) == "result"
    assert seen == [("waited", "mine" if given else "of cuda:1"), ("checked", "cuda:1", "mine" if given else None)]
