"""What the logit operators accept and refuse beside the plain refusals, without a GPU: a call that passes its checks ends with MLMC_ERR_CUDA."""
import ctypes as C

import pytest
import torch

from test_logits_host import B, P, ctx, distill, distill_grad  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="a made-up context: only where nothing can be launched")


@pytest.mark.parametrize("at, ld, ldg, N, ok", [
    (400, 200, 200, 4, True), (-400, 200, 200, 4, True),             # the other half of a [4, 200] buffer, 100 logits in each
    (404, 204, 204, 4, True), (-404, 204, 204, 4, True),             # with columns between them
    (400 + 800, 200, 200, 4, True), (400 - 1600, 200, 200, 4, True),  # the halves of other rows
    (396, 200, 200, 4, False), (404, 200, 200, 4, False), (-396, 200, 200, 4, False), (-404, 200, 200, 4, False),
    (800, 200, 200, 4, False), (1200, 300, 300, 4, False), (1200, 200, 200, 2, True),   # a row on, over logits; behind the last row
    (400, 200, 100, 4, False), (400, 200, 201, 4, False),            # other strides: rows meet
    (396, 200, 200, 1, False), (400, 200, 200, 1, True), (-400, 200, 200, 1, True)])
def test_gradient_rows_between_the_logits(ctx, at, ld, ldg, N, ok):
    want = B.MLMC_ERR_CUDA if ok else B.MLMC_ERR_ARG
    assert distill(ctx, N=N, ld=ld, ldg=ldg, grad=P + at) == distill_grad(ctx, N=N, ld=ld, ldg=ldg, grad=P + at) == want


def test_tensors_on_another_gpu_than_the_context():
    """A kernel of one GPU on another's memory would fault: the binding looks before it calls."""
    here = C.c_void_p(P)
    here.device = 1
    for at in ("cuda:0", "cuda:2"):
        with pytest.raises(ValueError):
            B._stream_of(here, torch.device(at))


@pytest.mark.parametrize("states, meet", [
    ([(P, 2 * P, 64, 1, 0, 64), (3 * P, 4 * P, 64, 1, 0, 64)], False),
    ([(P, P, 64, 1, 0, 64), (2 * P, 2 * P, 64, 1, 0, 64)], False),
    ([(P, 2 * P, 64, 1, 0, 64), (2 * P, P, 64, 1, 0, 64)], True),                       # a swap
    ([(P, P, 64, 1, 0, 64), (P, P, 64, 1, 0, 64)], True),                               # one state twice
    ([(P, 2 * P, 64, 1, 0, 64), (3 * P, 2 * P + 255, 64, 1, 0, 64)], True),             # 4 beams: the last byte
    ([(P, 2 * P, 64, 1, 0, 64), (3 * P, 2 * P + 256, 64, 1, 0, 64)], False),
    ([(P, 2 * P, 64, 1, 0, 64), (P, 3 * P, 64, 1, 0, 64)], False),                      # one source, two copies
    ([(P, 2 * P, 64, 1, 0, 64), (P + 32, 3 * P, 64, 1, 0, 64)], False),
    ([(P, P, 64, 1, 0, 64), (P + 192, 3 * P, 64, 1, 0, 64)], True),                     # read where another one writes
    ([(P, P, 256, 1, 0, 128), (P + 128, P + 128, 256, 1, 0, 128)], False),              # between one another: keys and values of a beam
    ([(P, P, 256, 1, 0, 128), (P + 127, P + 127, 256, 1, 0, 128)], True),
    ([(P, P, 512, 4, 64, 32), (P + 32, P + 32, 512, 4, 64, 32)], False),                # and of a head
    ([(P, P, 512, 4, 64, 33), (P + 32, P + 32, 512, 4, 64, 32)], True),
    ([(P, P, 512, 4, 64, 32), (P + 32, P + 32, 512, 2, 128, 32)], False),               # other strides
    ([(P, P, 512, 4, 64, 32), (P + 160, P + 160, 512, 2, 32, 32)], True)])              # its second piece
def test_states_that_meet(states, meet):
    for order in (states, states[::-1]):
        assert B._meet([B.mlmc_beam_state(*x) for x in order], 4) is meet


def test_states_that_meet_are_looked_for_in_many(monkeypatch):
    many = [B.mlmc_beam_state(P + 4096 * i, 64 * P + 4096 * i, 1024, 1, 0, 1024) for i in range(300)]
    assert not B._meet(many, 4)
    assert B._meet(many + [B.mlmc_beam_state(2 * P, 64 * P + 4096 * 150 + 4095, 1024, 1, 0, 1)], 4)
    monkeypatch.setattr(B, "_MOST_PIECES", 4)             # views between one another in more pieces than that are taken as they are
    assert not B._meet([B.mlmc_beam_state(P, P, 64, 1, 0, 64), B.mlmc_beam_state(P, P, 64, 1, 0, 64)], 4)
