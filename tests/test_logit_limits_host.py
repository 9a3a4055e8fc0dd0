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
