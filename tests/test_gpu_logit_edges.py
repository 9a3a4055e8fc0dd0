"""The logit operators where digits, forms and places are easily lost: against 64 bits, with bounds that count roundings.

u = 2^-24 is one rounding of fp32, 4 u an exponential, sum_tolerance(V) the relative error of a row's sum (its derivation stands beside it).
"""
import ctypes as C
import math

import pytest
import torch

from test_gpu_logits import B, DTYPES, INF, U, bits, check_distill, check_top, ctx, distill_reference, message, rows_of, sum_tolerance  # noqa: F401

pytestmark = pytest.mark.gpu


def messages_of(B, msg, rows):
    return B.LogitBuffers.of(msg.idx[rows].contiguous(), msg.val[rows].contiguous(), msg.count[rows].contiguous(), msg.rest[rows].contiguous())


# ------------------------------------------------------------------------------------------ digits of the gradient
@pytest.mark.parametrize("T", [1.0, 2.0, 30.0])
@pytest.mark.parametrize("N, V, k", [(40, 700, 8), (300, 5000, 8), (9, 50_257, 20), (310, 33_000, 6), (600, 66_001, 8)])
def test_gradient_outside_the_message_keeps_its_digits(B, ctx, N, V, k, T):
    """Flat rows of a student next to its teacher: of an unsent logit's gradient w T p_i (1 - q_r / p_r) all but 1e-5 or so cancels.

    1 - q_r / p_r = (p_r q_s - q_r p_s) / p_r, with p_s and q_s what is sent, so the difference is off by the errors of both products, each of
    at most three sums and exponentials: relative errors of terms as small as p_s.  What it is multiplied by is as exact as everywhere."""
    z = rows_of(V, N, torch.float32, V, scale=0.3)
    t = z.double()
    idx = torch.rand((N, V), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").topk(k, 1).indices
    val = (t.gather(1, idx) + 0.02 * T * torch.randn((N, k), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")).float()
    behind = t.scatter(1, idx, -INF)
    rest = torch.logsumexp((behind - val.double().max(1, keepdim=True).values) / T, 1).float()
    msg = B.LogitBuffers.of(idx.int().contiguous(), val.contiguous(), torch.full((N,), k, dtype=torch.int32, device="cuda"), rest)
    weight = torch.rand(N, device="cuda") + 0.5
    sent = torch.zeros((N, V), dtype=torch.bool, device="cuda").scatter_(1, idx, True)
    x = t / T
    ln_p = x - torch.logsumexp(x, 1, keepdim=True)
    p_s = ln_p.gather(1, idx).exp().sum(1, keepdim=True)
    p_r = torch.logsumexp(torch.where(sent, -INF, ln_p), 1, keepdim=True).exp()
    parts = torch.cat([val.double() / T, val.double().max(1, keepdim=True).values / T + rest.double()[:, None]], 1)
    q = torch.softmax(parts, 1)
    q_r, q_s = q[:, -1:], q[:, :-1].sum(1, keepdim=True)
    left = p_r * q_s - q_r * p_s
    scale = weight.double()[:, None] * T * ln_p.exp() / p_r
    want = scale * left
    assert float((left.abs() / p_r).median()) < 1e-3
    span = float((x.max(1).values - x.min(1).values).max())
    eps = sum_tolerance(V) + (8 + 3 * span) * U
    off = scale * (3 * eps * (p_r * q_s + q_r * p_s) + left.abs() * (3 * eps + (16 + 3 * span) * U)) + want.abs() * U + 1e-37
    for apart in (False, True):
        buf, grad = B.DistillBuffers(N), torch.full_like(z, 7.0)
        B.mlmc_distill(ctx, z, msg, T, True, weight, buf, None if apart else grad)
        if apart:
            B.mlmc_distill_grad(ctx, z, msg, T, True, weight, buf, grad)
        err = (grad.double() - want).abs()
        assert (err <= off)[~sent].all(), (apart, float((err / off)[~sent].max()))
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


def test_teacher_probabilities_next_to_a_large_rest(B, ctx):
    """Two buckets, a message of one entry and the rest: q = 1 / (1 + e^rest) and what is left of 1.  An exponential, the sum, the division and
    two products: 8 u.  The student says nothing of what is read off here, so the gradient is -q."""
    rest = torch.cat([torch.linspace(0.01, 80.0, 3000), torch.linspace(-80.0, -0.01, 3000), torch.tensor([-INF, 0.0, 84.0])]).cuda()
    N, V = rest.numel(), 9
    zero = torch.zeros((N, 1), device="cuda")
    msg = B.LogitBuffers.of(zero.int(), zero + 2.5, torch.ones(N, dtype=torch.int32, device="cuda"), rest)
    for others in (True, False):
        z = torch.zeros((N, V), device="cuda")
        if others:
            z[:, 0] = -INF
            want, at = torch.sigmoid(-rest.double()), 0
        else:
            z[:, 1], z[:, 2:] = -300.0, -INF
            want, at = torch.sigmoid(rest.double()), 1
        grad = torch.full_like(z, 7.0)
        B.mlmc_distill(ctx, z, msg, 1.0, True, None, B.DistillBuffers(N), grad)
        err = (-grad[:, at].double() - want).abs()
        assert (err <= 8 * U * want + 1e-37).all(), (others, float((err / want / U)[want > 0].max()))
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ where the gradient may lie
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N, V, gap", [(1, 300, 0), (7, 300, 0), (7, 301, 3), (40, 50_257, 1), (600, 9000, 0), (600, 66_001, 1)])
def test_gradient_in_the_other_columns_of_one_buffer(B, ctx, N, V, gap, dtype):
    memory = torch.full((N, 2 * V + gap), 7.0, dtype=dtype, device="cuda")
    for left in (True, False):
        z, grad = (memory[:, :V], memory[:, V + gap:]) if left else (memory[:, V + gap:], memory[:, :V])
        z.copy_(rows_of(V, N, dtype, V))
        kept = z.clone()
        msg = message(B, rows_of(V, N, torch.float32, V + 1), 12, 1.0)
        want, loss = torch.zeros((N, V), dtype=dtype, device="cuda"), B.DistillBuffers(N)
        B.mlmc_distill(ctx, z, msg, 1.0, True, None, loss, want)
        buf = B.DistillBuffers(N)
        B.mlmc_distill(ctx, z, msg, 1.0, True, None, buf, grad)
        assert torch.equal(grad, want) and torch.equal(buf.loss, loss.loss) and torch.equal(bits(z.contiguous()), bits(kept))
        grad.fill_(5.0)
        B.mlmc_distill_grad(ctx, z, msg, 1.0, True, None, buf, grad)
        B.mlmc_distill_grad(ctx, z, msg, 1.0, True, None, buf, want)
        assert torch.equal(grad, want) and torch.equal(bits(z.contiguous()), bits(kept))
        assert (memory[:, V:V + gap] == 7.0).all()
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ beams that are nearly equal
@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("V, scale", [(40, 1.0), (5000, 0.5), (50_257, 3.0)])
def test_continuations_of_two_beams_next_to_one_another(B, ctx, V, scale, T):
    """Best continuations up to 4e-6 apart: as far as the rows' sums tell beams apart, they come in order; a beam's own always do."""
    Bn, W, K = 300, 2, 6
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn((Bn * W, V), generator=g, device="cuda") * scale
    x = z.double() / T
    ln_p = (x - torch.logsumexp(x, 1, keepdim=True)).reshape(Bn, W, V)
    top = ln_p.max(2).values
    score = -5.0 - torch.rand((Bn, W), generator=g, device="cuda")
    apart = (torch.rand(Bn, generator=g, device="cuda").double() - 0.5) * 8e-6
    score[:, 1] = (score[:, 0].double() + top[:, 0] - top[:, 1] + apart).float()
    rows, out = B.LogitBuffers(Bn * W, K), B.BeamBuffers(Bn, K)
    B.mlmc_top_logits(ctx, z, None, T, rows)
    B.mlmc_beam_select(ctx, rows, V, W, T, score, None, -1, out)
    total = score.double()[:, :, None] + ln_p
    best, at = torch.sort(total.reshape(Bn, -1), dim=1, descending=True, stable=True)
    tol = sum_tolerance(V, K) + U * math.log(V)                  # of a row's logarithm, as in the tests of the selection
    flat = out.parent.long() * V + out.token.long()
    mine = total.reshape(Bn, -1).gather(1, flat)
    assert ((out.score.double() - mine).abs() <= tol + U * mine.abs()).all()
    assert (out.score[:, 1:] <= out.score[:, :-1]).all()
    assert ((mine - best[:, :K]).abs() <= 2 * tol).all()
    clear = (best[:, :K] - best[:, 1:K + 1] > 2 * tol).all(1)
    assert torch.equal(flat[clear], at[:, :K][clear])
    order = torch.sort(z.double(), dim=1, descending=True, stable=True).indices.reshape(Bn, W, V)
    for w in range(W):                                           # the beam's tokens are the first ones of its row, in order
        place = (out.parent == w).long().cumsum(1) - 1
        want = order[:, w].gather(1, place.clamp(min=0))
        assert torch.equal(out.token.long()[out.parent == w], want[out.parent == w])
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ refusals
def test_tensors_on_another_gpu_than_the_context(B, ctx):
    assert ctx.device == 0
    other = C.c_void_p(ctx.value)
    other.device = 1
    z, rows, buf, out = torch.zeros((4, 10), device="cuda"), B.LogitBuffers(4, 3), B.DistillBuffers(4), B.BeamBuffers(2, 2)
    for call in (lambda: B.mlmc_top_logits(other, z, None, 1.0, rows), lambda: B.mlmc_distill(other, z, rows, 1.0, True, None, buf, None),
                 lambda: B.mlmc_distill_grad(other, z, rows, 1.0, True, None, buf, z),
                 lambda: B.mlmc_beam_select(other, rows, 10, 2, 1.0, z[0, :4], None, -1, out),
                 lambda: B.mlmc_beam_reorder(other, out.parent, B.BeamStates([z], 2))):
        with pytest.raises(ValueError, match="GPU"):
            call()
