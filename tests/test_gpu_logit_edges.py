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


# ------------------------------------------------------------------------------------------ the rest, wherever it lies
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N, V, k", [(3, 1 << 20, 1024), (3, 1 << 20, 512), (4, 262_147, 700), (40, 131_075, 128), (330, 131_075, 128), (330, 262_147, 128),
                                     (300, 40_000, 300), (20, 9001, 1000), (500, 3001, 60), (330, 1244, 64), (300, 398, 99)])
def test_a_rest_of_a_few_logits(B, ctx, N, V, k, dtype):
    """All but the message and n <= 12 logits of 0 is -inf, or so low that it does not count: one of them that is lost, or taken twice, changes
    the rest by 1 / 12.  They lie at both ends of the row, around the borders of sections, and anywhere.  rest = ln n - max: a sum of n
    ones, an exponential or two on the way, the rounding of the result."""
    g = torch.Generator(device="cuda").manual_seed(V + k)
    for low, ld, offset in ((-INF, V + 5, 3), (-200.0, V, 0)):
        z = rows_of(V, N, dtype, 1, ld=ld, offset=offset)
        z.fill_(low)
        place = torch.rand((N, V), generator=g, device="cuda")
        border = torch.tensor([b * V // n + d for n in (2, 4, 8) for b in range(1, n) for d in (-9, -1, 0, 1, 8)], device="cuda").clamp(0, V - 1)
        few = torch.cat([torch.tensor([0, 1, V - 2, V - 1], device="cuda").expand(N, 4),
                         border[torch.randint(0, border.numel(), (N, 4), generator=g, device="cuda")],
                         torch.randint(0, V, (N, 4), generator=g, device="cuda")], 1)
        place.scatter_(1, few, -1.0)                                           # the message lies anywhere else
        sent = place.topk(k, 1).indices
        z.scatter_(1, few, torch.zeros((N, 12), dtype=dtype, device="cuda"))
        z.scatter_(1, sent, (20.0 + 4.0 * torch.rand((N, k), generator=g, device="cuda")).to(dtype))
        n = (z == 0).sum(1)
        out = B.LogitBuffers(N, k)
        B.mlmc_top_logits(ctx, z, None, 1.0, out)
        assert (out.count == k).all()
        assert torch.equal(out.idx.long().sort(1).values, sent.sort(1).values)
        want = n.double().log() - z.max(1).values.double()
        assert ((out.rest.double() - want).abs() <= (12 + 4 * 4) * U + 2 * U * want.abs()).all()
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


@pytest.mark.parametrize("N, V, k, dtype", [(400, 150_001, 50, torch.float32), (310, 262_147, 128, torch.float32), (300, 262_147, 256, torch.float32),
                                            (600, 160_001, 512, torch.bfloat16), (297, 1 << 20, 20, torch.bfloat16), (100, 1 << 20, 500, torch.bfloat16)])
def test_top_logits_of_many_very_long_rows(B, ctx, N, V, k, dtype):
    """A block per row, of groups of up to 16 trips, or sections of it."""
    check_top(B, ctx, rows_of(V, N, dtype, V + k), k, 1.0)
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ rows that are held in shared memory
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("V, k", [(66_001, 300), (131_075, 1024), (131_075, 257)])
def test_long_messages_of_rows_that_are_held(B, ctx, V, k, rest):
    """fp32 rows that clusters hold between their two passes, with more entries than the cluster's blocks have threads; the next row's
    message is asked for while this one's is in use, whatever its count says."""
    N = 605
    z = rows_of(V, N, torch.float32, 71, scale=2.0)
    t = torch.randn((N, V), generator=torch.Generator(device="cuda").manual_seed(72), device="cuda") * 1.5
    val, idx = t.topk(k, 1)
    behind = torch.cat([a.double().scatter(1, i, -INF).logsumexp(1) for a, i in zip(t.split(100), idx.split(100))])
    del t
    mix = torch.rand((N, k), generator=torch.Generator(device="cuda").manual_seed(73), device="cuda").argsort(1)      # in any order
    msg = B.LogitBuffers.of(idx.gather(1, mix).int().contiguous(), val.gather(1, mix).contiguous(),
                            torch.full((N,), k, dtype=torch.int32, device="cuda"), (behind - val[:, 0].double()).float())
    row = torch.arange(N, device="cuda")
    wrong = (row % 50 == 7) | (row == 0) | (row == N - 1)
    msg.count[wrong] = torch.where(row % 2 == 0, -1, k + 1)[wrong].int()
    msg.count[row % 50 == 8] = 0
    msg.count[row % 50 == 9] = 256
    buf, grad = B.DistillBuffers(N), torch.full((N, V), 7.0, device="cuda")
    B.mlmc_distill(ctx, z, msg, 1.0, rest, None, buf, grad)
    assert B.mlmc_get_status(ctx) == B.MLMC_ERR_ARG
    assert torch.isnan(buf.loss[wrong]).all() and torch.isnan(grad[wrong]).all()
    assert not torch.isnan(buf.loss[~wrong]).any() and not torch.isnan(grad[~wrong]).any()
    assert (buf.loss[row % 50 == 8] == 0).all() and (grad[row % 50 == 8] == 0).all()
    some = torch.tensor([1, 6, 8, 9, 10, 300, 359, 602, 603], device="cuda")
    loss, want, loss_off, off = distill_reference(z[some], messages_of(B, msg, some), 1.0, rest, None)
    assert ((buf.loss[some].double().cpu() - loss).abs() <= loss_off).all()
    assert ((grad[some].double() - want).abs() <= off + (want.abs() + off) * U + 1e-37).all()
    kept = z.clone()
    B.mlmc_distill(ctx, z, msg, 1.0, rest, None, buf, z)                       # over the logits
    assert torch.equal(bits(z)[~wrong], bits(grad)[~wrong]) and torch.isnan(z[wrong]).all()
    assert B.mlmc_get_status(ctx) == B.MLMC_ERR_ARG
    B.mlmc_distill(ctx, kept, msg, 1.0, rest, None, buf, None)                 # the loss by itself, the gradient by itself
    assert B.mlmc_get_status(ctx) == B.MLMC_ERR_ARG
    B.mlmc_distill_grad(ctx, kept, msg, 1.0, rest, None, buf, grad)
    assert torch.isnan(grad[wrong]).all()
    assert ((grad[some].double() - want).abs() <= off + (want.abs() + off) * U + 1e-37).all()
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ padding
@pytest.mark.parametrize("dtype", DTYPES)
def test_two_call_gradient_of_every_row_of_a_padded_batch(B, ctx, dtype):
    V, N = 9000, 40
    z = rows_of(V, N, dtype, 4)
    count = torch.arange(N, device="cuda") % 4 * 5                               # 0, 5, 10, 15 of 15 places
    msg = message(B, rows_of(V, N, torch.float32, 5), 15, 1.0, count)
    weight = torch.rand(N, device="cuda")
    loss, want, loss_off, off = distill_reference(z, msg, 1.0, True, weight)
    z[count == 0] = float("nan")
    buf, grad = B.DistillBuffers(N), torch.full_like(z, 7.0)
    B.mlmc_distill(ctx, z, msg, 1.0, True, weight, buf, None)
    B.mlmc_distill_grad(ctx, z, msg, 1.0, True, weight, buf, grad)
    assert ((buf.loss.double().cpu() - loss).abs() <= loss_off).all() and (buf.loss[count == 0] == 0).all()
    assert ((grad.double() - want).abs() <= off + (want.abs() + off) * torch.finfo(dtype).eps / 2 + 1e-37).all() and (grad[count == 0] == 0).all()
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ the temperature's range
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1e-3, 0.05, 30.0, 1e3])
def test_distillation_at_the_ends_of_the_temperature(B, ctx, T, dtype, rest):
    for N, V, k in ((5, 400, 30), (3, 8193, 64), (2, 60_001, 40)):
        z = rows_of(V, N, dtype, V, scale=2.0)
        t = z.float() * 0.7 + rows_of(V, N, torch.float32, V + 1, scale=1.0)
        check_distill(B, ctx, z, message(B, t, k, T), T, rest, torch.rand(N, device="cuda") + 0.1)
    # logits as far apart as the temperature makes them look near, and as near as it makes them look far
    z = (rows_of(3000, 4, torch.float32, 9, scale=2.0) * T).to(dtype)
    t = z.float() + rows_of(3000, 4, torch.float32, 10, scale=0.5) * T
    check_distill(B, ctx, z, message(B, t, 40, T), T, rest)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1e-3, 0.05, 30.0, 1e3])
def test_ends_of_the_type_at_the_ends_of_the_temperature(B, ctx, T, dtype):
    V, lowest = 3000, torch.finfo(dtype).min
    z = rows_of(V, 6, dtype, 9, scale=2.0)
    t = rows_of(V, 6, torch.float32, 10, scale=2.0)
    t[:, :60] += 20.0                       # messages of the first 60 indices
    z[0, 100:] = lowest                     # masked with the type's lowest value
    z[1, 100:] = -INF                       # masked with -inf: probability 0
    z[2] = lowest                           # all equal
    z[3, 7] = torch.finfo(dtype).max / max(2.0, 2.0 * T)   # one above everything: a loss of nearly T times that, below what fp32 has
    z[4, 60:] -= 300.0
    msg = message(B, t, 40, T)
    check_distill(B, ctx, z, msg, T, True)
    check_distill(B, ctx, z, msg, T, False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [30.0, 100.0, 1e3])
@pytest.mark.parametrize("N, V, k", [(300, 400, 30), (7, 50_257, 64), (40, 131_072, 100)])
def test_small_losses_keep_their_digits_at_high_temperatures(B, ctx, N, V, k, T, dtype):
    """The bound of the test at lower temperatures, which says where its terms come from."""
    z = rows_of(V, N, dtype, 61, scale=2.0)
    t = z.float() + 0.02 * T * rows_of(V, N, torch.float32, 62, scale=1.0)
    msg = message(B, t, k, T)
    buf = B.DistillBuffers(N)
    B.mlmc_distill(ctx, z, msg, T, True, None, buf, None)
    eps = sum_tolerance(V)
    x = z.double() / T
    ln_p = x - torch.logsumexp(x, 1, keepdim=True)
    sent = torch.zeros((N, V), dtype=torch.bool, device="cuda").scatter_(1, msg.idx.long(), True)
    ln_p = torch.cat([ln_p.gather(1, msg.idx.long()), torch.logsumexp(torch.where(sent, -INF, ln_p), 1, keepdim=True)], 1)
    ln_q = torch.log_softmax(torch.cat([msg.val.double() / T, msg.val[:, :1].double() / T + msg.rest[:, None].double()], 1), 1)
    q, apart = ln_q.exp(), (ln_q.exp() - ln_p.exp()).abs()
    want = T * T * (q * (ln_q - ln_p)).sum(1)
    spread = (ln_q.max(1).values - ln_q.min(1).values)
    off = T * T * (2 * eps * apart[:, -1] + 2 * U * apart.sum(1)) + want * (2 * eps + (24 + 6 * spread) * U) + T * T * eps * eps
    assert float(want.max()) < 0.05 * T * T
    assert ((buf.loss.double() - want).abs() <= off).all(), ((buf.loss.double() - want).abs() / off).max()
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


# ------------------------------------------------------------------------------------------ states that grow
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("W", [1, 4, 5])
def test_states_that_grow_by_a_token(B, ctx, W, in_place):
    """One table of states for a whole search: heads first, tokens first, a size of one, a part of a larger buffer."""
    Bn, room = 3, 19
    n = Bn * W
    g = torch.Generator(device="cuda").manual_seed(W)

    def caches():
        def fill(shape, dtype):
            return torch.randint(-100, 100, shape, generator=g, device="cuda").to(dtype)
        return [fill((n, 3, room, 24), torch.bfloat16), fill((n, 1, room, 7), torch.float32), fill((n, 5, room, 1), torch.uint8),
                fill((2, n, 3, room, 8), torch.bfloat16)[1], fill((n, 6, room, 16), torch.float32)[:, 2:4], fill((n, 2, room + 4, 3), torch.bfloat16)[:, :, 2:2 + room]]
    src = caches()
    dst = src if in_place else caches()
    states = B.BeamStates(src if in_place else list(zip(src, dst)), W, tokens=2)
    text = torch.randint(0, 1000, (n, room), generator=g, device="cuda")
    lines = B.BeamStates([text], W, tokens=1)
    for length in (1, 2, 3, 8, 9, room, 5, 0):
        parent = torch.randint(0, W, (Bn, W), generator=g, device="cuda").int()
        at = (torch.arange(Bn, device="cuda")[:, None] * W + parent).reshape(-1).long()
        want = [d.clone() for d in dst]
        for x, y in zip(src, want):
            y[:, :, :length] = x[at][:, :, :length]
        want_text = torch.cat([text[at][:, :length], text[:, length:]], 1)
        B.mlmc_beam_reorder(ctx, parent, states.first(length))
        B.mlmc_beam_reorder(ctx, parent, lines.first(length))
        assert all(torch.equal(x, y) for x, y in zip(dst, want)) and torch.equal(text, want_text)
    assert B.mlmc_get_status(ctx) == B.MLMC_OK


def test_tokens_that_cannot_be_moved(B, ctx):
    x = torch.zeros((4, 2, 10, 8), device="cuda")
    states = B.BeamStates([x, torch.zeros((4, 3, 12, 8), device="cuda")], 2, tokens=2)
    for bad in (lambda: states.first(-1), lambda: states.first(11), lambda: B.BeamStates([x], 2).first(1), lambda: B.BeamStates([x], 2, tokens=0),
                lambda: B.BeamStates([x], 2, tokens=4), lambda: B.BeamStates([x[:, :, ::2]], 2, tokens=2), lambda: B.BeamStates([x.transpose(2, 3)], 2, tokens=2),
                lambda: B.BeamStates([x[..., :4]], 2, tokens=2)):
        with pytest.raises(ValueError):
            bad()


def test_states_that_share_memory(B, ctx):
    """A cache of keys and values side by side is two states; a swap, and one state twice, would race."""
    n, g = 6, torch.Generator(device="cuda").manual_seed(1)
    both = torch.randn((n, 4, 2, 9, 8), generator=g, device="cuda")
    parent = torch.tensor([[2, 0, 0], [1, 1, 2]], dtype=torch.int32, device="cuda")
    at = torch.tensor([2, 0, 0, 4, 4, 5], device="cuda")
    want = both.clone()
    want[:, :, :, :5] = both[at][:, :, :, :5]
    B.mlmc_beam_reorder(ctx, parent, B.BeamStates([both[:, :, 0], both[:, :, 1]], 3, tokens=2).first(5))
    assert torch.equal(both, want)
    x, y = torch.zeros((n, 8), device="cuda"), torch.zeros((n, 8), device="cuda")
    for bad in ([(x, y), (y, x)], [x, x], [(x, y), x], [(x, y), (torch.ones_like(x), y)]):
        with pytest.raises(ValueError, match="memory"):
            B.BeamStates(bad, 3)
    B.BeamStates([(x, y), (x, torch.zeros_like(x))], 3)
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
