"""The losses, the clipping and the policy's steps of recurrent_lm.py as a training loop calls them: losses under a scale that the backward pass brings, rows that no sequence has,
gradients of any strides, and whole steps against PyTorch's own operations in 64 bits."""
import copy
import math

import pytest
import torch

import test_lm_distill
import test_lm_policy
from lm_helpers import EPS32, TORCH, close, randn
from paper_2108_11033_amd import recurrent_lm as rl
from test_recurrent_lm import _plain_logits

SCALE = 65536.0


# ------------------------------------------------------------------------------------------- losses under a scale
# Gradients whose sizes lie far below the type's smallest number before the scale: a weight of 2^-13 times a share of 2^-12 or less, in fp16 2^-24.  The bounds are those of
# gradients with the scale in their weights (a power of two, and another factor: one rounding more of the weight).
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("factor", [SCALE, -3000.0])
def test_policy_gradients_take_the_scale_before_they_are_rounded(dtype, factor, monkeypatch):
    monkeypatch.setattr(test_lm_policy, "HIGH", test_lm_policy.LOW)
    N, V, tau, kl = 40, 4099, 2.0, 0.05
    z, ids, old, ref, A, w = test_lm_policy.operands(dtype, N, V, tau, 0, 0, 17)
    w = (w * 2.0 ** -13).contiguous()
    w[7], ids[9] = 0, -1
    z.requires_grad_()
    loss, logp = rl.PolicyLoss.apply(z, ids, old, ref, A, w, tau, test_lm_policy.LOW, kl)
    (loss * factor).backward()
    wl, wp, _, sl, sp, _ = test_lm_policy.reference(z.detach(), ids, tau, old, ref, A, w, kl)
    wdz, sdz = test_lm_policy.reference(z.detach(), ids, tau, old, ref, A, w.double() * factor, kl)[2::3]
    close(logp, wp, sp, "f32", "logp")
    assert abs(float(loss.detach()) - float(wl.sum())) <= float(sl.sum()) + N * EPS32 * float(wl.abs().sum())
    close(z.grad, wdz, sdz + EPS32 * wdz.abs(), dtype, "dz")
    assert z.grad.dtype == TORCH[dtype] and not z.grad[7].any() and not z.grad[9].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_policy_gradients_without_weights_twice_and_of_nothing(dtype):
    N, V = 12, 50
    z, ids, old, _, A, _ = test_lm_policy.operands(dtype, N, V, 1.0, 0, 0, 19)
    z.requires_grad_()
    of = lambda weight: rl.PolicyLoss.apply(z, ids, old, None, A, weight, 1.0, 0.2, 0.0)[0]
    loss = of(None)
    one, = torch.autograd.grad(loss, z, retain_graph=True)
    twice, = torch.autograd.grad(loss, z, torch.tensor(2.0, device="cuda"), retain_graph=True)
    none, = torch.autograd.grad(loss, z, torch.tensor(0.0, device="cuda"))
    assert torch.equal(one, torch.autograd.grad(of(torch.ones(N, device="cuda")), z)[0]) and not none.any()
    large = one.abs() > 2.0 ** -13                                           # (below, fp16 rounds to a fixed step)
    assert large.any() and torch.equal(twice[large], 2 * one[large])


@pytest.mark.gpu
def test_logits_that_are_others_by_the_backward_pass_are_refused():
    """What it forms the gradient of 16-bit logits from are the logits that the loss was formed from, or none."""
    z, ids, old, _, A, _ = test_lm_policy.operands("f16", 12, 50, 1.0, 0, 0, 19)
    z.requires_grad_()
    loss = rl.PolicyLoss.apply(z, ids, old, None, A, None, 1.0, 0.2, 0.0)[0]
    with torch.no_grad():
        z.add_(1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("factor", [SCALE, -3000.0])
def test_distillation_gradients_take_the_scale_before_they_are_rounded(dtype, factor):
    N, V, k, tau = 40, 4099, 16, 2.0
    z, top, ids, w = test_lm_distill._operands(dtype, N, V, k, 0, 0, 23)
    w = (w * 2.0 ** -13).contiguous()
    w[7], ids[9] = 0, -1
    z.requires_grad_()
    loss = rl.DistillTopK.apply(z, top, ids, tau, w)
    (loss * factor).backward()
    want, _, sl, _ = test_lm_distill.reference(z.detach(), top, ids, tau, w)
    _, wdz, _, sdz = test_lm_distill.reference(z.detach(), top, ids, tau, w.double() * factor)
    assert abs(float(loss.detach()) - float(want.sum())) <= float(sl.sum()) + N * EPS32 * float(want.abs().sum())
    close(z.grad, wdz, sdz + EPS32 * wdz.abs(), dtype, "dz")
    assert z.grad.dtype == TORCH[dtype] and not z.grad[7].any() and not z.grad[9].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_losses_captured_with_their_gradients(dtype):
    """Both losses, forward and backward, in a graph: every replay, on new logits and under a new scale, gives what eager calls give."""
    N, V, k = 30, 5000, 8
    z, ids, old, ref, A, w = test_lm_policy.operands(dtype, N, V, 1.0, 0, 0, 29)
    _, top, lists, _ = test_lm_distill._operands(dtype, N, V, k, 0, 0, 31)
    scale = torch.ones((), device="cuda")
    z.requires_grad_()

    def step():
        loss, logp = rl.PolicyLoss.apply(z, ids, old, ref, A, w, 1.0, 0.2, 0.05)
        other = rl.DistillTopK.apply(z, top, lists, 2.0, w)
        return [loss.detach(), logp, other.detach(), *torch.autograd.grad(loss, z, scale), *torch.autograd.grad(other, z, scale)]

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        captured = step()
    for seed in range(4):
        with torch.no_grad():
            z.copy_(randn(seed, N, V))
            scale.fill_([1.0, SCALE, -3.0, 0.5][seed])
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(captured, step()):
            assert torch.equal(got, want), seed
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- rows that no sequence has
@pytest.mark.gpu
@pytest.mark.parametrize("first,end", [(0, 50), (3, 64), (10, 41)])
def test_the_delta_rule_leaves_zeros_where_no_sequence_is(first, end):
    """A batch that is padded to a size: outputs and gradients of the rows before the first sequence and behind the last are 0, whatever their operands, and the memory, held."""
    N, keys, heads, dk, dv = 64, 1, 2, 16, 24
    rows = [randn(i, N, *s) for i, s in enumerate([(keys, dk), (keys, dk), (heads, dv)])] + [-randn(5, N, heads).abs(), torch.rand(N, heads, device="cuda")]
    s0, starts = randn(6, 2, heads, dk, dv), torch.tensor([first, 30, end], device="cuda")
    dy, ds = randn(7, N, heads, dv), randn(8, 2, heads, dk, dv)

    def call(rows, s0, starts, dy):
        leaves = [t.clone().requires_grad_() for t in (*rows, s0)]
        y, s_last = rl.GatedDeltaRule.apply(*leaves, starts, dk ** -0.5, 1e-6)
        stale = [torch.full((n,), math.nan, device="cuda") for n in [N * keys * dk, N * heads * dv, N * heads] for _ in range(6)]
        del stale                                                            # what fresh tensors may find in their memory
        return [y, s_last, *torch.autograd.grad([y, s_last], leaves, [dy, ds])]

    inside = slice(first, end)
    want = call([t[inside] for t in rows], s0, starts - first, dy[inside])
    padded = [t.clone() for t in rows]
    for t in padded:
        t[:first], t[end:] = math.nan, math.nan
    dy[:first], dy[end:] = math.nan, math.nan
    stale = [torch.full((N * heads * dv,), math.nan, device="cuda") for _ in range(6)]
    del stale
    got = call(padded, s0, starts, dy)
    for name, a, b in zip(("y", "s_last", "dq", "dk", "dv", "ddecay", "dbeta", "ds0"), got, want):
        if a.shape == b.shape:
            assert torch.equal(a, b), name
        else:
            assert torch.equal(a[inside], b) and not a[:first].any() and not a[end:].any(), name


# ------------------------------------------------------------------------------------------- clipping
@pytest.mark.gpu
def test_one_parameter_is_clipped_too():
    p = torch.zeros(3, 4, device="cuda", requires_grad=True)
    p.grad = torch.full((3, 4), 2.0, device="cuda")
    norm = rl.clip_gradients(p, 1.0)
    assert abs(float(norm) - math.sqrt(48)) <= 6 * EPS32 * 7 and float((p.grad.double() - 1 / math.sqrt(12)).abs().max()) <= 12 * EPS32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_of_any_strides_are_clipped(dtype):
    """Gradients of transposed parameters, and parts of a wider buffer: each is clipped where it lies, and nothing around it."""
    buffer = randn(1, 20, 30).to(TORCH[dtype])
    around = buffer.clone()
    grads = [randn(2, 12, 7).to(TORCH[dtype]).t(), buffer[3:9, 5:20], randn(3, 2, 5, 6, 4).to(TORCH[dtype]).to(memory_format=torch.channels_last), randn(4, 33).to(TORCH[dtype])]
    before = [t.clone() for t in grads]
    parameters = []
    for t in grads:
        parameters.append(torch.zeros_like(t).requires_grad_())
        parameters[-1].grad = t
    norm = rl.clip_gradients(parameters, 0.5, unscale=0.25)
    want = 0.25 * math.sqrt(sum(float((t.double() ** 2).sum()) for t in before))
    assert abs(float(norm) - want) <= want * 6 * EPS32
    for p, t, b in zip(parameters, grads, before):
        assert p.grad is t
        clipped = b.double() * (0.25 * 0.5 / want)
        close(t, clipped, clipped.abs() * 10 * EPS32, dtype, f"{tuple(b.shape)}")
    around[3:9, 5:20] = buffer[3:9, 5:20]
    assert torch.equal(around, buffer)


def test_a_gradient_that_is_there_twice_is_refused():
    for shape in ((3, 4), (4, 3)):
        p = torch.zeros(4, 3).t() if shape == (3, 4) else torch.zeros(shape)
        p.requires_grad_().grad = torch.zeros_like(p)
        with pytest.raises(ValueError, match="twice"):
            rl.clip_gradients([p, p], 1.0)


# ------------------------------------------------------------------------------------------- steps of the policy
LENGTHS = [5, 0, 1, 22, 9, 0]                                                # two empty texts, one of a token
RATE, CLIP, KL, MOST, TEMPERATURE, EPOCHS = 1.0, 0.02, 0.1, 0.5, 1.5, 3


def _policy_operands(device):
    starts = [sum(LENGTHS[:i]) for i in range(len(LENGTHS) + 1)]
    gen = torch.Generator().manual_seed(12)
    model = rl.RecurrentLM(96, 64, 2, 4)
    return (model.to(device), starts, *(torch.randint(0, 96, (starts[-1],), generator=gen).to(device), torch.randn(starts[-1], generator=gen).to(device)))


def _plain_reinforce(model, starts, tokens, advantage):
    """Steps by the gradient in 64 bits: the losses, every step's ratios and the model after them.  Token t + 1 of a text is the word sampled after token t, whose advantage it has; every
    token counts 1 / N, a text's last one with a loss of 0."""
    model, N = copy.deepcopy(model).double(), len(tokens)
    rows = torch.tensor([t for a, b in zip(starts, starts[1:]) for t in range(a, b - 1)], device=tokens.device)
    losses, ratios, old = [], [], None
    for _ in range(EPOCHS):
        lp = torch.log_softmax(_plain_logits(model, tokens, starts)[rows] / TEMPERATURE, 1)[torch.arange(len(rows)), tokens[rows + 1]]
        old = lp.detach() if old is None else old
        r, d, A = torch.exp(lp - old), old - lp, advantage.double()[rows]
        loss = (KL * (torch.exp(d) - d - 1) - torch.minimum(r * A, r.clamp(1 - CLIP, 1 + CLIP) * A)).sum() / N
        model.zero_grad()
        loss.backward()
        norm = torch.sqrt(sum((p.grad ** 2).sum() for p in model.parameters()))
        with torch.no_grad():
            for p in model.parameters():
                p -= RATE * p.grad * min(1.0, MOST / float(norm))
        losses.append(float(loss.detach()))
        ratios.append((r.detach(), float(norm)))
    return losses, ratios, model


def test_the_policys_steps_do_what_they_are_there_for():
    """Of the 64-bit form alone: the steps leave the clipping's bounds on both sides, no ratio lies so near one that fp32 might see it on the other side, some norms are clipped."""
    _, ratios, _ = _plain_reinforce(*_policy_operands("cpu"))
    last, first = ratios[-1][0], ratios[0][0]
    assert torch.equal(first, torch.ones_like(first)) and bool((last > 1 + CLIP).any()) and bool((last < 1 - CLIP).any())
    for r, _ in ratios[1:]:
        assert min(float((r - 1 - CLIP).abs().min()), float((r - 1 + CLIP).abs().min())) > 1e-3 * CLIP
    assert any(norm > MOST for _, norm in ratios)


@pytest.mark.gpu
def test_the_policys_steps_against_plain_operations(monkeypatch):
    """With steps by the gradient itself in place of the optimizer's, which divides what is off by what is left of it."""
    monkeypatch.setattr(torch.optim, "Adam", lambda parameters, lr: torch.optim.SGD(parameters, lr=lr))
    model, starts, tokens, advantage = _policy_operands("cuda")
    before = {n: p.detach().double().clone() for n, p in model.named_parameters()}
    want, ratios, after = _plain_reinforce(model, starts, tokens, advantage)
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = rl.reinforce(model, [(tokens, seq, advantage)], rate=RATE, temperature=TEMPERATURE, clip=CLIP, kl=KL, max_norm=MOST, epochs=EPOCHS)
    # two layers of fp32 arithmetic: logits off by less than 1e-4 of their size, gradients by less than 2e-4 of theirs in the 2-norm, and so what each of the steps adds; a loss
    # is a mean of advantages times ratios that are off by as much as the logits
    logits = float(_plain_logits(after, tokens, starts).detach().abs().max())
    assert len(got) == EPOCHS
    for a, b in zip(got, want):
        assert abs(a - b) <= 1e-4 * (1 + logits / TEMPERATURE) * float(advantage.abs().mean()), (got, want)
    for (n, p), (_, q) in zip(model.named_parameters(), after.named_parameters()):
        moved = q.detach() - before[n]
        assert float((p.detach().double() - q.detach()).norm()) <= EPOCHS * (2e-4 * float(moved.norm()) + EPS32 * float(q.detach().norm())) + 1e-9, n
    assert any(float((q.detach() - before[n]).norm()) > 1e-2 for n, q in after.named_parameters())
