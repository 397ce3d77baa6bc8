"""A training step of a layer with matrix states: norm, gated delta rule, head, clipped policy loss, gradients clipped by their norm, in the functions of recurrent_lm.py, against
PyTorch's own operations in 64 bits; captured and replayed; and the served steps that go on from its states."""
import pytest
import torch

from gdr_reference import run as reference

STARTS = [0, 70, 70, 71, 200]
V, H, KEY_HEADS, HEADS, DK, DV = 96, 64, 2, 4, 16, 24
EPS, SCALE = 1e-6, 16 ** -0.5


def _parameters(seed=0):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *shape: (torch.randn(shape, generator=gen) / shape[-1] ** 0.5).cuda().requires_grad_()
    return dict(embedding=rand(V, H), gamma=torch.ones(H, device="cuda", requires_grad=True), beta=torch.zeros(H, device="cuda", requires_grad=True), q=rand(KEY_HEADS * DK, H),
                k=rand(KEY_HEADS * DK, H), v=rand(HEADS * DV, H), gates=rand(2 * HEADS, H), s0=rand(len(STARTS) - 1, HEADS, DK, DV), out=rand(H, HEADS * DV), head=rand(V, H))


def _batch():
    gen = torch.Generator().manual_seed(5)
    tokens, words = (torch.randint(0, V, (STARTS[-1],), generator=gen).cuda() for _ in range(2))
    words[torch.tensor([69, 70, 199])] = -1                                  # no word follows a text's last
    rows = lambda: torch.randn(STARTS[-1], generator=gen).cuda()
    return tokens, words, -4.6 + 0.1 * rows(), -4.6 + 0.1 * rows(), rows(), torch.full((STARTS[-1],), 1 / STARTS[-1], device="cuda")


def _step(p, batch, seq):
    from paper_2108_11033_amd.recurrent_lm import GatedDeltaRule, LayerNorm, PolicyLoss, clip_gradients
    tokens, words, old, ref, advantage, weight = batch
    N = tokens.numel()
    x = p["embedding"][tokens]
    n = LayerNorm.apply(x, p["gamma"], p["beta"])
    g = n @ p["gates"].t()
    y, s_last = GatedDeltaRule.apply((n @ p["q"].t()).view(N, KEY_HEADS, DK), (n @ p["k"].t()).view(N, KEY_HEADS, DK), (n @ p["v"].t()).view(N, HEADS, DV),
                                     -torch.nn.functional.softplus(g[:, :HEADS] - 2), torch.sigmoid(g[:, HEADS:]), p["s0"], seq, SCALE, EPS)
    logits = (x + y.reshape(N, -1) @ p["out"].t()) @ p["head"].t()
    loss, logp = PolicyLoss.apply(logits, words, old, ref, advantage, weight, 1.0, 0.2, 0.05)
    loss.backward()
    return loss.detach(), logp, s_last, clip_gradients(p.values(), 0.05)


def _plain(p, batch):
    q = {n: t.detach().double().requires_grad_() for n, t in p.items()}
    tokens, words, old, ref, advantage, weight = (t.double() if t.is_floating_point() else t for t in batch)
    N = tokens.numel()
    x = q["embedding"][tokens]
    n = torch.nn.functional.layer_norm(x, (H,), q["gamma"], q["beta"], 1e-5)
    g = n @ q["gates"].t()
    unit = lambda t: t / torch.sqrt((t * t).sum(-1, keepdim=True) + EPS)
    Q, K = (unit((n @ q[i].t()).view(N, KEY_HEADS, DK)).repeat_interleave(HEADS // KEY_HEADS, 1) for i in ("q", "k"))
    vs, a, b = (n @ q["v"].t()).view(N, HEADS, DV), torch.exp(-torch.nn.functional.softplus(g[:, :HEADS] - 2)), torch.sigmoid(g[:, HEADS:])
    ys, lasts = [], []
    for i, (first, end) in enumerate(zip(STARTS, STARTS[1:])):
        S = q["s0"][i]
        for t in range(first, end):
            S = S * a[t, :, None, None]
            S = S + K[t][:, :, None] * (b[t][:, None] * (vs[t] - (K[t][:, :, None] * S).sum(1)))[:, None, :]
            ys.append(SCALE * (Q[t][:, :, None] * S).sum(1))
        lasts.append(S)
    logits = (x + torch.stack(ys).reshape(N, -1) @ q["out"].t()) @ q["head"].t()
    said = words >= 0
    lp = torch.log_softmax(logits, 1).gather(1, words.clamp(min=0)[:, None])[:, 0]
    r, d = torch.exp(lp - old), ref - lp
    loss = (torch.where(said, 0.05 * (torch.exp(d) - d - 1) - torch.minimum(r * advantage, r.clamp(0.8, 1.2) * advantage), 0.0) * weight).sum()
    loss.backward()
    norm = torch.sqrt(sum((t.grad ** 2).sum() for t in q.values())).detach()
    return loss.detach(), torch.where(said, lp, 0.0).detach(), torch.stack(lasts).detach(), norm, {n: t.grad * min(1.0, 0.05 / float(norm)) for n, t in q.items()}


@pytest.mark.gpu
def test_a_training_step():
    p, batch, seq = _parameters(), _batch(), torch.tensor(STARTS, dtype=torch.int32, device="cuda")
    loss, logp, s_last, norm = _step(p, batch, seq)
    want = _plain(p, batch)
    # three products and a recurrence in fp32 one after another, of 64 to 200 terms: below 1e-4 of the values' size
    near = lambda a, b: float((a.detach().double() - b).norm()) <= 1e-4 * float(b.norm())
    assert near(loss, want[0]) and near(logp, want[1]) and near(s_last, want[2]) and near(norm[0], want[3])
    for n, t in p.items():
        assert float((t.grad.double() - want[4][n]).norm()) <= 2e-4 * float(want[4][n].norm()) + 1e-9, n
    assert float(norm) > 0.05 and abs(float(torch.sqrt(sum((t.grad.double() ** 2).sum() for t in p.values()))) - 0.05) <= 1e-6


@pytest.mark.gpu
def test_replays_of_the_operators_of_a_step():
    """The recurrence in both directions, the loss and the clipping captured into one graph: every replay, on new inputs too, gives what an eager call gives."""
    import paper_2108_11033_amd as g
    N, nseq, keys, values = STARTS[-1], len(STARTS) - 1, KEY_HEADS * DK, HEADS * DV
    seq = torch.tensor(STARTS, dtype=torch.int32, device="cuda")
    empty = lambda *s: torch.empty(s, device="cuda")
    scratch = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device="cuda")
    q, k, v, decay, beta, s0, z = empty(N, keys), empty(N, keys), empty(N, values), empty(N, HEADS), empty(N, HEADS), empty(nseq, HEADS, DK, DV), empty(N, values)
    ids = torch.zeros(N, dtype=torch.int32, device="cuda")
    old, advantage = empty(N), empty(N)

    def fill(seed):
        gen = torch.Generator("cuda").manual_seed(seed)
        for t in (q, k, v, s0, old, advantage):
            t.normal_(generator=gen)
        decay.uniform_(-0.5, 0, generator=gen)
        beta.uniform_(0, 1, generator=gen)
        old.mul_(0.1).sub_(4.6)
        ids.random_(0, values, generator=gen)

    def call(o, stream):
        # the outputs serve as logits, so that the loss' gradient is the recurrence's
        g.gdr_sequence(q, k, v, "f32", keys, keys, values, decay, beta, HEADS, s0, seq, nseq, N, HEADS, KEY_HEADS, DK, DV, SCALE, EPS, o["y"], values, o["s_last"], o["states"], o["ws"],
                       stream)
        g.policy_loss(o["y"], "f32", values, ids, N, values, o["loss"], o["logp"], o["dz"], values, o["room"], old_logp=old, advantage=advantage, stream=stream)
        g.gdr_sequence_backward(q, k, v, "f32", keys, keys, values, decay, beta, HEADS, s0, seq, nseq, N, HEADS, KEY_HEADS, DK, DV, SCALE, EPS, o["states"], o["dz"], values, None, o["dq"],
                                keys, o["dk"], keys, o["dv"], values, o["ddecay"], o["dbeta"], HEADS, o["ds0"], o["ws"], stream)
        lst = g.GradList([o[n] for n in ("dq", "dk", "dv", "ddecay", "dbeta", "ds0")])
        g.grad_clip(lst, 0.5, 1.0, o["norm"], o["sums"], stream)

    def outputs():
        lst = g.GradList([empty(N, keys), empty(N, keys), empty(N, values), empty(N, HEADS), empty(N, HEADS), empty(nseq, HEADS, DK, DV)])
        return dict(y=empty(N, values), s_last=empty(nseq, HEADS, DK, DV), loss=empty(N), logp=empty(N), dz=empty(N, values), dq=empty(N, keys), dk=empty(N, keys), dv=empty(N, values),
                    ddecay=empty(N, HEADS), dbeta=empty(N, HEADS), ds0=empty(nseq, HEADS, DK, DV), norm=empty(1), states=scratch(g.gdr_states(N, nseq, HEADS, DK, DV)),
                    ws=scratch(g.gdr_workspace(N, nseq, HEADS, KEY_HEADS, DK, DV)), room=scratch(g.policy_loss_workspace(N, values)), sums=scratch(lst.workspace))
    results = ["y", "s_last", "loss", "logp", "dz", "dq", "dk", "dv", "ddecay", "dbeta", "ds0", "norm"]
    fill(0)
    eager, captured, beside = outputs(), outputs(), outputs()
    call(eager, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        call(captured, stream)
    side = torch.cuda.Stream()
    for seed in range(4):
        fill(seed)
        torch.cuda.synchronize()
        graph.replay()
        call(beside, side)                                                   # two calls at once, each with its own buffers
        call(eager, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for n in results:
            assert torch.equal(captured[n], eager[n]) and torch.equal(beside[n], eager[n]), (seed, n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(captured[n], eager[n]) for n in results)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_layers_gradients_in_16_bits(dtype):
    """Parameters of other types than the kernels read, rows that are no whole tensors, gradients in the operands' types."""
    from paper_2108_11033_amd.recurrent_lm import GatedDeltaRule
    gen = torch.Generator("cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)
    N = STARTS[-1]
    both = rand(N, 2 * KEY_HEADS, DK).to(dtype)
    leaves = [both[:, :KEY_HEADS].detach().requires_grad_(), both[:, KEY_HEADS:].detach().requires_grad_(), rand(N, HEADS, DV).to(dtype).requires_grad_(),
              (-rand(N, HEADS).abs()).to(dtype).requires_grad_(), torch.rand(N, HEADS, device="cuda", generator=gen).requires_grad_(), rand(4, HEADS, DK, DV).requires_grad_()]
    seq = torch.tensor(STARTS, device="cuda")                                # (64 bits)
    y, s_last = GatedDeltaRule.apply(*leaves, seq, SCALE, EPS)
    dy, ds_last = torch.randn_like(y), torch.randn_like(s_last)
    grads = torch.autograd.grad([y, s_last], leaves, [dy, ds_last])
    name = "f16" if dtype == torch.float16 else "bf16"
    flat = lambda t: t.detach().reshape(N, -1)
    want = reference(flat(leaves[0]), flat(leaves[1]), flat(leaves[2]), leaves[3].detach().float(), leaves[4].detach(), leaves[5].detach(), STARTS, HEADS, KEY_HEADS, DK, DV, SCALE, EPS,
                     dy=flat(dy), ds_last=ds_last, dtype=name)
    for t, leaf, n in zip(grads, leaves, ("dq", "dk", "dv", "ddecay", "dbeta", "ds0")):
        assert t.dtype == leaf.dtype and t.shape == leaf.shape
        value, slack = (x.reshape(t.shape) for x in want[n])
        half = torch.finfo(t.dtype).eps / 2
        assert bool(((t.double() - value).abs() <= half * value.abs() * 1.01 + slack + 2.0 ** -25).all()), n


@pytest.mark.gpu
def test_refusals_of_the_functions():
    from paper_2108_11033_amd.recurrent_lm import GatedDeltaRule, PolicyLoss, clip_gradients
    N, z = 8, lambda *s: torch.zeros(s, device="cuda")
    good = [z(N, 2, 4), z(N, 2, 4), z(N, 4, 3), z(N, 4), z(N, 4), z(1, 4, 4, 3), torch.tensor([0, N], device="cuda"), 1.0, 0.0]
    for at, bad in ((0, z(N, 2, 5)), (1, z(N, 2, 4).half()), (2, z(N, 3, 3)), (2, z(N - 1, 4, 3)), (3, z(N, 3)), (4, z(N, 2)), (5, z(1, 4, 3, 4)), (5, z(2, 4, 4, 3)), (6, torch.zeros(2, device="cuda")),
                    (2, torch.zeros(N, 4, 3))):
        with pytest.raises(ValueError):
            GatedDeltaRule.apply(*[bad if i == at else t for i, t in enumerate(good)])
    ids = torch.zeros(N, dtype=torch.int64, device="cuda")
    loss = [z(N, 10), ids, None, None, z(N), z(N), 1.0, 0.2, 0.0]
    for at, bad in ((0, z(N, 10, 1)), (1, z(N)), (1, ids[:3]), (2, z(3)), (4, z(N + 1)), (5, z(1)), (4, torch.zeros(N))):
        with pytest.raises(ValueError):
            PolicyLoss.apply(*[bad if i == at else t for i, t in enumerate(loss)])
    p = torch.zeros(4, requires_grad=True)
    p.grad = torch.zeros(4)
    with pytest.raises(ValueError):
        clip_gradients([p], 1.0)


@pytest.mark.gpu
def test_words_beyond_32_bits_are_padding():
    from paper_2108_11033_amd.recurrent_lm import PolicyLoss
    logits = torch.randn(4, 10, device="cuda", requires_grad=True)
    ids = torch.tensor([3, -1, (1 << 32) + 3, 10], device="cuda")
    loss, logp = PolicyLoss.apply(logits, ids, None, None, torch.ones(4, device="cuda"), torch.ones(4, device="cuda"), 1.0, 0.2, 0.0)
    loss.backward()
    assert float(loss.detach()) == -1.0 and logp[0] != 0 and not logp[1:].any() and logits.grad[0].any() and not logits.grad[1:].any()


@pytest.mark.gpu
def test_training_of_the_model_runs():
    from paper_2108_11033_amd.recurrent_lm import RecurrentLM, distill, reinforce
    model = RecurrentLM(V, H, 1, 0).cuda()
    seq = torch.tensor(STARTS, dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (STARTS[-1],), device="cuda")
    losses = reinforce(model, [(tokens, seq, torch.randn(STARTS[-1], device="cuda"))], epochs=2)
    losses += distill(model, model, [(tokens, seq)], max_norm=1.0)
    assert len(losses) == 3 and all(x == x and abs(x) < 100 for x in losses)
