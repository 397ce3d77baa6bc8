"""The operators of a recurrent language model around this library's pruned products: layer norm, the gated linear
recurrence, distillation from a teacher's top logits, and the rules applied to the logits of a served step.

A case names its kind ("norm", "glr", "glr_step", "distill", "rules"), its element type and the sizes of its kind.
`prepare` makes what a program has in hand (inputs, output buffers, workspaces); `run` is one pass through one operator.
Where `own` is false the pass is written in elementary torch operations in fp32, rounded once at the end.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
TAU = 2.0


def listed():
    return [
        # The norm in front of a layer of 1024 units at one frame for eight callers: the smallest call, where latency counts.
        dict(name="norm_step_b8", kind="norm", mode="fwd", dtype="f16", N=8, C=1024, pad=0),
        # The forward norm of a batch whose width no vector load divides.
        dict(name="norm_fwd_odd", kind="norm", mode="fwd", dtype="f32", N=5003, C=1999, pad=0),
        # The backward norm of a training step: 32768 tokens of 1024 features.
        dict(name="norm_bwd_large", kind="norm", mode="bwd", dtype="bf16", N=32768, C=1024, pad=0),
        # One token for 32 callers through a recurrence of 1024 units, after the gates' pruned product.
        dict(name="glr_step_b32", kind="glr_step", dtype="f16", H=1024, batch=32),
        # Eight utterances of 64 frames through a layer of 1024 units, inference.
        dict(name="glr_frames_b8", kind="glr", mode="fwd", dtype="f16", N=512, H=1024, nseq=8, pad=0),
        # A training step on 40 texts of different lengths packed one after another (one empty, one of a single token).
        dict(name="glr_train_packed", kind="glr", mode="train", dtype="f16", N=24007, H=1000, nseq=40, pad=0),
        # A training step on one long text: no parallelism but along the sequence and the units.
        dict(name="glr_train_long", kind="glr", mode="train", dtype="bf16", N=65536, H=1024, nseq=1, pad=0),
        # Distillation of a small classifier of frames: 1000 classes, the teacher's ten best, loss and gradient.
        dict(name="distill_classes", kind="distill", dtype="f32", N=1024, V=1000, k=10, grad=True, pad=0),
        # Distillation of a language model: 8192 tokens, 32768 words, the teacher's 64 best, loss and gradient.
        dict(name="distill_train", kind="distill", dtype="bf16", N=8192, V=32768, k=64, grad=True, pad=0),
        # A short batch over a large vocabulary of odd size: fewer rows than compute units, rows that are not aligned.
        dict(name="distill_few_rows", kind="distill", dtype="f16", N=24, V=131075, k=128, grad=True, pad=0),
        # One caller's next word: logits as the pruned head product leaves them, 200 words so far.
        dict(name="rules_step_b1", kind="rules", dtype="f32", V=32768, batch=1, L=200, columns=True, nbias=16, pad=0),
        # 64 callers with long histories (up to 4096 words), a large vocabulary, grammars and biases.
        dict(name="rules_b64", kind="rules", dtype="bf16", V=131072, batch=64, L=4096, columns=False, nbias=64, pad=0),
    ]


# ---------------------------------------------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """The same; half of them whole multiples of 64, the others as they fall."""
    n = _log(rng, lo, hi)
    return min(hi, max(lo, (n + 32) // 64 * 64)) if rng.random() < 0.5 else n


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= most:
            return c


def _draw(rng):
    kind = rng.choice(["norm", "norm", "glr", "glr", "glr_step", "distill", "distill", "rules"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 3, 8])
    if kind == "norm":
        return dict(kind=kind, mode=rng.choice(["fwd", "bwd"]), dtype=dtype, N=_log(rng, 1, 65536), C=_size(rng, 64, 8192), pad=pad)
    if kind == "glr":
        N = _log(rng, 1, 65536)
        return dict(kind=kind, mode=rng.choice(["fwd", "train"]), dtype=dtype, N=N, H=_size(rng, 32, 4096),
                    nseq=_log(rng, 1, max(1, min(64, N // 4))), pad=pad)
    if kind == "glr_step":
        return dict(kind=kind, dtype=dtype, H=_size(rng, 64, 8192), batch=_log(rng, 1, 64))
    if kind == "distill":
        V = _size(rng, 500, 152000)
        return dict(kind=kind, dtype=dtype, N=_log(rng, 1, 8192), V=V, k=_log(rng, 1, 256), grad=True, pad=pad)
    return dict(kind=kind, dtype=dtype, V=_size(rng, 1000, 152000), batch=_log(rng, 1, 64), L=_log(rng, 1, 16384),
                columns=rng.random() < 0.4, nbias=_log(rng, 1, 128), pad=pad)


# ---------------------------------------------------------------------------------------------------- inputs
def _rows(gen, n, c, pad, dtype, scale=1.0, shift=0.0):
    """n x c normal values in rows of c + pad elements."""
    x = torch.randn((n, c + pad), dtype=torch.float32, device="cuda", generator=gen)
    return x.mul_(scale).add_(shift).to(TORCH[dtype])[:, :c]


def _buffer(n, c, pad, dtype):
    return torch.empty((n, c + pad), dtype=TORCH[dtype], device="cuda")[:, :c]


def _starts(case, seed):
    """Where the packed sequences of a case start, and the end of the last: random cuts, among them an empty sequence and
    one of a single token where there are four or more."""
    r = random.Random(int(seed) * 7919 + 17)
    n, s = case["N"], case["nseq"]
    cuts = sorted(r.randint(0, n) for _ in range(s - 1))
    if s >= 4:
        cuts[1] = cuts[0]
        cuts[2] = min(cuts[1] + 1, n)
        cuts.sort()
    return [0] + cuts + [n]


def _distinct(gen, n, v, k):
    """n rows of k distinct numbers below v, more of the low ones: a random start and odd steps through the vocabulary."""
    first = torch.randint(0, v, (n, 1), device="cuda", generator=gen)
    step = torch.randint(1, max(2, v // (k + 1)), (n, 1), device="cuda", generator=gen)
    return (first + step * torch.arange(k, device="cuda")[None, :]) % v


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rand = lambda *shape: torch.rand(shape, dtype=torch.float32, device="cuda", generator=gen)
    randn = lambda *shape: torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen)
    fp32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")
    scratch = lambda n: torch.empty((max(1, n),), dtype=torch.uint8, device="cuda")
    kind, dt, pad = case["kind"], case["dtype"], case.get("pad", 0)
    s = {"case": case, "stream": torch.cuda.current_stream()}
    if own:
        import paper_2108_11033_amd as g
        s["g"] = g
    if kind == "norm":
        N, C = case["N"], case["C"]
        # activations with a mean of their own and a few large features, as between trained layers
        s["x"] = _rows(gen, N, C, pad, dt, 1.5, 0.3)
        s["gamma"], s["beta"] = 1.0 + 0.2 * randn(C), 0.2 * randn(C)
        if case["mode"] == "fwd":
            s["y"], s["mean"], s["rstd"] = _buffer(N, C, pad, dt), fp32(N), fp32(N)
        else:
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().float()
            s["dy"] = _rows(gen, N, C, pad, dt)
            s["dx"], s["dgamma"], s["dbeta"] = _buffer(N, C, pad, dt), fp32(C), fp32(C)
            if own:
                s["ws"] = scratch(g.layer_norm_workspace(N, C))
    elif kind == "glr":
        N, H, q = case["N"], case["H"], case["nseq"]
        s["gates"] = _rows(gen, N, 3 * H, pad, dt)
        s["bias"] = 0.2 * randn(3 * H)
        s["bias"][:H] += 2.5                                  # forget gates of trained layers are mostly open
        s["h0"] = 0.5 * randn(q, H)
        s["starts"] = _starts(case, seed)
        s["seq_start"] = torch.tensor(s["starts"], dtype=torch.int32, device="cuda")
        s["y"], s["h_last"] = _buffer(N, H, pad, dt), fp32(q, H)
        if case["mode"] == "train":
            s["dy"], s["dh_last"] = _rows(gen, N, H, pad, dt), randn(q, H)
            s["dgates"], s["dbias"], s["dh0"] = _buffer(N, 3 * H, pad, dt), fp32(3 * H), fp32(q, H)
        if own:
            s["ws"] = scratch(g.glr_workspace(N, H))
            s["states"] = scratch(g.glr_states(N, H)) if case["mode"] == "train" else None
    elif kind == "glr_step":
        H, b = case["H"], case["batch"]
        s["gates"], s["bias"], s["h"] = randn(3 * H, b), 0.2 * randn(3 * H), 0.5 * randn(H, b)
        s["bias"][:H] += 2.5
        s["h_new"], s["y"] = fp32(H, b), _buffer(H, b, 0, dt)
    elif kind == "distill":
        N, V, k = case["N"], case["V"], case["k"]
        s["z"] = _rows(gen, N, V, pad, dt, 2.5)
        s["ids"] = _distinct(gen, N, V, k).to(torch.int32)
        # the teacher's logits, best first; some rows list fewer entries (number -1); some tokens are padding (weight 0)
        s["top"] = (2.0 * randn(N, k) + 6.0).sort(dim=1, descending=True)[0].contiguous()
        fewer = (rand(N, 1) < 0.2) & (torch.arange(k, device="cuda")[None, :] >= (k + 1) // 2)
        s["ids"] = torch.where(fewer, torch.full_like(s["ids"], -1), s["ids"]).contiguous()
        # (the mean over the tokens; in fp16 with the loss scale that keeps small gradients above the type's smallest numbers)
        s["weight"] = (rand(N) < 0.95).float() * ((1024.0 if dt == "f16" else 1.0) / N)
        s["loss"] = fp32(N)
        s["dz"] = _buffer(N, V, pad, dt) if case["grad"] else None
        if own:
            s["ws"] = scratch(g.distill_topk_workspace(N, V))
    else:
        V, b, L, nb = case["V"], case["batch"], case["L"], case["nbias"]
        shape = (V, b) if case["columns"] else (b, V)
        s["z"] = _rows(gen, shape[0], shape[1], pad, dt, 3.0)
        s["out"] = _buffer(shape[0], shape[1], pad, dt)
        s["history"] = (V * rand(b, L) ** 3).to(torch.int32).clamp_(0, V - 1)     # some words come often
        s["lens"] = (rand(b) * (L + 1)).to(torch.int32).clamp_(0, L)
        s["lens"][0] = L
        s["repetition"], s["frequency"], s["presence"] = 1.0 + 0.3 * rand(b), 0.3 * rand(b), 0.3 * rand(b)
        s["bias_ids"] = _distinct(gen, b, V, nb).to(torch.int32).contiguous()
        s["bias_values"] = 2.0 * randn(b, nb)
        words = torch.randint(-2 ** 31, 2 ** 31, (b, (V + 31) // 32), device="cuda", generator=gen)
        free = rand(b, 1) < 0.5                                                    # no grammar: everything is allowed
        s["allowed"] = torch.where(free, torch.full_like(words, -1), words).to(torch.int32).contiguous()
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"norm": _norm, "glr": _glr, "glr_step": _glr_step, "distill": _distill, "rules": _rules}[s["case"]["kind"]](s)


def _norm(s):
    case, dt = s["case"], s["case"]["dtype"]
    N, C = case["N"], case["C"]
    if own:
        x, ld = s["x"], s["x"].stride(0)
        if case["mode"] == "fwd":
            s["g"].layer_norm(x, dt, ld, s["gamma"], s["beta"], EPS, N, C, s["y"], s["y"].stride(0), s["mean"], s["rstd"], s["stream"])
            return s["y"]
        s["g"].layer_norm_backward(s["dy"], s["dy"].stride(0), x, ld, dt, s["gamma"], s["mean"], s["rstd"], N, C, s["dx"],
                                   s["dx"].stride(0), s["dgamma"], s["dbeta"], s["ws"], s["stream"])
        return [s["dx"], s["dgamma"], s["dbeta"]]
    x = s["x"].float()
    if case["mode"] == "fwd":
        d = x - x.mean(1, keepdim=True)
        return (d * (d.square().mean(1, keepdim=True) + EPS).rsqrt() * s["gamma"] + s["beta"]).to(TORCH[dt])
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    d = dy * s["gamma"]
    dx = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    return [dx.to(TORCH[dt]), (dy * xh).sum(0), dy.sum(0)]


def _scan(a, b):
    """h_t = a_t h_(t-1) + b_t down the rows, h_(-1) = 0, by doubling: after a step of d, row t holds the map from row t - 2d."""
    d, n = 1, a.shape[0]
    while d < n:
        b = torch.cat([b[:d], a[d:] * b[:-d] + b[d:]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _glr(s):
    case, dt = s["case"], s["case"]["dtype"]
    N, H, q = case["N"], case["H"], case["nseq"]
    train = case["mode"] == "train"
    if own:
        g, gates, ld = s["g"], s["gates"], s["gates"].stride(0)
        g.glr_sequence(gates, dt, ld, s["bias"], s["h0"], s["seq_start"], q, N, H, s["y"], s["y"].stride(0), s["h_last"],
                       s["states"], s["ws"], s["stream"])
        if not train:
            return [s["y"], s["h_last"]]
        g.glr_sequence_backward(gates, dt, ld, s["bias"], s["h0"], s["seq_start"], q, N, H, s["states"], s["dy"], s["dy"].stride(0),
                                s["dh_last"], s["dgates"], s["dgates"].stride(0), s["dbias"], s["dh0"], s["ws"], s["stream"])
        return [s["y"], s["h_last"], s["dgates"], s["dbias"], s["dh0"]]
    starts = s["seq_start"].long()
    some = (starts[1:] > starts[:-1]).nonzero()[:, 0]         # the sequences that hold a token
    first, last = starts[:-1][some], starts[1:][some] - 1
    z = s["gates"].float() + s["bias"]
    f, keep, c, o = torch.sigmoid(z[:, :H]), torch.sigmoid(-z[:, :H]), z[:, H:2 * H], torch.sigmoid(z[:, 2 * H:])
    del z
    a, b = f.clone(), keep * c
    b[first] += f[first] * s["h0"][some]
    a[first] = 0
    h = _scan(a, b)
    h_last = s["h0"].clone()
    h_last[some] = h[last]
    y = (o * h).to(TORCH[dt])
    if not train:
        return [y, h_last]
    dy = s["dy"].float()
    e = dy * o
    e[last] += s["dh_last"][some]
    a = torch.cat([f[1:], torch.zeros_like(f[:1])])           # what a row hands back to the one before
    a[last] = 0
    G = _scan(a.flip(0), e.flip(0)).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first] = s["h0"][some]
    dz = torch.cat([G * f * keep * (before - c), G * keep, dy * h * o * (1 - o)], dim=1)
    dh0 = s["dh_last"].clone()
    dh0[some] = (f * G)[first]
    return [y, h_last, dz.to(TORCH[dt]), dz.sum(0), dh0]


def _glr_step(s):
    case, dt = s["case"], s["case"]["dtype"]
    H, b = case["H"], case["batch"]
    if own:
        s["g"].glr_step(s["gates"], b, s["bias"], s["h"], b, s["h_new"], b, s["y"], dt, b, H, b, s["stream"])
        return [s["y"], s["h_new"]]
    z = s["gates"] + s["bias"][:, None]
    h = torch.sigmoid(z[:H]) * s["h"] + torch.sigmoid(-z[:H]) * z[H:2 * H]
    return [(torch.sigmoid(z[2 * H:]) * h).to(TORCH[dt]), h]


def _distill(s):
    case, dt = s["case"], s["case"]["dtype"]
    N, V, k = case["N"], case["V"], case["k"]
    if own:
        s["g"].distill_topk(s["z"], dt, s["z"].stride(0), s["top"], s["ids"], k, k, TAU, s["weight"], N, V, s["loss"], s["dz"],
                            s["dz"].stride(0) if case["grad"] else 0, s["ws"], s["stream"])
        return [s["loss"], s["dz"]] if case["grad"] else [s["loss"]]
    ids = s["ids"].long()
    there = ids >= 0
    t = torch.where(there, s["top"] / TAU, torch.full_like(s["top"], -math.inf))
    t = t - t.amax(1, keepdim=True)
    p = torch.exp(t)
    total = p.sum(1, keepdim=True)
    p = p / total
    logp = t - torch.log(total)
    z = s["z"].float() / TAU
    z = z - z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z).sum(1, keepdim=True))
    at = ids.clamp(min=0)
    terms = torch.where(there, p * (logp - (z.gather(1, at) - lse)), torch.zeros_like(p))
    loss = s["weight"] * (TAU * TAU * terms.sum(1))
    if not case["grad"]:
        return [loss]
    dz = torch.exp(z - lse).scatter_add_(1, at, torch.where(there, -p, torch.zeros_like(p)))
    return [loss, (dz * (TAU * s["weight"][:, None])).to(TORCH[dt])]


def _rules(s):
    case, dt = s["case"], s["case"]["dtype"]
    V, b, L, nb, cols = case["V"], case["batch"], case["L"], case["nbias"], case["columns"]
    if own:
        s["g"].logit_rules(s["z"], dt, s["z"].stride(0), V, b, s["out"], s["out"].stride(0), columns=cols, history=s["history"],
                           ld_history=L, max_history=L, history_len=s["lens"], repetition=s["repetition"], frequency=s["frequency"],
                           presence=s["presence"], bias_ids=s["bias_ids"], bias_values=s["bias_values"], nbias=nb, ld_bias=nb,
                           allowed=s["allowed"], ld_allowed=s["allowed"].stride(0), stream=s["stream"])
        return s["out"]
    z = (s["z"].t() if cols else s["z"]).float()
    said = torch.arange(L, device="cuda")[None, :] < s["lens"][:, None]
    count = torch.zeros((b, V), dtype=torch.float32, device="cuda").scatter_add_(1, s["history"].long(), said.float())
    rep = s["repetition"][:, None]
    z = torch.where(count > 0, torch.where(z > 0, z / rep, z * rep), z)
    z = z - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    z = z.scatter_add(1, s["bias_ids"].long(), s["bias_values"])
    bits = (s["allowed"][:, :, None] >> torch.arange(32, device="cuda")) & 1
    z = torch.where(bits.reshape(b, -1)[:, :V] > 0, z, torch.full_like(z, -math.inf)).to(TORCH[dt])
    return z.t().contiguous() if cols else z


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm64, "glr": _glr64, "glr_step": _step64, "distill": _distill64, "rules": _rules64}[case["kind"]](s)


def _norm64(s):
    x, g = s["x"].double(), s["gamma"].double()
    C = x.shape[1]
    if s["case"]["mode"] == "fwd":
        m = x.sum(1) / C
        v = ((x - m[:, None]) ** 2).sum(1) / C
        return (x - m[:, None]) / torch.sqrt(v + EPS)[:, None] * g + s["beta"].double()
    m, r, dy = s["mean"].double(), s["rstd"].double(), s["dy"].double()
    xh = (x - m[:, None]) * r[:, None]
    s1 = (dy * g).sum(1, keepdim=True)
    s2 = (dy * g * xh).sum(1, keepdim=True)
    return [(C * dy * g - s1 - xh * s2) * r[:, None] / C, (dy * xh).sum(0), dy.sum(0)]


def _glr64(s):
    """Token by token, every sequence from its own start."""
    case = s["case"]
    H, q = case["H"], case["nseq"]
    starts = torch.tensor(s["starts"], device="cuda")
    lens = starts[1:] - starts[:-1]
    longest = int(lens.max())
    order = torch.argsort(lens, descending=True, stable=True)       # sequences that still run come first
    begin = starts[:-1][order]
    running = [int(n) for n in (lens[order][None, :] > torch.arange(longest, device="cuda")[:, None]).sum(1).cpu()] if longest else []
    z = s["gates"].double() + s["bias"].double()
    f, c, o = 1 / (1 + torch.exp(-z[:, :H])), z[:, H:2 * H].contiguous(), 1 / (1 + torch.exp(-z[:, 2 * H:]))
    del z
    h_all = torch.empty_like(c)
    h = s["h0"].double()[order].clone()
    for t in range(longest):
        n = running[t]
        rows = begin[:n] + t
        ft = f[rows]
        h[:n] = c[rows] + ft * (h[:n] - c[rows])
        h_all[rows] = h[:n]
    back = torch.argsort(order)
    y, h_last = o * h_all, h[back]
    if case["mode"] != "train":
        return [y, h_last]
    dy = s["dy"].double()
    G_all, h_before = torch.empty_like(c), torch.empty_like(c)
    carry = s["dh_last"].double()[order].clone()                    # the gradient of a row's state from what follows it
    h0 = s["h0"].double()[order]
    for t in range(longest - 1, -1, -1):
        n = running[t]
        rows = begin[:n] + t
        total = carry[:n] + dy[rows] * o[rows]
        G_all[rows] = total
        h_before[rows] = h_all[rows - 1] if t else h0[:n]
        carry[:n] = total * f[rows]
    dz = torch.cat([G_all * (h_before - c) * f * (1 - f), G_all * (1 - f), dy * h_all * o * (1 - o)], 1)
    return [y, h_last, dz, dz.sum(0), carry[back]]


def _step64(s):
    H = s["case"]["H"]
    z = s["gates"].double() + s["bias"].double()[:, None]
    f, o = 1 / (1 + torch.exp(-z[:H])), 1 / (1 + torch.exp(-z[2 * H:]))
    h = f * s["h"].double() + (1 - f) * z[H:2 * H]
    return [o * h, h]


def _distill64(s):
    case = s["case"]
    N, grad = case["N"], case["grad"]
    losses, grads = [], []
    for i in range(0, N, 1024):
        z = s["z"][i:i + 1024].double() / TAU
        ids, top, w = s["ids"][i:i + 1024].long(), s["top"][i:i + 1024].double() / TAU, s["weight"][i:i + 1024].double()
        there = ids >= 0
        p = torch.where(there, torch.exp(top - top.max()), torch.zeros_like(top))
        p = p / p.sum(1, keepdim=True)
        logq = z - torch.logsumexp(z, 1, keepdim=True)
        q_at = logq.gather(1, ids.clamp(min=0))
        losses.append(w * TAU ** 2 * torch.where(there, p * (torch.log(p) - q_at), torch.zeros_like(p)).sum(1))
        if grad:
            d = torch.exp(logq).scatter_add_(1, ids.clamp(min=0), -p)
            grads.append(w[:, None] * TAU * d)
    return [torch.cat(losses)] + ([torch.cat(grads)] if grad else [])


def _rules64(s):
    case = s["case"]
    V, cols = case["V"], case["columns"]
    z = (s["z"].t() if cols else s["z"]).double()
    out = torch.empty_like(z, memory_format=torch.contiguous_format)
    for i in range(case["batch"]):
        n = int(s["lens"][i])
        count = torch.bincount(s["history"][i, :n].long(), minlength=V).double()
        r, fr, pr = s["repetition"][i].double(), s["frequency"][i].double(), s["presence"][i].double()
        row = z[i].clone()
        seen = count > 0
        row[seen] = torch.where(row[seen] > 0, row[seen] / r, row[seen] * r)
        row -= fr * count + pr * seen
        row[s["bias_ids"][i].long()] += s["bias_values"][i].double()
        v = torch.arange(V, device="cuda")
        row[((s["allowed"][i].long()[v // 32] >> (v % 32)) & 1) == 0] = -math.inf
        out[i] = row
    return out.t().contiguous() if cols else out


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Each input read once and each output written once; a training pass of the recurrence counts its gates once, although
    its forward and backward calls each read them."""
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind == "norm":
        n, c = case["N"], case["C"]
        if case["mode"] == "fwd":
            return {"bytes": 2 * n * c * e + 8 * c + 8 * n, "flops": 8.0 * n * c}
        return {"bytes": 3 * n * c * e + 12 * c + 8 * n, "flops": 16.0 * n * c}
    if kind == "glr":
        n, h, q = case["N"], case["H"], case["nseq"]
        state = 4 * (q * h)
        if case["mode"] == "fwd":
            return {"bytes": 4 * n * h * e + 12 * h + 2 * state, "flops": 12.0 * n * h}
        return {"bytes": 8 * n * h * e + 24 * h + 4 * state, "flops": 45.0 * n * h}
    if kind == "glr_step":
        h, b = case["H"], case["batch"]
        return {"bytes": h * b * (12 + 4 + 4 + e) + 12 * h, "flops": 12.0 * h * b}
    if kind == "distill":
        n, v, k = case["N"], case["V"], case["k"]
        return {"bytes": n * v * e * (2 if case["grad"] else 1) + n * (8 * k + 8), "flops": (7.0 if case["grad"] else 4.0) * n * v}
    v, b = case["V"], case["batch"]
    return {"bytes": b * (2 * v * e + v / 8 + 4 * case["L"] + 8 * case["nbias"] + 16), "flops": 6.0 * v * b}
