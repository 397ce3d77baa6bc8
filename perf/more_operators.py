"""Further operators of a recurrent language model: the gated delta rule (a recurrent layer whose state is a matrix for each
head), the clipped policy loss with a KL term, and clipping by the global gradient norm.

A case names its kind ("gdr", "gdr_step", "policy", "clip"), its element type and the sizes of its kind.
`prepare` makes what a program has in hand (inputs, output buffers, workspaces); `run` is one pass through one operator.
Where `own` is false the pass is written in elementary torch operations in fp32, rounded once at the end.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
NORM_EPS = 1e-6
CHUNK = 64                    # tokens that the plain form of the delta rule takes at a time


def listed():
    return [
        # One token for one caller through a layer of 16 heads: the smallest call, where latency counts.
        dict(name="gdr_step_b1", kind="gdr_step", dtype="f16", heads=16, key_heads=16, dk=64, dv=64, batch=1),
        # One token for 32 callers, four value heads to a key head: 33 MB of states read and written.
        dict(name="gdr_step_b32", kind="gdr_step", dtype="bf16", heads=16, key_heads=4, dk=128, dv=128, batch=32),
        # Eight utterances of 64 frames through a layer of 1024 units, inference.
        dict(name="gdr_frames_b8", kind="gdr", mode="fwd", dtype="f16", N=512, nseq=8, heads=16, key_heads=16, dk=64, dv=64, pad=0),
        # Three texts in fp32, heads of odd widths, rows that are not aligned.
        dict(name="gdr_odd", kind="gdr", mode="fwd", dtype="f32", N=5003, nseq=3, heads=6, key_heads=3, dk=40, dv=72, pad=3),
        # A training step on 40 texts of different lengths packed one after another (one empty, one of a single token), keys shared by four heads.
        dict(name="gdr_train_packed", kind="gdr", mode="train", dtype="bf16", N=24007, nseq=40, heads=16, key_heads=4, dk=64, dv=64, pad=0),
        # A training step on one long text: no parallelism but along the sequence, the heads and the columns of the states.
        dict(name="gdr_train_long", kind="gdr", mode="train", dtype="bf16", N=32768, nseq=1, heads=8, key_heads=8, dk=128, dv=128, pad=0),
        # The policy loss of a small classifier of frames: 1000 classes, loss and gradient.
        dict(name="policy_classes", kind="policy", dtype="f32", N=1024, V=1000, pad=0),
        # The policy loss of a language model: 8192 tokens, 32768 words, loss and gradient.
        dict(name="policy_train", kind="policy", dtype="bf16", N=8192, V=32768, pad=0),
        # A short batch over a large vocabulary of odd size: fewer rows than compute units, rows that are not aligned.
        dict(name="policy_few_rows", kind="policy", dtype="f16", N=24, V=131075, pad=0),
        # The gradients of a small recurrent language model (512 words, 256 units, 2 layers): few and small tensors.
        dict(name="clip_small", kind="clip", dtype="f32", out="f32", V=512, units=256, layers=2, loss_scale=1.0),
        # A model of odd sizes in fp16 with a loss scale, clipped in its own type.
        dict(name="clip_odd", kind="clip", dtype="f16", out="f16", V=8191, units=515, layers=9, loss_scale=1024.0),
        # 168 M gradients in bf16 (32768 words, 1024 units, 24 layers) into the fp32 buffers that an optimizer reads.
        dict(name="clip_large", kind="clip", dtype="bf16", out="f32", V=32768, units=1024, layers=24, loss_scale=1.0),
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
    most = {}
    for c in listed():
        w = work(c)
        most = {m: max(most.get(m, 0), w[m]) for m in w}
    while True:
        c = _draw(rng)
        if all(v <= most[m] for m, v in work(c).items()):
            return c


def _draw(rng):
    kind = rng.choice(["gdr", "gdr", "gdr", "gdr_step", "policy", "policy", "clip"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 3, 8])
    if kind in ("gdr", "gdr_step"):
        wide = lambda: rng.choice([64, 128, rng.randint(8, 128)])
        key_heads = _log(rng, 1, 16)
        c = dict(kind=kind, dtype=dtype, heads=key_heads * rng.choice([1, 1, 2, 4]), key_heads=key_heads, dk=wide(), dv=wide())
        if kind == "gdr_step":
            return dict(c, batch=_log(rng, 1, 64))
        N = _log(rng, 1, 32768)
        return dict(c, mode=rng.choice(["fwd", "train"]), N=N, nseq=_log(rng, 1, max(1, min(64, N // 4))), pad=pad)
    if kind == "policy":
        return dict(kind=kind, dtype=dtype, N=_log(rng, 1, 8192), V=_size(rng, 500, 152000), pad=pad)
    return dict(kind=kind, dtype=dtype, out=rng.choice([dtype, "f32"]), V=_size(rng, 500, 65536), units=_size(rng, 64, 2048),
                layers=_log(rng, 1, 32), loss_scale=1024.0 if dtype == "f16" else 1.0)


# ---------------------------------------------------------------------------------------------------- inputs
def _rows(gen, n, c, pad, dtype, scale=1.0):
    """n x c normal values in rows of c + pad elements."""
    x = torch.randn((n, c + pad), dtype=torch.float32, device="cuda", generator=gen)
    return x.mul_(scale).to(TORCH[dtype])[:, :c]


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


def _shapes(case):
    """The parameters of a recurrent language model: embedding and head, and of every layer two products, a bias and the norms' parameters."""
    V, H = case["V"], case["units"]
    return [(V, H), (V, H), (H,), (H,)] + [(3 * H, H), (H, H), (3 * H,), (H,), (H,)] * case["layers"]


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
    if kind in ("gdr", "gdr_step"):
        h, hk, dk, dv = case["heads"], case["key_heads"], case["dk"], case["dv"]
        s["scale"] = dk ** -0.5
        gates = lambda n: -torch.nn.functional.softplus(1.5 * randn(n, h) - 3.0)       # logarithms of decays, most of them near 1
    if kind == "gdr_step":
        b = case["batch"]
        s["q"], s["k"], s["v"] = randn(hk * dk, b), randn(hk * dk, b), randn(h * dv, b)
        s["decay"], s["beta"] = gates(b).t().contiguous(), torch.sigmoid(randn(h, b))
        s["state"] = 0.3 * randn(b, h, dk, dv)
        s["new"], s["y"] = fp32(b, h, dk, dv), _buffer(h * dv, b, 0, dt)
    elif kind == "gdr":
        N, q = case["N"], case["nseq"]
        s["q"], s["k"], s["v"] = _rows(gen, N, hk * dk, pad, dt), _rows(gen, N, hk * dk, pad, dt), _rows(gen, N, h * dv, pad, dt)
        s["decay"], s["beta"] = gates(N), torch.sigmoid(randn(N, h))
        s["s0"] = 0.3 * randn(q, h, dk, dv)
        s["starts"] = _starts(case, seed)
        s["seq_start"] = torch.tensor(s["starts"], dtype=torch.int32, device="cuda")
        s["y"], s["s_last"] = _buffer(N, h * dv, pad, dt), fp32(q, h, dk, dv)
        if case["mode"] == "train":
            s["dy"], s["ds_last"] = _rows(gen, N, h * dv, pad, dt), 0.3 * randn(q, h, dk, dv)
            s["dq"], s["dkey"], s["dvalue"] = _buffer(N, hk * dk, pad, dt), _buffer(N, hk * dk, pad, dt), _buffer(N, h * dv, pad, dt)
            s["ddecay"], s["dbeta"], s["ds0"] = fp32(N, h), fp32(N, h), fp32(q, h, dk, dv)
        if own:
            s["ws"] = scratch(g.gdr_workspace(N, q, h, hk, dk, dv))
            s["states"] = scratch(g.gdr_states(N, q, h, dk, dv)) if case["mode"] == "train" else None
    elif kind == "policy":
        N, V = case["N"], case["V"]
        s["z"] = _rows(gen, N, V, pad, dt, 2.5)
        s["ids"] = torch.randint(0, V, (N,), device="cuda", generator=gen).to(torch.int32)
        s["clip"], s["kl"], s["tau"] = 0.2, 0.05, 1.0
        # what the word's logarithm was when the text was sampled, and what the model that training started from gives it; a ratio within a
        # rounding of a border of the clipping has no side of its own, so none is drawn there
        now = torch.cat([torch.log_softmax(s["z"][i:i + 1024].float(), 1).gather(1, s["ids"][i:i + 1024, None].long())[:, 0] for i in range(0, N, 1024)])
        ratio = 0.15 * randn(N)
        for edge in (math.log1p(s["clip"]), math.log1p(-s["clip"])):
            ratio = torch.where((ratio - edge).abs() < 1e-3, torch.full_like(ratio, edge + 2e-3), ratio)
        s["old"] = now - ratio
        s["ref"] = s["old"] + 0.2 * randn(N)
        s["advantage"] = randn(N)
        # the mean over the tokens, some of them padding; in fp16 with a loss scale
        s["weight"] = (rand(N) < 0.95).float() * ((1024.0 if dt == "f16" else 1.0) / N)
        s["loss"], s["logp"], s["dz"] = fp32(N), fp32(N), _buffer(N, V, pad, dt)
        if own:
            s["ws"] = scratch(g.policy_loss_workspace(N, V))
    else:
        shapes = _shapes(case)
        # gradients as a loss scale leaves them; some parameters learn far more than others
        sizes = (torch.rand(len(shapes), generator=torch.Generator().manual_seed(int(seed))) * 4 - 6).exp2()
        s["grads"] = [(randn(*shape) * (float(size) * 0.02 * case["loss_scale"])).to(TORCH[dt]) for shape, size in zip(shapes, sizes)]
        s["flat"] = torch.empty((sum(x.numel() for x in s["grads"]),), dtype=TORCH[case["out"]], device="cuda")
        s["outs"] = [part.view(x.shape) for part, x in zip(s["flat"].split([x.numel() for x in s["grads"]]), s["grads"])]
        s["max_norm"], s["unscale"], s["norm"] = 1.0, 1.0 / case["loss_scale"], fp32(1)
        if own:
            s["list"] = g.GradList(s["grads"], s["outs"])
            s["ws"] = scratch(s["list"].workspace)
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"gdr": _gdr, "gdr_step": _gdr_step, "policy": _policy, "clip": _clip}[s["case"]["kind"]](s)


def _gdr(s):
    c, dt = s["case"], s["case"]["dtype"]
    N, q, h, hk, dk, dv = c["N"], c["nseq"], c["heads"], c["key_heads"], c["dk"], c["dv"]
    train = c["mode"] == "train"
    if own:
        g, ld = s["g"], [s[x].stride(0) for x in ("q", "k", "v")]
        g.gdr_sequence(s["q"], s["k"], s["v"], dt, *ld, s["decay"], s["beta"], h, s["s0"], s["seq_start"], q, N, h, hk, dk, dv,
                       s["scale"], NORM_EPS, s["y"], s["y"].stride(0), s["s_last"], s["states"], s["ws"], s["stream"])
        if not train:
            return [s["y"], s["s_last"]]
        g.gdr_sequence_backward(s["q"], s["k"], s["v"], dt, *ld, s["decay"], s["beta"], h, s["s0"], s["seq_start"], q, N, h, hk, dk, dv,
                                s["scale"], NORM_EPS, s["states"], s["dy"], s["dy"].stride(0), s["ds_last"], s["dq"], s["dq"].stride(0),
                                s["dkey"], s["dkey"].stride(0), s["dvalue"], s["dvalue"].stride(0), s["ddecay"], s["dbeta"], h, s["ds0"],
                                s["ws"], s["stream"])
        return [s["y"], s["s_last"], s["dq"], s["dkey"], s["dvalue"], s["ddecay"], s["dbeta"], s["ds0"]]
    # Tokens in chunks of one sequence each: place[chunk, i] is a row, or N (a row of zeros) behind the sequence's end.
    starts = torch.tensor(s["starts"], device="cuda")
    lens = starts[1:] - starts[:-1]
    parts = (lens + CHUNK - 1) // CHUNK
    total = sum((b - a + CHUNK - 1) // CHUNK for a, b in zip(s["starts"], s["starts"][1:]))
    of = torch.repeat_interleave(torch.arange(q, device="cuda"), parts, output_size=total)
    begin = torch.cumsum(parts, 0) - parts
    row = (torch.arange(total, device="cuda") - begin[of])[:, None] * CHUNK + torch.arange(CHUNK, device="cuda")
    place = torch.where(row < lens[of][:, None], starts[:-1][of][:, None] + row, N)
    some = (lens > 0).nonzero()[:, 0]
    first, last = begin[some], (begin + parts - 1)[some]

    def chunks(x, n):                                        # N x (n d) -> chunk, head, token, d
        x = torch.cat([x.float(), torch.zeros((1, x.shape[1]), device="cuda")])
        return x[place].view(total, CHUNK, n, -1).transpose(1, 2)

    def tokens(x):                                           # and back
        flat = torch.zeros((N + 1, x.shape[1] * x.shape[3]), device="cuda")
        flat[place.view(-1)] = x.transpose(1, 2).reshape(total * CHUNK, -1)
        return flat[:N]

    shared = lambda x: x.repeat_interleave(h // hk, 1)
    qr, kr = chunks(s["q"], hk), chunks(s["k"], hk)
    rq, rk = (qr.square().sum(-1, keepdim=True) + NORM_EPS).rsqrt(), (kr.square().sum(-1, keepdim=True) + NORM_EPS).rsqrt()
    Q, K, V = shared(qr * rq) * s["scale"], shared(kr * rk), chunks(s["v"], h)
    G = torch.cumsum(chunks(s["decay"], h).double(), 2)[..., 0]
    b = chunks(s["beta"], h)
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device="cuda").tril()
    decay = torch.where(lower, torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], 0.0)), 0.0).float()
    since, until = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]      # from the chunk's start, to its end
    over, whole = lower.tril(-1), torch.exp(G[..., -1]).float()[..., None, None]
    KT = K.transpose(-1, -2).contiguous()
    L = (K @ KT) * decay * over
    P = (Q @ KT) * decay
    # E = X - L b E with X = V - since K S: E = T X, T the inverse of 1 + L b, formed from blocks of twice the size each time
    A = L * b.transpose(-1, -2)
    T = torch.eye(CHUNK, device="cuda").expand_as(A).contiguous()
    n = 1
    while n < CHUNK:
        t = T.view(total, h, CHUNK // (2 * n), 2, n, CHUNK // (2 * n), 2, n)
        a = A.view(total, h, CHUNK // (2 * n), 2, n, CHUNK // (2 * n), 2, n)
        at = torch.arange(CHUNK // (2 * n), device="cuda")
        low = -(t[:, :, at, 1, :, at, 1] @ a[:, :, at, 1, :, at, 0] @ t[:, :, at, 0, :, at, 0])
        t[:, :, at, 1, :, at, 0] = low
        n *= 2
    # A chunk takes S to (whole - (K until)' b T since K) S + (K until)' b T V; these maps are joined by doubling.
    KU = (K * until).transpose(-1, -2).contiguous()
    W = b * (T @ (since * K))
    step = whole * torch.eye(dk, device="cuda") - KU @ W
    add = KU @ (b * (T @ V))
    add[first] += step[first] @ s["s0"][some]
    joined = step.clone()
    joined[first] = 0
    S = _join(joined, add)
    s_last = s["s0"].clone()
    s_last[some] = S[last]
    before = torch.cat([torch.zeros_like(S[:1]), S[:-1]])
    before[first] = s["s0"][some]
    KS, QS = since * (K @ before), since * (Q @ before)
    E = T @ (V - KS)
    U = b * E
    y = tokens(QS + P @ U).to(TORCH[dt])
    if not train:
        return [y, s_last]
    t_ = lambda x: x.transpose(-1, -2).contiguous()
    dO = chunks(s["dy"], h)
    # the states' gradients: at a chunk's end to its start by the same map transposed
    dU0 = t_(P) @ dO
    back = t_(since * Q) @ dO - t_(W) @ dU0
    end = t_(step)
    back[last] += end[last] @ s["ds_last"][some]
    joined = end.clone()
    joined[last] = 0
    dS = _join(joined.flip(0), back.flip(0)).flip(0)         # at the chunks' starts
    after = torch.cat([dS[1:], torch.zeros_like(dS[:1])])
    after[last] = s["ds_last"][some]
    ds0 = s["ds_last"].clone()
    ds0[some] = dS[first]
    dU = dU0 + until * (K @ after)
    Y = t_(T) @ (b * dU)                                     # the gradient of E, and of X and V
    dbeta = ((dU - t_(L) @ Y) * E).sum(-1)
    dP = (dO @ t_(U)) * decay
    dL = -(Y @ t_(U)) * decay * over
    dQ = since * (dO @ t_(before)) + dP @ K
    dK_row = dL @ K - since * (Y @ t_(before))
    dK_col = t_(dP) @ Q + t_(dL) @ K + until * (U @ t_(after))
    row, col, qq = (dK_row * K).sum(-1, keepdim=True), (dK_col * K).sum(-1, keepdim=True), (dQ * Q).sum(-1, keepdim=True)
    dG = (qq + row - col)[..., 0]
    at_end = torch.cat([S[:-1], torch.zeros_like(S[:1])])
    at_end[last] = S[last]
    dG[..., -1] += (at_end * after).sum((-1, -2))
    dg = dG.double().flip(2).cumsum(2).flip(2).float()
    joint = lambda x: x.reshape(total, hk, h // hk, CHUNK, dk).sum(2)
    dq = rq * joint(dQ * s["scale"] - Q / s["scale"] * qq)
    dkey = rk * joint(dK_row + dK_col - K * (row + col))
    out = [y, s_last, tokens(dq).to(TORCH[dt]), tokens(dkey).to(TORCH[dt]), tokens(Y).to(TORCH[dt])]
    return out + [tokens(dg[..., None]), tokens(dbeta[..., None]), ds0]


def _join(a, b):
    """S_n = a_n S_(n-1) + b_n over the first axis, S_(-1) = 0, by doubling: after a step of d, n holds the map from n - 2d."""
    d, n = 1, a.shape[0]
    while d < n:
        b = torch.cat([b[:d], a[d:] @ b[:-d] + b[d:]])
        a = torch.cat([a[:d], a[d:] @ a[:-d]])
        d *= 2
    return b


def _gdr_step(s):
    c, dt = s["case"], s["case"]["dtype"]
    h, hk, dk, dv, n = c["heads"], c["key_heads"], c["dk"], c["dv"], c["batch"]
    if own:
        s["g"].gdr_step(s["q"], s["k"], s["v"], n, n, n, s["decay"], s["beta"], n, s["state"], s["new"], s["y"], dt, n, h, hk, dk, dv,
                        s["scale"], NORM_EPS, n, s["stream"])
        return [s["y"], s["new"]]
    q, k = (s[x].t().reshape(n, hk, dk) for x in ("q", "k"))
    q = (q * (q.square().sum(2, keepdim=True) + NORM_EPS).rsqrt() * s["scale"]).repeat_interleave(h // hk, 1)
    k = (k * (k.square().sum(2, keepdim=True) + NORM_EPS).rsqrt()).repeat_interleave(h // hk, 1)
    v = s["v"].t().reshape(n, h, dv)
    S = s["state"] * torch.exp(s["decay"].t())[..., None, None]
    u = s["beta"].t()[..., None] * (v - (k[..., None] * S).sum(2))
    S = S + k[..., None] * u[:, :, None, :]
    return [(q[..., None] * S).sum(2).reshape(n, h * dv).t().to(TORCH[dt]).contiguous(), S]


def _policy(s):
    case, dt = s["case"], s["case"]["dtype"]
    N, V, tau, clip, kl = case["N"], case["V"], s["tau"], s["clip"], s["kl"]
    if own:
        s["g"].policy_loss(s["z"], dt, s["z"].stride(0), s["ids"], N, V, s["loss"], s["logp"], s["dz"], s["dz"].stride(0), s["ws"],
                           old_logp=s["old"], ref_logp=s["ref"], advantage=s["advantage"], weight=s["weight"], temperature=tau,
                           clip_low=clip, clip_high=clip, kl=kl, stream=s["stream"])
        return [s["loss"], s["logp"], s["dz"]]
    z = s["z"].float() / tau
    z = z - z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z).sum(1, keepdim=True))
    at = s["ids"].long()[:, None]
    logp = (z.gather(1, at) - lse)[:, 0]
    r, A, d = torch.exp(logp - s["old"]), s["advantage"], s["ref"] - logp
    plain, cut = r * A, r.clamp(1 - clip, 1 + clip) * A
    loss = s["weight"] * (kl * (torch.exp(d) - d - 1) - torch.minimum(plain, cut))
    slope = torch.where(plain <= cut, -plain, torch.zeros_like(plain)) + kl * (1 - torch.exp(d))
    factor = (s["weight"] * slope / tau)[:, None]
    dz = (-factor * torch.exp(z - lse)).scatter_add_(1, at, factor)
    return [loss, logp, dz.to(TORCH[dt])]


def _clip(s):
    if own:
        s["g"].grad_clip(s["list"], s["max_norm"], s["unscale"], s["norm"], s["ws"], s["stream"])
        return [s["norm"], s["flat"]]
    squares = torch.stack([x.double().square().sum() for x in s["grads"]])
    norm = s["unscale"] * squares.sum().sqrt()
    factor = (s["unscale"] * torch.clamp(s["max_norm"] / norm, max=1.0)).float()
    return [norm.float()[None], torch.cat([(x.float() * factor).to(s["flat"].dtype).view(-1) for x in s["grads"]])]


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    if case["kind"] == "gdr" and case["N"] / case["nseq"] > 40000:
        return None
    s = prepare(case, seed)
    return {"gdr": _gdr64, "gdr_step": _step64, "policy": _policy64, "clip": _clip64}[case["kind"]](s)


def _unit(x):
    """(x / its length, 1 / its length)."""
    r = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) + NORM_EPS)
    return x * r, r


def _gdr64(s):
    """Token by token, every sequence from its own start; backward through states that are formed again from every 64th."""
    c = s["case"]
    N, q, h, hk, dk, dv = c["N"], c["nseq"], c["heads"], c["key_heads"], c["dk"], c["dv"]
    starts = torch.tensor(s["starts"], device="cuda")
    lens = starts[1:] - starts[:-1]
    longest = int(lens.max())
    order = torch.argsort(lens, descending=True, stable=True)       # sequences that still run come first
    begin = starts[:-1][order]
    running = [int(n) for n in (lens[order][None, :] > torch.arange(longest, device="cuda")[:, None]).sum(1).cpu()] if longest else []
    raw = lambda name, n: s[name].double().reshape(N, n, -1)
    kn, kr = _unit(raw("k", hk))
    qn, qr = _unit(raw("q", hk))
    v, a, b = raw("v", h), torch.exp(s["decay"].double()), s["beta"].double()
    of = lambda x, rows: x[rows].repeat_interleave(h // hk, 1)
    y = torch.empty_like(v)
    S = s["s0"].double()[order].clone()

    def advance(S, t):
        """S after token t of every running sequence; what the token met: decayed states, differences."""
        n = running[t]
        rows = begin[:n] + t
        k = of(kn, rows)
        D = S[:n] * a[rows][..., None, None]
        e = v[rows] - (k[:, :, None, :] @ D)[:, :, 0]
        return D + k[..., None] * (b[rows][..., None] * e)[:, :, None, :], D, e, rows

    kept = []
    for t in range(longest):
        if t % 64 == 0:
            kept.append(S[:running[t]].clone())
        new, _, _, rows = advance(S, t)
        S[:running[t]] = new
        y[rows] = s["scale"] * (of(qn, rows)[:, :, None, :] @ new)[:, :, 0]
    back = torch.argsort(order)
    s_last = S[back]
    if c["mode"] != "train":
        return [y.reshape(N, -1), s_last]
    dy = raw("dy", h)
    dqn, dkn = (torch.zeros((N, h, dk), dtype=torch.float64, device="cuda") for _ in range(2))
    dvalue, ddecay, dbeta = torch.zeros_like(v), torch.zeros_like(a), torch.zeros_like(b)
    dS = s["ds_last"].double()[order].clone()
    for block in range(len(kept) - 1, -1, -1):
        S, met = kept[block], []
        for t in range(64 * block, min(longest, 64 * block + 64)):
            old = S
            new, D, e, rows = advance(old, t)
            met.append((t, old[:running[t]], new, D, e, rows))
            S = new
        for t, old, new, D, e, rows in reversed(met):
            n = running[t]
            k, bt, dyt = of(kn, rows), b[rows][..., None], dy[rows]
            dqn[rows] = s["scale"] * (new @ dyt[..., None])[..., 0]
            g = dS[:n] + s["scale"] * of(qn, rows)[..., None] * dyt[:, :, None, :]
            du = (k[:, :, None, :] @ g)[:, :, 0]
            de = bt * du
            dkn[rows] = (g @ (bt * e)[..., None])[..., 0] - (D @ de[..., None])[..., 0]
            dbeta[rows] = (du * e).sum(-1)
            dvalue[rows] = de
            dD = g - k[..., None] * de[:, :, None, :]
            ddecay[rows] = (dD * D).sum((-1, -2))
            dS[:n] = dD * a[rows][..., None, None]
        del met
    joint = lambda x: x.reshape(N, hk, h // hk, dk).sum(2)
    through = lambda d, x, r: (r * (d - x * (d * x).sum(-1, keepdim=True))).reshape(N, -1)
    return [y.reshape(N, -1), s_last, through(joint(dqn), qn, qr), through(joint(dkn), kn, kr), dvalue.reshape(N, -1), ddecay, dbeta, dS[back]]


def _step64(s):
    c = s["case"]
    h, hk, dk, dv, n = c["heads"], c["key_heads"], c["dk"], c["dv"], c["batch"]
    y, new = torch.empty((h * dv, n), dtype=torch.float64, device="cuda"), torch.empty_like(s["state"], dtype=torch.float64)
    for j in range(h):
        i = j // (h // hk)
        q, k = (_unit(s[x].double()[i * dk:(i + 1) * dk].t())[0] for x in ("q", "k"))
        D = torch.exp(s["decay"][j].double())[:, None, None] * s["state"][:, j].double()
        e = s["v"][j * dv:(j + 1) * dv].double().t() - torch.matmul(k[:, None], D)[:, 0]
        new[:, j] = D + s["beta"][j].double()[:, None, None] * torch.matmul(k[:, :, None], e[:, None])
        y[j * dv:(j + 1) * dv] = s["scale"] * torch.matmul(q[:, None], new[:, j])[:, 0].t()
    return [y, new]


def _policy64(s):
    case = s["case"]
    N, tau, lo, hi = case["N"], s["tau"], 1 - s["clip"], 1 + s["clip"]
    losses, logps, grads = [], [], []
    for i in range(0, N, 1024):
        part = slice(i, min(N, i + 1024))
        logq = torch.log_softmax(s["z"][part].double() / tau, 1)
        ids = s["ids"][part].long()
        rows = torch.arange(ids.shape[0], device="cuda")
        lp = logq[rows, ids]
        old, ref, A, w = (s[x][part].double() for x in ("old", "ref", "advantage", "weight"))
        r = torch.exp(lp - old)
        # where the ratio has left its bounds in the advantage's direction, the objective stands still
        held = ((A > 0) & (r > hi)) | ((A < 0) & (r < lo))
        gain = torch.where(held, A * r.clamp(lo, hi), A * r)
        losses.append(w * (s["kl"] * (torch.exp(ref - lp) - (ref - lp) - 1) - gain))
        logps.append(lp)
        dlp = w * (s["kl"] * (1 - torch.exp(ref - lp)) - torch.where(held, torch.zeros_like(gain), gain))
        d = -torch.exp(logq)
        d[rows, ids] += 1
        grads.append(d * dlp[:, None] / tau)
    return [torch.cat(losses), torch.cat(logps), torch.cat(grads)]


def _clip64(s):
    total = math.sqrt(sum(float((x.double() ** 2).sum()) for x in s["grads"])) / s["case"]["loss_scale"]
    factor = min(1.0, s["max_norm"] / total) / s["case"]["loss_scale"]
    return [torch.tensor([total], dtype=torch.float64), torch.cat([x.double().flatten() * factor for x in s["grads"]])]


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Each input read once and each output written once.  Operations of the delta rule are those of its definition: a token of a head decays
    its dk x dv states, takes two products with them and adds one outer product; a training pass does that once more and its gradients."""
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind in ("gdr", "gdr_step"):
        h, hk, dk, dv = case["heads"], case["key_heads"], case["dk"], case["dv"]
        if kind == "gdr_step":
            b = case["batch"]
            return {"bytes": b * (8 * h * dk * dv + 4 * (2 * hk * dk + h * dv + 2 * h) + e * h * dv), "flops": 7.0 * b * h * dk * dv}
        n, state = case["N"], 4 * case["nseq"] * h * dk * dv
        row = e * (2 * hk * dk + 2 * h * dv) + 8 * h
        if case["mode"] == "fwd":
            return {"bytes": n * row + 2 * state, "flops": 7.0 * n * h * dk * dv}
        return {"bytes": 2 * n * row + 4 * state, "flops": 26.0 * n * h * dk * dv}
    if kind == "policy":
        n, v = case["N"], case["V"]
        return {"bytes": 2 * n * v * e + 28 * n, "flops": 7.0 * n * v}
    count = sum(math.prod(shape) for shape in _shapes(case))
    return {"bytes": count * (e + SIZE[case["out"]]), "flops": 3.0 * count}
