"""A small recurrent language model with pruned layers: retrained from its dense teacher's top logits, then served token by
token -- the operators of include/grim_lm.h with the BCR products between them.

    embedding -> [ layer norm -> gate product (3H x H) -> gated linear recurrence -> output product (H x H) -> + ] x layers
              -> layer norm -> head product (V x H) -> logits

Training keeps a dense copy of the weights under their masks (PyTorch's matrix products on rows of tokens); serving packs
what the masks keep and runs everything in columns, one per caller, as grim_bcr_spmv leaves it.

    python -m paper_2108_11033_amd.recurrent_lm            # a teacher, a student pruned 4x, 60 steps of distillation, some text
"""
from __future__ import annotations

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from . import binding, lm

EPS = 1e-5
DTYPES = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}


def _scratch(n: int, device) -> torch.Tensor:
    return torch.empty((max(1, n),), dtype=torch.uint8, device=device)


def _fp32(t: torch.Tensor) -> torch.Tensor:
    """A parameter or state as the kernels read it, whatever type a model holds it in."""
    return t.detach().float().contiguous()


def _check(fits: bool, what: str):
    if not fits:
        raise ValueError(what)


def _check_place(*tensors: torch.Tensor):
    """The kernels take addresses: each has to be memory of the GPU that they are launched on."""
    for t in tensors:
        _check(t.is_cuda and t.device.index == torch.cuda.current_device(), f"an operand lies on {t.device}, not on the current GPU")


def _whole(t: torch.Tensor) -> bool:
    return not (t.is_floating_point() or t.is_complex() or t.dtype == torch.bool)


# ---------------------------------------------------------------------------------------------- training
class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta):
        _check(x.dim() == 2 and gamma.numel() == beta.numel() == x.shape[1],
               f"rows of {tuple(x.shape)} with parameters of {tuple(gamma.shape)} and {tuple(beta.shape)}")
        _check_place(x, gamma, beta)
        x = x.contiguous()
        N, C = x.shape
        ctx.like = [(t.shape, t.dtype) for t in (gamma, beta)]
        gamma, beta = _fp32(gamma), _fp32(beta)
        y, mean, rstd = torch.empty_like(x), x.new_empty(N, dtype=torch.float32), x.new_empty(N, dtype=torch.float32)
        lm.layer_norm(x, DTYPES[x.dtype], C, gamma, beta, EPS, N, C, y, C, mean, rstd, torch.cuda.current_stream())
        ctx.save_for_backward(x, gamma, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, gamma, mean, rstd = ctx.saved_tensors
        N, C = x.shape
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)      # (sums in fp32)
        lm.layer_norm_backward(dy.contiguous(), C, x, C, DTYPES[x.dtype], gamma, mean, rstd, N, C, dx, C, dgamma, dbeta,
                               _scratch(lm.layer_norm_workspace(N, C), x.device), torch.cuda.current_stream())
        return dx, *(t.view(shape).to(dtype) for t, (shape, dtype) in zip((dgamma, dbeta), ctx.like))


class GatedRecurrence(torch.autograd.Function):
    """(outputs, last states in fp32) of packed sequences: gates N x 3H, bias 3H, h0 a row of H per sequence; seq_start holds the sequences'
    starts and the end, one number more than there are sequences: 0 first, ascending, N last."""

    @staticmethod
    def forward(ctx, gates, bias, h0, seq_start):
        _check(gates.dim() == 2 and gates.shape[1] >= 3 and gates.shape[1] % 3 == 0 and bias.numel() == gates.shape[1],
               f"gates of {tuple(gates.shape)} with biases of {tuple(bias.shape)}")
        N, H = gates.shape[0], gates.shape[1] // 3
        _check(h0.dim() >= 1 and h0.shape[0] >= 1 and h0.numel() == h0.shape[0] * H, f"states of {tuple(h0.shape)} for sequences of {H} units")
        _check(seq_start.numel() == h0.shape[0] + 1 and _whole(seq_start),
               f"states of {h0.shape[0]} sequences with starts of {tuple(seq_start.shape)} ({seq_start.dtype})")
        _check_place(gates, bias, h0, seq_start)
        gates, seq_start = gates.contiguous(), seq_start.int().contiguous()
        ctx.types = bias.dtype, h0.dtype
        bias, h0 = _fp32(bias), _fp32(h0)
        y, h_last = gates.new_empty(N, H), torch.empty_like(h0)
        states = _scratch(lm.glr_states(N, H), gates.device)
        lm.glr_sequence(gates, DTYPES[gates.dtype], 3 * H, bias, h0, seq_start, h0.shape[0], N, H, y, H, h_last, states,
                        _scratch(lm.glr_workspace(N, H), gates.device), torch.cuda.current_stream())
        ctx.save_for_backward(gates, bias, h0, seq_start, states)
        return y, h_last

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh_last):
        gates, bias, h0, seq_start, states = ctx.saved_tensors
        N, H = gates.shape[0], gates.shape[1] // 3
        dgates, dbias, dh0 = torch.empty_like(gates), torch.empty_like(bias), torch.empty_like(h0)
        lm.glr_sequence_backward(gates, DTYPES[gates.dtype], 3 * H, bias, h0, seq_start, h0.shape[0], N, H, states, dy.contiguous(), H,
                                 dh_last.contiguous(), dgates, 3 * H, dbias, dh0, _scratch(lm.glr_workspace(N, H), gates.device),
                                 torch.cuda.current_stream())
        return dgates, dbias.to(ctx.types[0]), dh0.to(ctx.types[1]), None


class GatedDeltaRule(torch.autograd.Function):
    """(outputs, last states in fp32) of packed sequences: q and k N x key heads x Dk, v N x heads x Dv, decay (logarithms, at most 0) and beta N x heads, s0 sequences x heads x
    Dk x Dv; seq_start holds the sequences' starts and the end, in ascending order: rows in front of the first start and behind the end (a batch that is padded) have outputs and gradients
    of 0.  norm_eps > 0: queries and keys count divided by their lengths."""

    @staticmethod
    def forward(ctx, q, k, v, decay, beta, s0, seq_start, scale, norm_eps):
        _check(q.dim() == v.dim() == 3 and q.shape == k.shape and q.shape[0] == v.shape[0] and q.shape[1] >= 1 and v.shape[1] % q.shape[1] == 0 and q.dtype == k.dtype == v.dtype,
               f"queries of {tuple(q.shape)}, keys of {tuple(k.shape)} and values of {tuple(v.shape)} ({q.dtype}, {k.dtype}, {v.dtype})")
        N, hk, Dk = q.shape
        h, Dv = v.shape[1:]
        _check(decay.shape == beta.shape == (N, h), f"{N} rows of {h} heads with decays of {tuple(decay.shape)} and betas of {tuple(beta.shape)}")
        _check(s0.dim() == 4 and s0.shape[0] >= 1 and s0.shape[1:] == (h, Dk, Dv), f"states of {tuple(s0.shape)} for {h} heads of {Dk} x {Dv}")
        _check(seq_start.numel() == s0.shape[0] + 1 and _whole(seq_start),
               f"states of {s0.shape[0]} sequences with starts of {tuple(seq_start.shape)} ({seq_start.dtype})")
        _check_place(q, k, v, decay, beta, s0, seq_start)
        ctx.types = decay.dtype, beta.dtype, s0.dtype
        q, k, v, seq_start = q.contiguous(), k.contiguous(), v.contiguous(), seq_start.int().contiguous()
        decay, beta, s0 = _fp32(decay), _fp32(beta), _fp32(s0)
        ctx.sizes = (s0.shape[0], N, h, hk, Dk, Dv, scale, norm_eps)
        y, s_last = torch.zeros_like(v), torch.empty_like(s0)                   # (the kernels leave rows of no sequence as they are)
        states = _scratch(lm.gdr_states(N, s0.shape[0], h, Dk, Dv), q.device)
        lm.gdr_sequence(q, k, v, DTYPES[q.dtype], hk * Dk, hk * Dk, h * Dv, decay, beta, h, s0, seq_start, *ctx.sizes, y, h * Dv, s_last, states,
                        _scratch(lm.gdr_workspace(N, s0.shape[0], h, hk, Dk, Dv), q.device), torch.cuda.current_stream())
        ctx.save_for_backward(q, k, v, decay, beta, s0, seq_start, states)
        return y, s_last

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds_last):
        q, k, v, decay, beta, s0, seq_start, states = ctx.saved_tensors
        nseq, N, h, hk, Dk, Dv = ctx.sizes[:6]
        dq, dk, dv, ddecay, dbeta = (torch.zeros_like(t) for t in (q, k, v, decay, beta))
        ds0 = torch.empty_like(s0)
        lm.gdr_sequence_backward(q, k, v, DTYPES[q.dtype], hk * Dk, hk * Dk, h * Dv, decay, beta, h, s0, seq_start, *ctx.sizes, states, dy.contiguous(), h * Dv,
                                 ds_last.contiguous(), dq, hk * Dk, dk, hk * Dk, dv, h * Dv, ddecay, dbeta, h, ds0,
                                 _scratch(lm.gdr_workspace(N, nseq, h, hk, Dk, Dv), q.device), torch.cuda.current_stream())
        return dq, dk, dv, *(t.to(dtype) for t, dtype in zip((ddecay, dbeta, ds0), ctx.types)), None, None, None


class DistillTopK(torch.autograd.Function):
    """The sum over rows of weight times the distillation loss.  The teacher's logits and the weights get no gradient; that of the logits is formed as PolicyLoss
    forms it, in fp32 with the loss, in 16 bits after the factor of the backward pass.  The lists are N x k (numbers of any whole type: those outside 0 .. V-1 are absent), weight N."""

    @staticmethod
    def forward(ctx, logits, top_logits, top_ids, temperature, weight):
        _check(logits.dim() == 2, f"logits are rows of a vocabulary, not {tuple(logits.shape)}")
        N, V = logits.shape
        _check(top_ids.dim() == 2 and top_ids.shape[0] == N and top_logits.shape == top_ids.shape and _whole(top_ids),
               f"{N} rows of logits with lists of {tuple(top_logits.shape)} logits and {tuple(top_ids.shape)} numbers ({top_ids.dtype})")
        _check(weight.numel() == N, f"{N} rows of logits with weights of {tuple(weight.shape)}")
        _check_place(logits, top_logits, top_ids, weight)
        logits, top_logits, weight = logits.contiguous(), _fp32(top_logits), _fp32(weight)
        if top_ids.dtype != torch.int32:                       # (before they are cut to 32 bits)
            top_ids = top_ids.long()
            top_ids = torch.where((top_ids >= 0) & (top_ids < V), top_ids, -1).int()
        top_ids = top_ids.contiguous()
        ctx.temperature = temperature
        dz = torch.empty_like(logits) if logits.dtype == torch.float32 else None
        loss = DistillTopK._call(logits, top_logits, top_ids, temperature, weight, dz)
        ctx.save_for_backward(*((logits, top_logits, top_ids, weight) if dz is None else (dz,)))
        return loss.sum()

    @staticmethod
    @once_differentiable
    def backward(ctx, upstream):
        if len(ctx.saved_tensors) == 1:
            dz = ctx.saved_tensors[0] * upstream
        else:
            logits, top_logits, top_ids, weight = ctx.saved_tensors
            dz = torch.empty_like(logits)
            DistillTopK._call(logits, top_logits, top_ids, ctx.temperature, weight * upstream, dz)
        return dz, None, None, None, None

    @staticmethod
    def _call(logits, top_logits, top_ids, temperature, weight, dz):
        N, V = logits.shape
        loss = logits.new_empty(N, dtype=torch.float32)
        lm.distill_topk(logits, DTYPES[logits.dtype], V, top_logits, top_ids, top_ids.shape[1], top_ids.shape[1], temperature, weight, N, V,
                        loss, dz, V, _scratch(lm.distill_topk_workspace(N, V), logits.device), torch.cuda.current_stream())
        return loss


class PolicyLoss(torch.autograd.Function):
    """(the sum over rows of the clipped policy loss, the words' logarithms) of N x V logits.  ids: the sampled words, N (of any whole type; a row whose word lies outside 0 .. V-1 is
    padding); old_logp and ref_logp: what the policy that sampled them and the reference give them, or None; advantage N; weight N, or None (1).  Only the logits get a gradient.  That of
    fp32 logits is formed with the loss, in one pass over them; that of 16-bit logits in the backward pass, from the logits again, with the factor that arrives there (a loss scale) in the
    weights, so that it is rounded to 16 bits once, after the factor: before it, an element below 2^-25 in fp16 would be 0 whatever the scale.  (Both passes, and with the gradient
    formed with the loss and multiplied by the factor later: 8192 x 32768 in bf16 320 and 966 us; 24 x 131075 in fp16, where the host's time counts, 97 and 79.)"""

    @staticmethod
    def forward(ctx, logits, ids, old_logp, ref_logp, advantage, weight, temperature, clip, kl):
        _check(logits.dim() == 2, f"logits are rows of a vocabulary, not {tuple(logits.shape)}")
        N, V = logits.shape
        given = [t for t in (old_logp, ref_logp, advantage, weight) if t is not None]
        _check(ids.numel() == N and _whole(ids) and all(t.numel() == N for t in given),
               f"{N} rows of logits with words of {tuple(ids.shape)} ({ids.dtype}) and rows of {[tuple(t.shape) for t in given]}")
        _check_place(logits, ids, *given)
        logits = logits.contiguous()
        if ids.dtype != torch.int32:                           # (before they are cut to 32 bits)
            ids = ids.long()
            ids = torch.where((ids >= 0) & (ids < V), ids, -1).int()
        ids = ids.contiguous()
        rows = [None if t is None else _fp32(t) for t in (old_logp, ref_logp, advantage, weight)]
        ctx.numbers = temperature, clip, kl
        loss, logp = logits.new_empty(N, dtype=torch.float32), logits.new_empty(N, dtype=torch.float32)
        dz = torch.empty_like(logits) if logits.dtype == torch.float32 else None
        PolicyLoss._call(logits, ids, rows, ctx.numbers, loss, logp, dz)
        ctx.save_for_backward(*((logits, ids, *rows) if dz is None else (dz,)))
        ctx.mark_non_differentiable(logp)
        return loss.sum(), logp

    @staticmethod
    @once_differentiable
    def backward(ctx, upstream, _):
        if len(ctx.saved_tensors) == 1:
            dz = ctx.saved_tensors[0] * upstream
        else:
            logits, ids, *rows = ctx.saved_tensors
            rows[3] = upstream.expand(logits.shape[0]).contiguous() if rows[3] is None else rows[3] * upstream
            dz = torch.empty_like(logits)
            PolicyLoss._call(logits, ids, rows, ctx.numbers, None, None, dz)
        return dz, None, None, None, None, None, None, None, None

    @staticmethod
    def _call(logits, ids, rows, numbers, loss, logp, dz):
        N, V = logits.shape
        lm.policy_loss(logits, DTYPES[logits.dtype], V, ids, N, V, loss, logp, dz, V, _scratch(lm.policy_loss_workspace(N, V), logits.device), old_logp=rows[0], ref_logp=rows[1],
                       advantage=rows[2], weight=rows[3], temperature=numbers[0], clip_low=numbers[1], clip_high=numbers[1], kl=numbers[2], stream=torch.cuda.current_stream())


@torch.no_grad()
def clip_gradients(parameters, max_norm: float, unscale: float = 1.0) -> torch.Tensor:
    """Every gradient times unscale min(1, max_norm / norm), in place; the norm (of all, unscaled), one number on the GPU.  A parameter, or any number of them."""
    if isinstance(parameters, torch.Tensor):                   # (whose rows have no gradients of their own)
        parameters = [parameters]
    grads = [p.grad for p in parameters if p.grad is not None]
    _check(len({id(t) for t in grads}) == len(grads), "a gradient is there twice")
    _check_place(*grads)
    together = [t.contiguous() for t in grads]                 # (copies of those that are not, clipped and copied back)
    group = lm.GradList(together)
    dev = torch.device("cuda", torch.cuda.current_device())
    norm = torch.empty(1, device=dev)
    lm.grad_clip(group, max_norm, unscale, norm, _scratch(group.workspace, dev), torch.cuda.current_stream())
    for t, clipped in zip(grads, together):
        if clipped is not t:
            t.copy_(clipped)
    return norm


class RecurrentLM(torch.nn.Module):
    """Dense weights, each product's under a mask of ones and zeros (all ones until prune())."""

    def __init__(self, vocabulary: int, units: int, layers: int, seed: int = 0):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *shape: torch.nn.Parameter(torch.randn(shape, generator=gen) / shape[-1] ** 0.5)
        self.units, self.layers = units, layers
        self.embedding = torch.nn.Parameter(torch.randn((vocabulary, units), generator=gen))
        self.gates = torch.nn.ParameterList([rand(3 * units, units) for _ in range(layers)])
        self.outs = torch.nn.ParameterList([rand(units, units) for _ in range(layers)])
        bias = torch.zeros(3 * units)
        bias[:units] = 2.0                                     # forget gates start mostly open
        self.biases = torch.nn.ParameterList([torch.nn.Parameter(bias.clone()) for _ in range(layers)])
        self.gammas = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(units)) for _ in range(layers + 1)])
        self.betas = torch.nn.ParameterList([torch.nn.Parameter(torch.zeros(units)) for _ in range(layers + 1)])
        self.head = rand(vocabulary, units)
        self.blocks = {}                                       # name of a product -> (BR, BC, kept rows, kept columns) per block

    def products(self):
        return {**{f"gates{i}": w for i, w in enumerate(self.gates)}, **{f"outs{i}": w for i, w in enumerate(self.outs)}, "head": self.head}

    def prune(self, BR: int, BC: int, kr: int, kc: int):
        """Keeps, in every BR x BC block of every product, the kr rows and then the kc columns of the largest norms."""
        for name, w in self.products().items():
            M, K = w.shape
            sq = w.detach().float().view(M // BR, BR, K // BC, BC).permute(0, 2, 1, 3).square()      # strip, column block, row, column
            rows = sq.sum(3).topk(kr, dim=2).indices.sort(2).values
            some = torch.zeros_like(sq[..., 0]).scatter_(2, rows, 1.0)
            cols = (sq * some[..., None]).sum(2).topk(kc, dim=2).indices.sort(2).values
            keep = some[..., None] * torch.zeros_like(sq[:, :, 0]).scatter_(2, cols, 1.0)[:, :, None]
            mask = keep.permute(0, 2, 1, 3).reshape(M, K).to(w.dtype)
            self.blocks[name] = (BR, BC, rows.cpu().numpy(), cols.cpu().numpy())
            self.register_buffer("mask_" + name, mask)

    def weight(self, name: str) -> torch.Tensor:
        w = self.products()[name]
        mask = getattr(self, "mask_" + name, None)
        return w if mask is None else w * mask

    def forward(self, tokens, seq_start, h0=None):
        """Logits of packed sequences of tokens (N x V) and every layer's last states."""
        x = self.embedding[tokens]
        last = []
        for i in range(self.layers):
            state = h0[i] if h0 is not None else x.new_zeros((seq_start.numel() - 1, self.units), dtype=torch.float32)
            n = LayerNorm.apply(x, self.gammas[i], self.betas[i])
            y, h = GatedRecurrence.apply(n @ self.weight(f"gates{i}").t(), self.biases[i], state, seq_start)
            x = x + y @ self.weight(f"outs{i}").t()
            last.append(h)
        return LayerNorm.apply(x, self.gammas[-1], self.betas[-1]) @ self.weight("head").t(), last


def distill(student: RecurrentLM, teacher: RecurrentLM, batches, k: int = 16, temperature: float = 2.0, rate: float = 1e-2, max_norm: float | None = None):
    """One step of distillation per batch of (tokens, seq_start), gradients clipped by their norm if max_norm is given; the losses."""
    optimizer = torch.optim.Adam(student.parameters(), lr=rate)
    losses = []
    for tokens, seq_start in batches:
        with torch.no_grad():
            top = teacher(tokens, seq_start)[0].topk(k, dim=1)
        logits, _ = student(tokens, seq_start)
        weight = torch.full((tokens.numel(),), 1.0 / tokens.numel(), device=tokens.device)
        loss = DistillTopK.apply(logits, top.values.float().contiguous(), top.indices.int().contiguous(), temperature, weight)
        optimizer.zero_grad()
        loss.backward()
        if max_norm is not None:
            clip_gradients(student.parameters(), max_norm)
        optimizer.step()
        losses.append(float(loss.detach()))
    return losses


def reinforce(model: RecurrentLM, batches, rate: float = 1e-3, temperature: float = 1.0, clip: float = 0.2, kl: float = 0.05, max_norm: float = 1.0, epochs: int = 2):
    """Steps of the clipped policy loss per batch of (tokens, seq_start, advantage): token t + 1 of a text is the word that was sampled after token t, and advantage[t] is that word's (that
    of a text's last token counts for nothing, as none follows it; the loss is the sum over the words by the number of tokens).  The policy that the texts came from, and the reference of
    the KL term, is the model before the batch's first step.  The losses."""
    optimizer = torch.optim.Adam(model.parameters(), lr=rate)
    losses = []
    for tokens, seq_start, advantage in batches:
        ends = seq_start[1:].long() - 1
        words = torch.cat([tokens[1:], tokens[:1]]).int()
        words[ends[ends >= 0]] = -1                            # (an empty text ends where the one before it does)
        weight = torch.full((tokens.numel(),), 1.0 / tokens.numel(), device=tokens.device)
        old = None
        for _ in range(epochs):
            logits, _ = model(tokens, seq_start)
            loss, logp = PolicyLoss.apply(logits, words, old, old, advantage, weight, temperature, clip, kl)
            old = logp if old is None else old
            optimizer.zero_grad()
            loss.backward()
            clip_gradients(model.parameters(), max_norm)
            optimizer.step()
            losses.append(float(loss.detach()))
    return losses


# ---------------------------------------------------------------------------------------------- serving
class Server:
    """A pruned model for `batch` callers, one token per step.  Products are BCR products in fp16; states stay in fp32."""

    def __init__(self, model: RecurrentLM, batch: int):
        _check_place(*model.parameters())
        self.model, self.batch = model, batch
        self.gammas, self.betas, self.biases = ([_fp32(p) for p in group] for group in (model.gammas, model.betas, model.biases))
        self.packed = {name: self._pack(model, name) for name in model.products()}
        dev = model.embedding.device
        fp32, fp16 = (lambda *s: torch.empty(s, device=dev)), (lambda *s: torch.empty(s, dtype=torch.float16, device=dev))
        H, V = model.units, model.head.shape[0]
        self.h = [torch.zeros((H, batch), device=dev) for _ in range(model.layers)]
        self.gates, self.y, self.out, self.norm, self.logits = fp32(3 * H, batch), fp16(H, batch), fp32(H, batch), fp32(batch, H), fp32(V, batch)

    @staticmethod
    def _pack(model, name):
        BR, BC, rows, cols = model.blocks[name]
        nb = rows.shape[0] * rows.shape[1]
        ptr = lambda n: np.arange(nb + 1, dtype=np.int32) * n
        w = model.weight(name).detach().half().cpu().numpy()
        return binding.pack(w, "f16", BR, BC, ptr(rows.shape[2]), rows.astype(np.uint16).ravel(), ptr(cols.shape[2]),
                            cols.astype(np.uint16).ravel())

    def _norm(self, x, i, stream):
        """Layer norm of the callers' rows, as the columns of the next product."""
        lm.layer_norm(x, "f32", x.shape[1], self.gammas[i], self.betas[i], EPS, self.batch, x.shape[1], self.norm, x.shape[1],
                      stream=stream)
        return self.norm.t().to(torch.float16).contiguous()

    @torch.no_grad()
    def step(self, tokens: torch.Tensor, **rules) -> torch.Tensor:
        """Takes one token of each caller; the logits of the next, V x batch, with the rules of lm.logit_rules applied."""
        m, b, stream = self.model, self.batch, torch.cuda.current_stream()
        H, V = m.units, self.logits.shape[0]
        x = m.embedding[tokens].float()
        _check(x.shape == (b, H), f"embeddings of {tuple(x.shape)} for {b} callers: one token of each")
        for i in range(m.layers):
            binding.spmm(self.packed[f"gates{i}"], self._norm(x, i, stream), b, b, self.gates, b, stream)
            lm.glr_step(self.gates, b, self.biases[i], self.h[i], b, self.h[i], b, self.y, "f16", b, H, b, stream)
            binding.spmm(self.packed[f"outs{i}"], self.y, b, b, self.out, b, stream)
            x = x + self.out.t()
        binding.spmm(self.packed["head"], self._norm(x, m.layers, stream), b, b, self.logits, b, stream)
        if rules:
            lm.logit_rules(self.logits, "f32", b, V, b, self.logits, b, columns=True, stream=stream, **rules)
        return self.logits


def generate(server: Server, prompt: torch.Tensor, steps: int, repetition: float = 1.3) -> torch.Tensor:
    """The likeliest word after word for every caller, words said before made less likely (batch x (1 + steps))."""
    b = server.batch
    said = torch.zeros((b, steps + 1), dtype=torch.int32, device=prompt.device)
    said[:, 0] = prompt
    lens = torch.ones((b,), dtype=torch.int32, device=prompt.device)
    strength = torch.full((b,), repetition, device=prompt.device)
    for t in range(steps):
        logits = server.step(said[:, t].long(), history=said, ld_history=steps + 1, max_history=steps + 1, history_len=lens,
                             repetition=strength)
        said[:, t + 1] = logits.argmax(0).int()
        lens += 1
    return said


def main(vocabulary: int = 512, units: int = 256, layers: int = 2, steps: int = 60, seed: int = 0):
    dev = torch.device("cuda:0")
    teacher = RecurrentLM(vocabulary, units, layers, seed).to(dev)
    student = RecurrentLM(vocabulary, units, layers, seed).to(dev)
    student.prune(16, 32, 8, 16)
    gen = torch.Generator().manual_seed(seed + 1)
    lengths = [200, 1, 311, 0, 256, 256]                      # texts of different lengths, one after another
    starts = torch.tensor([0] + np.cumsum(lengths).tolist(), dtype=torch.int32, device=dev)
    batches = [(torch.randint(0, vocabulary, (sum(lengths),), generator=gen).to(dev), starts) for _ in range(steps)]
    losses = distill(student, teacher, batches)
    print(f"distillation loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps of {sum(lengths)} tokens")
    server = Server(student, batch=4)
    print(generate(server, torch.arange(4, device=dev), 12).cpu().numpy())
    return losses


if __name__ == "__main__":
    main()
