"""What stands around the melded layers in a fine-tuning step, as PyTorch modules and functions: norms joined with the residual
stream, SwiGLU from 8-bit checkpoints, frozen linear layers on 4-bit codes, log-probabilities and the paired preference loss.

Plumbing only: every computation is a C-ABI call.  The melded layers keep nothing of their inputs but O_A, so with the
checkpoints here a block's saved activations are those of its attention, one byte and 1/32 for each element of the norms' streams,
of gate and of up.

First derivatives only: under create_graph gradients come as ever, and following them (a penalty on a gradient) raises RuntimeError.
"""
from typing import Optional, Sequence, Tuple

import torch

from . import binding as _b
from .nn import MeldedGroup, MeldedLoRALinear

_U8 = torch.uint8


def _rows(t: torch.Tensor) -> torch.Tensor:
    """[..., n] as [T, n] whose rows may lie apart, as the kernels take them."""
    t2 = t.reshape(-1, t.shape[-1])
    ok = t2.shape[1] == 1 or t2.stride(1) == 1
    if t2.shape[0] > 1:
        ok = ok and t2.stride(0) >= t2.shape[1] and t2.stride(0) % 16 == 0
    return t2 if ok and t2.data_ptr() % 16 == 0 else t2.clone(memory_format=torch.contiguous_format)     # also of a dense one that begins elsewhere


def _dense_bf16(t: torch.Tensor, width: int) -> torch.Tensor:
    t2 = t.reshape(-1, width).to(torch.bfloat16).contiguous()
    return t2 if t2.data_ptr() % 16 == 0 else t2.clone()


def _check_rows(a, b, what: str) -> None:
    """Leading shapes that name the same rows in the same order: alike up to ones in front, or one of them flat."""
    if a == b:
        return
    short, long = sorted((tuple(a), tuple(b)), key=len)
    alike = (1,) * (len(long) - len(short)) + short == long
    if not alike and not (min(len(a), len(b)) <= 1 and torch.Size(a).numel() == torch.Size(b).numel()):
        raise ValueError(f"{what}: rows of shapes {tuple(a)} and {tuple(b)}")


def _codes(T: int, n: int, dev) -> Tuple[torch.Tensor, torch.Tensor]:
    return torch.empty(T, n, dtype=_U8, device=dev), torch.empty(T, (n + 31) // 32, dtype=_U8, device=dev)


class _Refused(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tie, *grads):
        return grads

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the kernels around the melded layers have first derivatives only: their gradients cannot be differentiated")


def _tie(x: torch.Tensor) -> torch.Tensor:
    """The last output of a function here, saved last: it holds nothing, and stands for the function in the graph of its gradients.  (The functions do not have
    missing gradients made up: there would always be one for it.)"""
    return torch.empty(0, dtype=torch.float32, device=x.device)


def _first_order(backward):
    """A backward pass of kernels.  Under create_graph its gradients depend on the function's inputs through a node that refuses to be followed;
    with no graph a penalty on them would be dropped without a word."""

    def run(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads[:-1])
        with torch.no_grad():
            out = backward(ctx, *grads[:-1])
        again = iter(_Refused.apply(ctx.saved_tensors[-1], *(v.detach() for v in out if isinstance(v, torch.Tensor))))
        return tuple(next(again) if isinstance(v, torch.Tensor) else v for v in out)

    return run


class _NormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, b, w, w_post, gate, scale, eps, checkpoint):
        ctx.set_materialize_grads(False)
        if b is not None:
            _check_rows(x.shape[:-1], b.shape[:-1], "stream and branch")
        x2, b2 = _rows(x), None if b is None else _rows(b)
        T, d, dev, dt = x2.shape[0], x2.shape[1], x.device, x.dtype
        checkpoint = checkpoint and any(ctx.needs_input_grad)
        h, rstd = torch.empty(T, d, dtype=dt, device=dev), torch.empty(T, dtype=torch.float32, device=dev)
        s = None if b is None else torch.empty(T, d, dtype=dt, device=dev)
        rstd_b = None if w_post is None else torch.empty(T, dtype=torch.float32, device=dev)
        reads_b = w_post is not None or (gate is not None and gate.requires_grad)
        sq = s_exp = bq = b_exp = None
        if checkpoint:
            sq, s_exp = _codes(T, d, dev)
            if reads_b:
                bq, b_exp = _codes(T, d, dev)
        _b.norm_fwd(x2, w, h, rstd, b=b2, s=s, scale=scale, gate=gate, w_post=w_post, rstd_b=rstd_b, sq=sq, s_exp=s_exp, bq=bq, b_exp=b_exp, eps=eps)
        saved_s = sq if checkpoint else x2 if s is None else s
        saved_b = None if not reads_b else bq if checkpoint else b2
        ctx.save_for_backward(saved_s, s_exp, saved_b, b_exp, rstd, rstd_b, w, w_post, gate, tie := _tie(x))
        ctx.scale, ctx.shape, ctx.branch = scale, x.shape, None if b is None else b.shape
        h = h.reshape(x.shape)
        return (h, tie) if s is None else (s.reshape(x.shape), h, tie)

    @staticmethod
    @_first_order
    def backward(ctx, *grads):
        ds, dh = (None, grads[0]) if ctx.branch is None else grads
        s, s_exp, b, b_exp, rstd, rstd_b, w, w_post, gate, _ = ctx.saved_tensors
        T, d, dev = s.shape[0], s.shape[1], s.device
        dh2 = torch.zeros(T, d, dtype=w.dtype, device=dev) if dh is None else _rows(dh)
        ds2 = None if ds is None else _rows(ds)
        need = ctx.needs_input_grad
        dx = torch.empty(T, d, dtype=w.dtype, device=dev)
        db = torch.empty(T, d, dtype=w.dtype, device=dev) if need[1] else None
        new = lambda on: torch.empty(d, dtype=torch.float32, device=dev) if on else None  # noqa: E731
        dw, dw_post, dgate = new(need[2]), new(need[3]), new(need[4])
        ws = torch.empty(_b.norm_workspace_bytes(T, d), dtype=_U8, device=dev) if need[2] or need[3] or need[4] else None
        _b.norm_bwd(dh2, s, w, rstd, dx, ds=ds2, b=b, db=db, scale=ctx.scale, gate=gate, w_post=w_post, rstd_b=rstd_b, s_exp=s_exp, b_exp=b_exp, dw=dw,
                    dw_post=dw_post, dgate=dgate, ws=ws)
        of = lambda v, p: None if v is None else v.to(p.dtype)  # noqa: E731
        return (dx.reshape(ctx.shape), None if db is None else db.reshape(ctx.branch), of(dw, w), of(dw_post, w_post), of(dgate, gate), None, None, None)


class BlockNorm(torch.nn.Module):
    """Joins a branch to the residual stream and normalizes the stream:  stream, h = norm(x, branch).

    s = x + scale * gate * u with u the branch, or with `post_norm` RMSNorm(branch); h = RMSNorm(s).  Without a branch s is x.
    `checkpoint` keeps the backward pass's inputs, where there is to be one, in 8 bits.  Weights are trained if `trainable`."""

    def __init__(self, d: int, post_norm: bool = False, gate: bool = False, scale: float = 1.0, eps: float = 1e-5, checkpoint: bool = True, trainable: bool = False,
                 dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        ones = lambda: torch.nn.Parameter(torch.ones(d, dtype=dtype, device=device), requires_grad=trainable)  # noqa: E731
        self.weight = ones()
        self.post_weight = ones() if post_norm else None
        self.gate = ones() if gate else None
        self.scale, self.eps, self.checkpoint = scale, eps, checkpoint

    def forward(self, x: torch.Tensor, branch: Optional[torch.Tensor] = None):
        keeps = self.checkpoint and torch.is_grad_enabled()
        if branch is None:
            return x, _NormFn.apply(x, None, self.weight, None, None, 1.0, self.eps, keeps)[0]
        return _NormFn.apply(x, branch, self.weight, self.post_weight, self.gate, self.scale, self.eps, keeps)[:2]


class _SwigluFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, u, checkpoint):
        ctx.set_materialize_grads(False)
        _check_rows(g.shape[:-1], u.shape[:-1], "gate and up")
        g2, u2 = _rows(g), _rows(u)
        T, m = g2.shape
        checkpoint = checkpoint and any(ctx.needs_input_grad)
        h = torch.empty(T, m, dtype=g.dtype, device=g.device)
        gq = g_exp = uq = u_exp = None
        if checkpoint:
            (gq, g_exp), (uq, u_exp) = _codes(T, m, g.device), _codes(T, m, g.device)
        _b.swiglu_fwd(g2, u2, h, gq=gq, g_exp=g_exp, uq=uq, u_exp=u_exp)
        ctx.save_for_backward(gq if checkpoint else g2, uq if checkpoint else u2, g_exp, u_exp, tie := _tie(g))
        ctx.up = u.shape
        return h.reshape(g.shape), tie

    @staticmethod
    @_first_order
    def backward(ctx, dh):
        g, u, g_exp, u_exp, _ = ctx.saved_tensors
        dh2 = _rows(dh)
        dg, du = (torch.empty(dh2.shape, dtype=dh.dtype, device=dh.device) for _ in range(2))
        _b.swiglu_bwd(dh2, g, u, dg, du, g_exp=g_exp, u_exp=u_exp)
        return dg.reshape(dh.shape), du.reshape(ctx.up), None


def swiglu(g: torch.Tensor, u: torch.Tensor, checkpoint: bool = True) -> torch.Tensor:
    """silu(g) * u; with `checkpoint`, g and u are kept for the backward pass in 8 bits."""
    return _SwigluFn.apply(g, u, checkpoint and torch.is_grad_enabled())[0]


class _TokenLogprobFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels):
        ctx.set_materialize_grads(False)
        _check_rows(logits.shape[:-1], labels.shape, "logits and labels")
        x = logits.reshape(-1, logits.shape[-1])
        apart = (x.shape[1] == 1 or x.stride(1) == 1) and (x.shape[0] == 1 or x.stride(0) >= x.shape[1])
        x = x if apart else x.contiguous()
        T, V = x.shape
        logp, lse, low = (torch.empty(T, dtype=torch.float32, device=x.device) for _ in range(3))
        l2 = labels.reshape(-1).contiguous()
        _b.token_logprob(x, l2, logp, lse, torch.empty(_b.logprob_workspace_bytes(T, V), dtype=_U8, device=x.device), lse_low=low)
        ctx.save_for_backward(x, l2, lse, low, tie := _tie(x))
        ctx.shape = logits.shape
        return logp.reshape(labels.shape), tie

    @staticmethod
    @_first_order
    def backward(ctx, d_logp):
        x, labels, lse, low, _ = ctx.saved_tensors
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _b.token_logprob_bwd(d_logp.reshape(-1).contiguous(), x, labels, lse, dx, lse_low=low)
        return dx.reshape(ctx.shape), None


def token_logprobs(logits: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
    """log softmax(logits)[label] for logits [..., V] and int64 labels [...], fp32; labels outside the vocabulary (-100) give 0."""
    return _TokenLogprobFn.apply(logits, labels)[0]


class _PreferenceFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, ref_logp, offsets, beta, smoothing):
        ctx.set_materialize_grads(False)
        p2, r2 = logp.reshape(-1).contiguous(), ref_logp.reshape(-1).contiguous()
        T, P, dev = p2.shape[0], (offsets.shape[0] - 1) // 2, logp.device
        loss, rewards, d = (torch.empty(s, dtype=torch.float32, device=dev) for s in (1, (2, P), T))
        _b.preference_loss(p2, r2, offsets, loss, rewards, d, torch.empty(_b.logprob_workspace_bytes(T, 1, P), dtype=_U8, device=dev), beta=beta, smoothing=smoothing)
        ctx.save_for_backward(d, tie := _tie(d))
        ctx.shape = logp.shape
        ctx.mark_non_differentiable(rewards)
        return loss[0], rewards, tie

    @staticmethod
    @_first_order
    def backward(ctx, d_loss, d_rewards):
        d, _ = ctx.saved_tensors
        return (d * d_loss).reshape(ctx.shape), None, None, None, None


def preference_loss(logp: torch.Tensor, ref_logp: torch.Tensor, offsets: torch.Tensor, beta: float = 0.1, smoothing: float = 0.0):
    """Loss and rewards [2, P] of the sequences that `offsets` (int64 [2 P + 1], on the GPU) cuts the tokens into: chosen, then rejected."""
    return _PreferenceFn.apply(logp, ref_logp, offsets, beta, smoothing)[:2]


def _mx4(t: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """4-bit codes and exponents of a matrix."""
    t2 = _rows(t)
    q, e = (torch.empty(s, dtype=_U8, device=t.device) for s in _b.mx_shapes(t2.shape[0], t2.shape[1], _b.MX_E2M1))
    _b.mx_quantize(t2, _b.MX_E2M1, q, e)
    return q, e


def _mx4_product(x2, wq, w_exp, m, codes=None):
    """x2 [T, n] through codes [m, n / 2]; `codes`: those of x2, where another layer has formed them.  Returns y and the codes of x2."""
    T, n = (x2.shape if x2 is not None else (codes[0].shape[0], codes[0].shape[1] * 2))
    dev = wq.device
    xq, x_exp = codes or (torch.empty(s, dtype=_U8, device=dev) for s in _b.mx_shapes(T, n, _b.MX_E2M1))
    y = torch.empty(T, m, dtype=torch.bfloat16, device=dev)
    _b.mx4_linear(None if codes else x2, wq, w_exp, xq, x_exp, y)
    return y, (xq, x_exp)


class _Mx4Fn(torch.autograd.Function):
    """Linear layers of one input: it is quantized once."""

    @staticmethod
    def forward(ctx, x, *layers):
        x2 = _dense_bf16(x, x.shape[-1])
        outs, codes = [], None
        for l in layers:
            y, codes = _mx4_product(x2, l.wq, l.w_exp, l.out_features, codes)
            outs.append(y.reshape(*x.shape[:-1], l.out_features))
        ctx.layers, ctx.shape, ctx.dtype = layers, x.shape, x.dtype
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(tie := _tie(x))
        return (*outs, tie)

    @staticmethod
    @_first_order
    def backward(ctx, *dys):
        if not ctx.needs_input_grad[0]:
            return (None,) * (1 + len(ctx.layers))
        total = None
        for l, dy in zip(ctx.layers, dys):
            if dy is None:
                continue
            if l.wtq is None:
                raise RuntimeError("this layer was built without input_grad=True, so it holds no codes of its transposed weight")
            dx, _ = _mx4_product(_dense_bf16(dy, l.out_features), l.wtq, l.wt_exp, l.in_features)
            total = dx if total is None else total.add_(dx)
        return (None if total is None else total.to(ctx.dtype).reshape(ctx.shape),) + (None,) * len(ctx.layers)


class Mx4Linear(torch.nn.Module):
    """Frozen linear layer on 4-bit microscaled codes (17/32 of a byte for each weight): a reference model, or generation.

    `input_grad` also keeps the codes of the transposed weight, on which the gradient of the input is formed."""

    def __init__(self, weight: torch.Tensor, input_grad: bool = False):
        super().__init__()
        m, n = weight.shape
        if n % 32 or m % (32 if input_grad else 16):
            raise ValueError(f"{m} x {n}: the input width is a multiple of 32, the output width of 16, or of 32 with input_grad")
        self.in_features, self.out_features = n, m
        w = weight.detach()
        w = w if w.dtype in (torch.float32, torch.bfloat16) else w.float()
        wq, w_exp = _mx4(w)
        self.register_buffer("wq", wq)
        self.register_buffer("w_exp", w_exp)
        wtq, wt_exp = _mx4(w.t().contiguous()) if input_grad else (None, None)
        self.register_buffer("wtq", wtq)
        self.register_buffer("wt_exp", wt_exp)

    @classmethod
    def from_melded(cls, layer: MeldedLoRALinear, input_grad: bool = False) -> "Mx4Linear":
        """The melded weight as it is now (its FP8 codes over their scale)."""
        w = layer.wq[: layer.out_features].view(torch.float8_e4m3fn).float() / layer.s_w
        return cls(w, input_grad)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return _Mx4Fn.apply(x, self)[0]


class Mx4Group:
    """4-bit layers with a common input, which is quantized once.  `group(x)` returns one output per layer."""

    def __init__(self, *layers: Mx4Linear):
        if not layers or any(l.in_features != layers[0].in_features for l in layers):
            raise ValueError("a group needs layers of one input width")
        self.layers = list(layers)

    def __call__(self, x: torch.Tensor):
        return _Mx4Fn.apply(x, *self.layers)[:-1]


def _group(layers: Sequence[torch.nn.Module]):
    if all(isinstance(l, MeldedLoRALinear) for l in layers):
        return MeldedGroup(*layers)
    if all(isinstance(l, Mx4Linear) for l in layers):
        return Mx4Group(*layers)
    return lambda x: tuple(l(x) for l in layers)


class FusedBlock(torch.nn.Module):
    """LLaMA decoder block that hands on the residual stream and the branch that has not joined it yet:  x, branch = block(x, branch).

    The next norm joins the two, so neither the sum nor the norm is a pass of its own; `BlockNorm` behind the last block does the same.
    `linear(in, out)` builds a projection (melded, 4-bit, or any other); norms as in `BlockNorm`."""

    def __init__(self, d_model: int, n_heads: int, d_mlp: int, linear, device="cuda", checkpoint: bool = True, **norm):
        super().__init__()
        self.n_heads, self.checkpoint = n_heads, checkpoint
        self.norm1, self.norm2 = (BlockNorm(d_model, checkpoint=checkpoint, device=device, **norm) for _ in range(2))
        self.q, self.k, self.v, self.o = (linear(d_model, d_model) for _ in range(4))
        self.gate, self.up = linear(d_model, d_mlp), linear(d_model, d_mlp)
        self.down = linear(d_mlp, d_model)

    def forward(self, x: torch.Tensor, branch: Optional[torch.Tensor] = None):
        B, S, D = x.shape
        x, h = self.norm1(x, branch)
        q, k, v = (t.reshape(B, S, self.n_heads, D // self.n_heads).transpose(1, 2) for t in _group((self.q, self.k, self.v))(h))
        a = torch.nn.functional.scaled_dot_product_attention(q, k, v, is_causal=True)
        x, h = self.norm2(x, self.o(a.transpose(1, 2).reshape(B, S, D)))
        gate, up = _group((self.gate, self.up))(h)
        return x, self.down(swiglu(gate, up, self.checkpoint))

    def projections(self):
        return [self.q, self.k, self.v, self.o, self.gate, self.up, self.down]


class FusedDecoder(torch.nn.Module):
    """Embedding, blocks, final norm and head: logits of token ids [B, S].  Embedding and head are frozen.  Whole sequences only: no keys and values are
    kept, so a one-token step (which the norms and the 4-bit layers have forms for) is that of a model with a cache of its own."""

    def __init__(self, embedding: torch.Tensor, head: torch.Tensor, blocks: Sequence[FusedBlock], final: BlockNorm):
        super().__init__()
        self.register_buffer("embedding", embedding)
        self.register_buffer("head", head)
        self.blocks, self.final = torch.nn.ModuleList(blocks), final

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        x, branch = torch.nn.functional.embedding(tokens, self.embedding), None
        for block in self.blocks:
            x, branch = block(x, branch)
        return torch.nn.functional.linear(self.final(x, branch)[1], self.head)


def _next_labels(tokens: torch.Tensor, prompt_lengths: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
    """What a position predicts: the next token, where that is of the answer; -100 elsewhere."""
    at = torch.arange(tokens.shape[1], device=tokens.device) + 1
    labels = torch.cat([tokens[:, 1:], torch.full_like(tokens[:, :1], -100)], 1)
    return torch.where((at >= prompt_lengths[:, None]) & (at < lengths[:, None]), labels, torch.full_like(labels, -100))


def preference_step(policy, reference, tokens: torch.Tensor, prompt_lengths: torch.Tensor, lengths: torch.Tensor, beta: float = 0.1, smoothing: float = 0.0):
    """Loss and rewards of pairs: tokens [2 P, S] (chosen answers first, rows filled up with anything), of which row i has `lengths[i]`, the first
    `prompt_lengths[i]` its prompt's.  Call backward() on the loss, then an optimizer."""
    labels = _next_labels(tokens, prompt_lengths, lengths)
    inside = torch.arange(tokens.shape[1], device=tokens.device) < lengths[:, None]
    tokens = torch.where(inside, tokens, torch.zeros_like(tokens))              # an embedding looks up what rows are filled up with, too
    with torch.no_grad():
        ref = token_logprobs(reference(tokens), labels)
    logp = token_logprobs(policy(tokens), labels)
    rows, S = tokens.shape
    offsets = torch.arange(rows + 1, device=tokens.device) * S
    return preference_loss(logp, ref, offsets, beta, smoothing)
