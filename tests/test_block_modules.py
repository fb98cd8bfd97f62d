"""Modules and functions around the melded layers on the CPU: what they hand to the library's calls, which are replaced here by plain torch forms."""
import pytest
import torch

from paper_2510_24061_amd import block


class Calls:
    """Plain forms of the calls, with the binding's checks of shapes, and a record of what was asked for."""

    MX_E2M1 = 1

    def __init__(self):
        self.asked = []

    def norm_workspace_bytes(self, T, d):
        return 16

    def logprob_workspace_bytes(self, T, V, P=1):
        return 16

    def norm_fwd(self, x, w, h, rstd, b=None, s=None, scale=1.0, gate=None, w_post=None, rstd_b=None, sq=None, s_exp=None, bq=None, b_exp=None, eps=1e-5):
        self.asked.append(("norm_fwd", sq is not None, bq is not None))
        v = x.float()
        if b is not None:
            assert b.shape == x.shape
            u = b.float()
            if w_post is not None:
                rstd_b.copy_((u.square().mean(1) + eps).rsqrt())
                u = u * rstd_b[:, None] * w_post.float()
            v = v + scale * u * (1.0 if gate is None else gate.float())
            s.copy_(v)
        rstd.copy_((v.square().mean(1) + eps).rsqrt())
        h.copy_(v * rstd[:, None] * w.float())

    def norm_bwd(self, dh, s, w, rstd, dx, ds=None, b=None, db=None, scale=1.0, gate=None, w_post=None, rstd_b=None, s_exp=None, b_exp=None, dw=None, dw_post=None,
                 dgate=None, ws=None):
        self.asked.append(("norm_bwd", dh, ds))
        hat = s.float() * rstd[:, None]
        g = w.float() * dh.float()
        dx.copy_(rstd[:, None] * (g - hat * (g * hat).mean(1, keepdim=True)) + (0.0 if ds is None else ds.float()))
        if db is not None:
            db.copy_(scale * dx.float())
        if dw is not None:
            dw.copy_((dh.float() * hat).sum(0))

    def swiglu_fwd(self, g, u, h, gq=None, g_exp=None, uq=None, u_exp=None):
        assert g.shape == u.shape == h.shape
        self.asked.append(("swiglu_fwd", gq is not None, g.data_ptr() % 16 == 0 and u.data_ptr() % 16 == 0))
        h.copy_(torch.nn.functional.silu(g.float()) * u.float())

    def swiglu_bwd(self, dh, g, u, dg, du, g_exp=None, u_exp=None):
        s = torch.sigmoid(g.float())
        dg.copy_(dh.float() * u.float() * s * (1 + g.float() * (1 - s)))
        du.copy_(dh.float() * g.float() * s)

    def token_logprob(self, logits, labels, logp, lse, ws, lse_low=None):
        assert logits.stride(0) >= logits.shape[1] or logits.shape[0] == 1
        assert labels.shape == logp.shape == (logits.shape[0],)
        counts = (labels >= 0) & (labels < logits.shape[1])
        lse.copy_(torch.logsumexp(logits.float(), 1) * counts)
        logp.copy_((logits.float().gather(1, labels.clamp(0, logits.shape[1] - 1)[:, None])[:, 0] - lse) * counts)
        if lse_low is not None:
            lse_low.zero_()

    def token_logprob_bwd(self, d_logp, logits, labels, lse, dlogits, lse_low=None):
        p = torch.softmax(logits.float(), 1).neg()
        p[torch.arange(len(labels)), labels] += 1.0
        dlogits.copy_(d_logp[:, None] * p)

    def preference_loss(self, logp, ref_logp, offsets, loss, rewards, d_logp, ws, beta=0.1, smoothing=0.0):
        assert all(t.dtype == torch.float32 for t in (logp, ref_logp, loss, rewards, d_logp))
        o, P = offsets.tolist(), rewards.shape[1]
        with torch.enable_grad():
            p = logp.detach().requires_grad_()
            r = beta * torch.stack([(p[a:b] - ref_logp[a:b]).sum() for a, b in zip(o, o[1:])]).reshape(2, P)
            value = torch.nn.functional.softplus(r[1] - r[0]).mean()
            d_logp.copy_(torch.autograd.grad(value, p)[0])
        loss.fill_(value.item())
        rewards.copy_(r.detach())


for _name in ("norm_fwd", "norm_bwd", "swiglu_fwd", "swiglu_bwd", "token_logprob", "token_logprob_bwd", "preference_loss"):
    setattr(Calls, _name, torch.no_grad()(getattr(Calls, _name)))               # autograd does not see a kernel's work


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(block, "_b", c)
    return c


def norm(d, **kw):
    return block.BlockNorm(d, dtype=torch.float32, device="cpu", **kw)


# ---- derivatives of the derivatives ---------------------------------------------------------------------------------------------
def first_order(name):
    """(differentiable inputs, output) of one of the functions"""
    g = torch.Generator().manual_seed(1)
    t = lambda *s: torch.randn(*s, generator=g, requires_grad=True)  # noqa: E731
    if name == "norm":
        x, b = t(3, 32), t(3, 32)
        return (x, b), norm(32, checkpoint=False)(x, b)[1].sum()
    if name == "swiglu":
        x, y = t(3, 32), t(3, 32)
        return (x, y), block.swiglu(x, y, checkpoint=False).sum()
    if name == "logprobs":
        x = t(3, 7)
        return (x,), block.token_logprobs(x, torch.tensor([1, 2, 3])).sum()
    if name == "loss":
        x = t(6)
        return (x,), block.preference_loss(x, torch.zeros(6), torch.tensor([0, 3, 6]))[0]
    x = t(3, 32)
    layer = block.Mx4Linear.__new__(block.Mx4Linear)
    torch.nn.Module.__init__(layer)
    layer.in_features, layer.out_features = 32, 16
    layer.wq, layer.w_exp, layer.wtq, layer.wt_exp = (torch.zeros(1) for _ in range(4))
    return (x,), layer(x).float().square().sum()


@pytest.mark.parametrize("name", ["norm", "swiglu", "logprobs", "loss", "mx4"])
@pytest.mark.parametrize("through_loss", [False, True])
def test_a_second_derivative_is_refused(calls, monkeypatch, name, through_loss):
    """Under create_graph the first derivatives come as before; a penalty on them is refused, not dropped (plain forms beside it count as ever)."""
    monkeypatch.setattr(block, "_mx4_product", lambda x2, wq, w_exp, m, codes=None: (torch.ones(3, m, dtype=torch.bfloat16), (x2, None)))
    inputs, out = first_order(name)
    plain = torch.autograd.grad(out, inputs, retain_graph=True)
    value = out.square() if through_loss else out
    grads = torch.autograd.grad(value, inputs, create_graph=True)
    factor = 2 * out.detach() if through_loss and name != "mx4" else 1.0       # the product's stand-in gives ones
    assert all(torch.allclose(a, b * factor) and a.requires_grad for a, b in zip(grads, plain))
    own = inputs[0].square().sum()
    with pytest.raises(RuntimeError, match="differentiat"):
        torch.autograd.grad(own + sum(v.square().sum() for v in grads), inputs)


def test_create_graph_without_a_second_derivative(calls):
    x, y = torch.randn(2, 32, requires_grad=True), torch.randn(2, 32, requires_grad=True)
    block.swiglu(x, y, checkpoint=False).sum().backward(create_graph=True)
    want = torch.autograd.grad((torch.nn.functional.silu(x) * y).sum(), (x, y))
    assert torch.allclose(x.grad, want[0], atol=1e-6) and torch.allclose(y.grad, want[1], atol=1e-6)


def test_only_what_is_asked_for(calls):
    """An input without a gradient gets none, also where the other has one."""
    x, y = torch.randn(2, 32, requires_grad=True), torch.randn(2, 32)
    g, = torch.autograd.grad(block.swiglu(x, y, checkpoint=False).sum(), x, create_graph=True)
    assert g.shape == x.shape and y.grad is None


def test_loss_under_another_default_type(calls):
    """The loss's buffers are fp32 whatever torch's default is."""
    kept = torch.get_default_dtype()
    torch.set_default_dtype(torch.bfloat16)
    try:
        loss, rewards = block.preference_loss(torch.zeros(6, dtype=torch.float32), torch.zeros(6, dtype=torch.float32), torch.tensor([0, 3, 6]))
    finally:
        torch.set_default_dtype(kept)
    assert loss.dtype == rewards.dtype == torch.float32


# ---- checkpoints ------------------------------------------------------------------------------------------------------------------
def test_checkpoints_are_written_where_a_backward_pass_reads_them(calls):
    n = norm(32, post_norm=True)
    x, y = torch.randn(3, 32), torch.randn(3, 32)
    run = lambda x, y: (n(x, y), n(x), block.swiglu(x, y), [a[1] for a in calls.asked if a[0].endswith("fwd")], calls.asked.clear())[3]  # noqa: E731
    assert run(x.requires_grad_(), y) == [True, True, True]
    assert run(x, y.requires_grad_()) == [True, True, True]
    assert run(x.detach(), y) == [True, False, True]                            # what depends on y
    assert run(x.detach(), y.detach()) == [False, False, False]                 # no input needs a gradient
    with torch.no_grad():
        assert run(x, y) == [False, False, False]
    with torch.inference_mode():
        assert run(x, y) == [False, False, False]
    n.weight.requires_grad_()
    assert run(x.detach(), y.detach()) == [True, True, False]                   # a norm's weight is trained


# ---- shapes and memory ------------------------------------------------------------------------------------------------------------
def test_logits_whose_rows_lie_over_each_other(calls):
    row = torch.randn(1, 9)
    x = row.expand(4, 9)                                                        # one row four times, without memory of its own
    labels = torch.tensor([0, 3, 8, -100])
    want = torch.log_softmax(row, 1)[0, labels.clamp(min=0)] * (labels >= 0)
    assert torch.allclose(block.token_logprobs(x, labels), want)
    row.requires_grad_()
    block.token_logprobs(row.expand(4, 9), torch.tensor([0, 3, 8, 1])).sum().backward()
    want = -4 * torch.softmax(row.detach(), 1)
    want[0, [0, 3, 8, 1]] += 1.0
    assert torch.allclose(row.grad, want, atol=1e-6)
    sliding = torch.randn(12).unfold(0, 9, 1)                                   # rows one element apart
    assert torch.allclose(block.token_logprobs(sliding, labels), torch.log_softmax(sliding, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0] * (labels >= 0))


def test_dense_inputs_off_the_16_byte_boundaries(calls, monkeypatch):
    """A dense view that begins anywhere is copied: contiguous() would hand back the same memory."""
    flat = torch.randn(2, 1 + 3 * 32)
    g, u = (f[1:].view(3, 32) for f in flat)
    if g.data_ptr() % 16 == 0:
        g, u = (f[:-1].view(3, 32) for f in flat)
    assert g.is_contiguous() and g.data_ptr() % 16
    out = block.swiglu(g, u)
    assert calls.asked[-1][2] and torch.allclose(out, torch.nn.functional.silu(g) * u, atol=1e-6)
    seen = []
    monkeypatch.setattr(block, "_mx4_product", lambda x2, wq, w_exp, m, codes=None: (seen.append(x2), (torch.ones(3, m, dtype=torch.bfloat16), None))[1])
    layer = first_layer()
    half = torch.randn(1 + 3 * 32).bfloat16()[1:].view(3, 32).requires_grad_()
    assert half.data_ptr() % 16
    y = layer(half)
    y.backward(torch.randn(1 + 3 * 16).bfloat16()[1:].view(3, 16))
    assert len(seen) == 2 and all(t.is_contiguous() and t.data_ptr() % 16 == 0 for t in seen) and torch.equal(seen[0], half)


def first_layer():
    layer = block.Mx4Linear.__new__(block.Mx4Linear)
    torch.nn.Module.__init__(layer)
    layer.in_features, layer.out_features = 32, 16
    layer.wq, layer.w_exp, layer.wtq, layer.wt_exp = (torch.zeros(1) for _ in range(4))
    return layer


@pytest.mark.parametrize("x,y", [((2, 3, 32), (3, 2, 32)), ((2, 1, 32), (1, 2, 32)), ((4, 32), (2, 2, 2, 16)), ((2, 2, 3, 32), (4, 3, 32))])
def test_inputs_of_different_shapes_are_refused(calls, x, y):
    """As many rows in another order are not the same rows."""
    a, b = torch.randn(x), torch.randn(y)
    with pytest.raises(ValueError):
        norm(32)(a, b)
    with pytest.raises(ValueError):
        block.swiglu(a, b)
    if y[-1] == 32:
        with pytest.raises(ValueError):
            block.token_logprobs(a, torch.zeros(y[:-1], dtype=torch.int64))


@pytest.mark.parametrize("x,y", [((2, 3, 32), (2, 3, 32)), ((1, 6, 32), (6, 32)), ((6, 32), (1, 1, 6, 32)), ((2, 3, 32), (6, 32)), ((6, 32), (2, 3, 32))])
def test_leading_ones_and_flat_rows_are_taken(calls, x, y):
    """The results have the first one's shape, every gradient that of its own input."""
    a, b = torch.randn(x, requires_grad=True), torch.randn(y, requires_grad=True)
    s, h = norm(32, checkpoint=False)(a, b)
    z = block.swiglu(a, b, checkpoint=False)
    assert s.shape == h.shape == z.shape == a.shape
    (s.sum() + h.square().sum() + z.sum()).backward()
    assert a.grad.shape == a.shape and b.grad.shape == b.shape
    a64, b64 = a.detach().double().requires_grad_(), b.detach().double().requires_grad_()
    s64 = a64.reshape(6, 32) + b64.reshape(6, 32)
    h64 = s64 * (s64.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    (s64.sum() + h64.square().sum() + (torch.nn.functional.silu(a64.reshape(6, 32)) * b64.reshape(6, 32)).sum()).backward()
    assert torch.allclose(a.grad.double(), a64.grad, atol=1e-5) and torch.allclose(b.grad.double(), b64.grad, atol=1e-5)
    labels = torch.arange(6).reshape(y[:-1])
    assert torch.allclose(block.token_logprobs(a, labels).reshape(-1), torch.log_softmax(a.reshape(6, 32), 1)[torch.arange(6), torch.arange(6)], atol=1e-5)


# ---- the preference step -----------------------------------------------------------------------------------------------------------
def test_what_rows_are_filled_up_with_reaches_no_embedding(calls):
    """Rows may be filled up with anything: -100, or ids beyond the vocabulary."""
    V, d = 11, 8
    embedding, head = torch.randn(V, d), torch.randn(V, d)
    model = lambda tokens: torch.nn.functional.embedding(tokens, embedding).cumsum(1) @ head.t()  # noqa: E731
    g = torch.Generator().manual_seed(0)
    tokens = torch.randint(0, V, (4, 9), generator=g)
    prompts, lengths = torch.tensor([2, 0, 2, 1]), torch.tensor([9, 5, 1, 7])
    plain = block.preference_step(model, model, tokens, prompts, lengths)
    filled = torch.where(torch.arange(9) < lengths[:, None], tokens, torch.tensor([-100, 10 ** 6, -1, V])[:, None])
    kept = filled.clone()
    loss, rewards = block.preference_step(model, model, filled, prompts, lengths)
    assert torch.equal(loss, plain[0]) and torch.equal(rewards, plain[1]) and torch.equal(filled, kept)
