"""Log-probabilities and gradients of rows whose size is far from their differences: all of one value (the type's lowest among them), and rows whose
label has nearly all of the probability.

Tolerances, element by element.  logp = (x_label - max) - log(sum) does not depend on what is added to the whole row: its error is that of a difference
(2^-24 of it) and of the logarithm of a sum that is off by some 2^-24 in each of the levels of its tree: 64 * 2^-24 of max(1, |logp|).  A probability is
exp(x - lse), whose argument is rounded to 2^-24 of |x - lse| twice: (64 + 4 |x - lse|) 2^-24 of it.  Where only the rounded lse is given, and below 64 in size,
half of its last place is 2^-19 = 32 * 2^-24 at most.  The label's d (1 - p) has a rounding of the difference and one of the product besides, 2^-24 each.
bf16 has eight significant bits: outputs are rounded once, by 2^-8 of themselves at most."""
import math

import pytest
import torch

import paper_2510_24061_amd as fq
from block_ops_common import draw, gen

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
U = 2.0 ** -24


def forward(x, labels):
    T, V = x.shape
    logp, lse, low = (torch.full((T,), float("nan"), device="cuda") for _ in range(3))
    fq.token_logprob(x, labels, logp, lse, torch.full((fq.logprob_workspace_bytes(T, V),), 0xFF, dtype=torch.uint8, device="cuda"), lse_low=low)
    again = [torch.full((T,), float("nan"), device="cuda") for _ in range(2)]
    fq.token_logprob(x, labels, *again, torch.empty(fq.logprob_workspace_bytes(T, V), dtype=torch.uint8, device="cuda"))
    assert torch.equal(logp, again[0]) and torch.equal(lse, again[1])          # asking for the low part changes nothing else
    return logp, lse, low


def softmax64(x, labels):
    x = x.double()
    e = x - x.amax(1, keepdim=True)
    e = e - e.exp().sum(1, keepdim=True).log()
    return e.gather(1, labels[:, None])[:, 0], e                               # of the labels, of all: differences only


def check(x, labels, d, slack=0.0):
    """x [T, V] (CPU): log-probabilities, and gradients with and without the low part, in place too."""
    c, l, dc = x.cuda(), labels.cuda(), d.cuda()
    logp, lse, low = forward(c, l)
    want, e = softmax64(x, labels)
    assert bool(((logp.cpu().double() - want).abs() <= 64 * U * want.abs().clamp(min=1.0)).all())
    p, at = e.exp(), torch.arange(x.shape[0])
    grad = -d.double()[:, None] * p
    grad[at, labels] = d.double() * -torch.expm1(e[at, labels])
    off = (64 + 4 * e.abs()) * U * p
    off[at, labels] += 2 * U * -torch.expm1(e[at, labels])
    once = 2.0 ** -8 * grad.abs() if x.dtype == torch.bfloat16 else 0.0
    for part, more in ((low, 0.0), (None, 32 * U)):
        out = torch.full_like(c, float("nan"))
        fq.token_logprob_bwd(dc, c, l, lse, out, lse_low=part)
        bound = d.abs().double()[:, None] * (off + more * p) * (1 + 2.0 ** -8) + once + 2.0 ** -126
        bad = (out.cpu().double() - grad).abs() > bound
        assert not bad.any(), (part is not None, torch.nonzero(bad)[:4], out.cpu()[bad][:4], grad[bad][:4])
        over = c.clone()
        fq.token_logprob_bwd(dc, over, l, lse, over, lse_low=part)
        assert torch.equal(over, out)
        apart = torch.full((x.shape[0], x.shape[1] + 3), 7.0, dtype=x.dtype, device="cuda")
        fq.token_logprob_bwd(dc, c, l, lse, apart[:, 1:1 + x.shape[1]], lse_low=part)
        assert torch.equal(apart[:, 1:1 + x.shape[1]], out) and bool((apart[:, 0] == 7.0).all()) and bool((apart[:, 1 + x.shape[1]:] == 7.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 1000, 8200, 32001, 131072])
def test_rows_of_one_value(V, dtype):
    """Probabilities of 1 / V, whatever the value: the type's lowest and largest (a mask over everything), and ordinary ones."""
    info = torch.finfo(dtype)
    values = [info.min, info.max, 0.0, 30.0, -1e4, 3e4, 1e30, 63.0, 65.0, -200.0]
    x = torch.tensor(values).to(dtype)[:, None].repeat(1, V)
    labels = torch.arange(len(values)) * 7919 % V
    check(x, labels, draw(gen(V), len(values)))
    logp, _, _ = forward(x.cuda(), labels.cuda())
    assert float((logp.cpu().double() + math.log(V)).abs().max()) <= 64 * U * max(1.0, math.log(V))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [50, 1000, 32001])
@pytest.mark.parametrize("offset", [0.0, 30.0, 5000.0])
def test_confident_rows_far_from_zero(V, dtype, offset):
    """The label has all but 1e-6 or so of the probability: logp near -1e-6, and a gradient whose label's part is the others' sum."""
    T = 9
    x = draw(gen(V), T, V).to(dtype).float()
    labels = torch.arange(T) * 31 % V
    x = x + offset
    x[torch.arange(T), labels] = offset + math.log(V) + 14.0 + torch.arange(T) * 0.125
    check(x.to(dtype), labels, draw(gen(5), T))


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_rows_beside_ordinary_ones(dtype):
    """Many rows, one in three of nothing but the type's lowest value, labels that do not count among them."""
    T, V = 600, 4099
    x = draw(gen(1), T, V, std=2.0).to(dtype)
    x[::3] = torch.finfo(dtype).min
    x[1::9, : V // 2] = torch.finfo(dtype).min
    labels = torch.randint(V // 2 + 1, V, (T,), generator=gen(2))
    check(x, labels, draw(gen(3), T))
    none = labels.clone()
    none[::2] = -100
    logp, lse, low = forward(x.cuda(), none.cuda())
    assert not logp[::2].any() and not lse[::2].any() and not low[::2].any()
    out = torch.full_like(x, float("nan")).cuda()
    fq.token_logprob_bwd(draw(gen(3), T).cuda(), x.cuda(), none.cuda(), lse, out)
    assert not out[::2].any() and out.isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_rows_have_no_low_part(dtype):
    x = torch.zeros(4, 300, dtype=dtype)
    x[0] = -float("inf")
    x[1, 5], x[2, 5] = float("inf"), float("nan")
    logp, lse, low = forward_any(x, torch.zeros(4, dtype=torch.int64))
    assert float(lse[0]) == -float("inf") and lse[1].isnan() and lse[2].isnan() and not low[:3].any()
    out = torch.full_like(x, 7.0).cuda()
    fq.token_logprob_bwd(torch.ones(4, device="cuda"), x.cuda(), torch.zeros(4, dtype=torch.int64, device="cuda"), lse, out, lse_low=low)
    assert not out[0].any() and out[1].isnan().all() and out[2].isnan().all() and out[3].isfinite().all()


def forward_any(x, labels):
    T, V = x.shape
    out = [torch.full((T,), float("nan"), device="cuda") for _ in range(3)]
    fq.token_logprob(x.cuda(), labels.cuda(), out[0], out[1], torch.empty(fq.logprob_workspace_bytes(T, V), dtype=torch.uint8, device="cuda"), lse_low=out[2])
    return out


def test_autograd_of_a_masked_row():
    from paper_2510_24061_amd.block import token_logprobs
    V = 777
    x = torch.zeros(2, 3, V, device="cuda")
    x[0, 1] = torch.finfo(torch.float32).min
    x[1, 2, 5] = 40.0
    x.requires_grad_()
    labels = torch.full((2, 3), 5, device="cuda")
    logp = token_logprobs(x, labels)
    logp.sum().backward()
    logp = logp.detach()
    want = torch.softmax(x.detach().cpu().double(), -1).neg()
    want[..., 5] += 1.0
    assert abs(float(logp[0, 1]) + math.log(V)) <= 64 * U * math.log(V)
    assert bool(((x.grad.cpu().double() - want).abs() <= 128 * U * want.abs() + 64 * U * (want[..., 5:6].abs() < 1e-3)).all())


def test_refusals():
    x, labels = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    out, ws = [torch.empty(4, device="cuda") for _ in range(3)], torch.empty(64, dtype=torch.uint8, device="cuda")
    for low in (out[2][:3], out[2].double(), out[2].cpu()):
        with pytest.raises(ValueError):
            fq.token_logprob(x, labels, out[0], out[1], ws, lse_low=low)
        with pytest.raises(ValueError):
            fq.token_logprob_bwd(out[0], x, labels, out[1], x.clone(), lse_low=low)
