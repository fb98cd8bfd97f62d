"""Norms and SwiGLU element by element, against 64 bits: one wrong element of a tensor does not hide in its norm.  Among the shapes are those with several
rows side by side in a workgroup of the norms' backward pass and more than one turn of its row loop, the last turn filled in part.

Bounds.  U = 2^-24; a bf16 output is rounded once, by 2^-8 of itself at most (eight significant bits).  A row's sum in fp32 goes through at most 16 terms a lane
and 10 levels of a tree, each term with a few roundings of its own: 64 U of the sum of absolute terms covers it, and what is formed of it.  With A = mean |w dh s^|:
  h: 64 U |h|;  s: 64 U (|x| + |scale gate u|);  dx: e = 64 U (|ds| + rstd (|w dh| + |s^| A))
  du = scale gate dx carries |scale gate| (e + 4 U |dx|) =: e'; db behind a norm carries rstd_b (|w_post| e' + |b^| mean(|w_post b^| e')) and its own sum's 64 U
  dw: (T + 64) U sum |terms|;  dw_post and dgate: that, and their terms' share of e' and e
SwiGLU: sigma is 1 / (1 + 2^(-g log2 e)), its argument rounded twice: (|g| + 8) 2^-22 of it; the products add 4 U each."""
import pytest
import torch

import paper_2510_24061_amd as fq
from block_ops_common import mx_values, norm_bwd64, norm_fwd64
from test_gpu_norm import DTYPES, FORMS, backward, cuda, draw, forward, gen, make
from test_gpu_swiglu import forward as swiglu_forward
from test_gpu_swiglu import make as swiglu_make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SCALE = 0.5


def once(v, dtype):
    return 2.0 ** -8 * v.abs() if dtype == torch.bfloat16 else 0.0


def within(got, want, bound, what):
    off = (got.detach().cpu().double() - want).abs()
    bad = ~(off <= bound + 2.0 ** -126)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist(), float((off / (bound + 2.0 ** -126)).max()))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", [(5001, 272), (1999, 528), (4099, 1040), (9001, 80), (2050, 2064), (515, 4096), (3, 16), (521, 8208), (517, 16384)])
def test_norms(T, d, dtype, form, codes):
    t = make(T, d, dtype, **form)
    c = cuda(t)
    f = forward(c, codes=codes)
    want = norm_fwd64(t["x"], t["w"], t["b"], SCALE, t["gate"], t["w_post"], dtype=dtype)
    branch, post = form["branch"], form["post"]
    coef = torch.full((d,), SCALE, dtype=torch.float64) * (1.0 if t["gate"] is None else t["gate"].double())
    s = f["s"].cpu() if branch else t["x"]
    if branch:
        u = t["b"].double() * ((want["rstd_b"][:, None] * t["w_post"].double()) if post else 1.0)
        within(s, t["x"].double() + coef * u, 64 * U * (t["x"].double().abs() + (coef * u).abs()) + once(want["s"], dtype), "s")
    h = norm_fwd64(s, t["w"], dtype=dtype)["h"]
    within(f["h"], h, 64 * U * h.abs() + once(h, dtype), "h")

    g = gen(T)
    dh, ds = draw(g, T, d).to(dtype), draw(g, T, d).to(dtype)
    saved = dict(s=f["sq"] if codes else s.cuda(), s_exp=f.get("s_exp"), b=f.get("bq") if codes else c["b"], b_exp=f.get("b_exp"), rstd=f["rstd"], rstd_b=f["rstd_b"])
    o = backward(c, saved, dh.cuda(), ds.cuda(), codes)
    s64 = mx_values(f["sq"].cpu(), f["s_exp"].cpu(), False) if codes else s.double()
    b64 = None if not branch else mx_values(f["bq"].cpu(), f["b_exp"].cpu(), False) if codes else t["b"].double()
    rb = None if f["rstd_b"] is None else f["rstd_b"].cpu()
    want = norm_bwd64(dh, s64, t["w"], f["rstd"].cpu(), ds, b64, SCALE, t["gate"], t["w_post"], rb)
    r = f["rstd"].cpu().double()[:, None]
    hat, gw = s64 * r, t["w"].double() * dh.double()
    e = 64 * U * (ds.double().abs() + r * (gw.abs() + hat.abs() * (gw * hat).abs().mean(1, keepdim=True)))
    within(o["dx"], want["dx"], e + once(want["dx"], dtype), "dx")
    within(o["dw"], want["dw"], (T + 64) * U * want["dw_terms"], "dw")
    if not branch:
        return
    e1 = coef.abs() * (e + 4 * U * want["dx"].abs())
    if post:
        wp, r2 = t["w_post"].double(), rb.double()[:, None]
        bhat = b64 * r2
        g2 = wp * coef * want["dx"]
        e2 = r2 * (wp.abs() * e1 + bhat.abs() * (wp.abs() * bhat.abs() * e1).mean(1, keepdim=True)) + 64 * U * r2 * (g2.abs() + bhat.abs() * (g2 * bhat).abs().mean(1, keepdim=True))
        within(o["dw_post"], want["dw_post"], (T + 64) * U * want["dw_post_terms"] + (e1 * bhat.abs()).sum(0), "dw_post")
    else:
        e2 = e1
    within(o["db"], want["db"], e2 + once(want["db"], dtype), "db")
    if o.get("dgate") is not None:
        u = b64 * (rb.double()[:, None] * t["w_post"].double()) if post else b64
        within(o["dgate"], want["dgate"], (T + 64) * U * want["dgate_terms"] + SCALE * (e * u.abs()).sum(0), "dgate")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,m", [(1, 16), (37, 688), (1000, 1040), (301, 11008)])
def test_swiglu(T, m, dtype, codes):
    a, b = swiglu_make(T, m, dtype)
    o = swiglu_forward(a.cuda(), b.cuda())
    a64, b64 = a.double(), b.double()
    off = (a64.abs() + 8) * 2.0 ** -22
    h = torch.nn.functional.silu(a64) * b64
    within(o["h"], h, (off + 8 * U) * h.abs() + once(h, dtype), "h")
    dh = draw(gen(T), T, m).to(dtype)
    dg, du = (torch.full((T, m), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    if codes:
        fq.swiglu_bwd(dh.cuda(), o["gq"], o["uq"], dg, du, g_exp=o["g_exp"], u_exp=o["u_exp"])
        a64, b64 = mx_values(o["gq"].cpu(), o["g_exp"].cpu(), False), mx_values(o["uq"].cpu(), o["u_exp"].cpu(), False)
        off = (a64.abs() + 8) * 2.0 ** -22
    else:
        fq.swiglu_bwd(dh.cuda(), a.cuda(), b.cuda(), dg, du)
    s, d64 = torch.sigmoid(a64), dh.double()
    want = d64 * a64 * s
    within(du, want, (off + 8 * U) * want.abs() + once(want, dtype), "du")
    want = d64 * b64 * s * (1 + a64 * (1 - s))
    # 1 + g (1 - sigma) may cancel; 1 - sigma carries sigma's error and a rounding
    parts = (d64 * b64).abs() * s * ((1 + (a64 * (1 - s)).abs()) * (off + 16 * U) + a64.abs() * (s * off + 2 * U))
    within(dg, want, parts + once(want, dtype), "dg")


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("post,gate", [(False, False), (True, True)])
@pytest.mark.parametrize("use", ["stream", "normalized"])
def test_block_norm_with_one_output_unused(monkeypatch, post, gate, use, checkpoint):
    """Nothing is passed for the gradient of an output that the loss does not have, and the result is that of zeros."""
    from paper_2510_24061_amd import block
    d = 272
    g = gen(1)
    norm = block.BlockNorm(d, post_norm=post, gate=gate, scale=SCALE, checkpoint=checkpoint, trainable=True, dtype=torch.float32)
    with torch.no_grad():
        for p in norm.parameters():
            p.copy_(1 + draw(g, d, std=0.2))
    x, b, dy = draw(g, 5, 7, d).cuda(), draw(g, 5, 7, d).cuda(), draw(g, 5, 7, d).cuda()
    given, call = [], block._b.norm_bwd
    monkeypatch.setattr(block._b, "norm_bwd", lambda dh, *a, **kw: (given.append((bool(dh.any()), kw["ds"] is not None)), call(dh, *a, **kw))[1])
    results = []
    for zeros in (False, True):
        xx, bb = x.clone().requires_grad_(), b.clone().requires_grad_()
        norm.zero_grad(set_to_none=True)
        s, h = norm(xx, bb)
        loss = (s * dy).sum() if use == "stream" else (h * dy).sum()
        if zeros:
            loss = loss + ((h if use == "stream" else s) * 0.0).sum()
        loss.backward()
        results.append([xx.grad, bb.grad] + [p.grad for p in norm.parameters()])
    assert given == [(False, True), (False, True)] if use == "stream" else given == [(True, False), (True, True)]
    assert all(torch.equal(p, q) for p, q in zip(*results))
