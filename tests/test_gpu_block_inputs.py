"""What the modules around the melded layers take besides dense aligned tensors, through the kernels (the plumbing itself: test_block_modules)."""
import pytest
import torch

from block_ops_common import F32_TOL, draw, gen, rel

pytestmark = pytest.mark.gpu


def off_boundary(t):
    """The same values, dense, one element behind a 16-byte boundary."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    view = flat[1:].view(t.shape)
    view.copy_(t)
    assert view.is_contiguous() and view.data_ptr() % 16
    return view


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tensors_off_the_16_byte_boundaries(dtype):
    from paper_2510_24061_amd.block import BlockNorm, Mx4Linear, swiglu
    g = gen(1)
    a, b = (draw(g, 5, 64).to(dtype).cuda() for _ in range(2))
    norm, layer = BlockNorm(64, dtype=dtype), Mx4Linear(draw(g, 32, 64).cuda(), input_grad=True)
    for f in (lambda x, y: swiglu(x, y), lambda x, y: norm(x, y)[1], lambda x, y: layer(x), lambda x, y: layer(y)):
        results = []
        for x, y in ((a, b), (off_boundary(a), off_boundary(b))):
            x, y = x.detach().requires_grad_(), y.detach().requires_grad_()
            out = f(x, y)
            out.backward(off_boundary(torch.ones_like(out)))
            results.append([out.detach(), x.grad, y.grad])
        assert all(p is q is None or torch.equal(p, q) for p, q in zip(*results))


def test_one_row_of_logits_for_many_labels():
    from paper_2510_24061_amd.block import token_logprobs
    row = draw(gen(2), 1, 1001, std=2.0).cuda().requires_grad_()
    labels = torch.arange(7, device="cuda") * 100
    logp = token_logprobs(row.expand(7, 1001), labels)
    logp.sum().backward()
    r64 = row.detach().double().requires_grad_()
    want = torch.log_softmax(r64, 1)[0, labels]
    want.sum().backward()
    assert rel(logp, want) <= F32_TOL and rel(row.grad, r64.grad) <= 2 * F32_TOL


def test_gradients_cannot_be_differentiated():
    from paper_2510_24061_amd.block import BlockNorm, Mx4Linear, preference_loss, swiglu, token_logprobs
    g = gen(3)
    x, y = (draw(g, 4, 64).cuda().requires_grad_() for _ in range(2))
    norm, layer = BlockNorm(64, dtype=torch.float32), Mx4Linear(draw(g, 32, 64).cuda(), input_grad=True)
    labels, offsets = torch.tensor([1, 2, 3, 4]).cuda(), torch.tensor([0, 2, 4]).cuda()
    for f in (lambda: swiglu(x, y).sum(), lambda: norm(x, y)[1].sum(), lambda: layer(x).sum(), lambda: token_logprobs(x, labels).sum(),
              lambda: preference_loss(token_logprobs(x, labels), torch.zeros(4, device="cuda"), offsets)[0]):
        first, = torch.autograd.grad(f(), x)
        again, = torch.autograd.grad(f(), x, create_graph=True)
        assert torch.equal(first, again)
        with pytest.raises(RuntimeError, match="differentiated"):
            torch.autograd.grad(again.square().sum() + x.sum(), x)


def test_evaluation_writes_no_checkpoints():
    """The same results, and of the memory only the outputs."""
    from paper_2510_24061_amd.block import BlockNorm, swiglu
    x, y = (draw(gen(k), 256, 4096).bfloat16().cuda() for k in (4, 5))
    norm = BlockNorm(4096, post_norm=True)
    with torch.enable_grad():
        want = [t.detach() for t in (*norm(x.clone().requires_grad_(), y), swiglu(x.clone().requires_grad_(), y))]
    torch.cuda.synchronize()
    with torch.no_grad():
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = [*norm(x, y), swiglu(x, y)]
        used = torch.cuda.max_memory_allocated() - before
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and used <= 3 * x.numel() * 2 + 65536


def test_preference_step_over_filled_rows():
    """Token ids behind a row's length are not looked up: -100 and ids beyond the vocabulary give what 0 gives."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import preference_step as example
    from paper_2510_24061_amd.block import preference_step
    policy, reference, _ = example.build(blocks=1)
    tokens, prompts, lengths = example.pairs(P=2, S=40)
    inside = torch.arange(40, device="cuda") < lengths[:, None]
    results = []
    for filler in (0, -100, 10 ** 9):
        with torch.no_grad():
            loss, rewards = preference_step(policy, reference, torch.where(inside, tokens, torch.full_like(tokens, filler)), prompts, lengths)
        results.append((loss, rewards))
    assert all(torch.equal(a, b) for r in results[1:] for a, b in zip(r, results[0])) and results[0][0].isfinite()
