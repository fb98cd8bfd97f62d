"""Preference loss with infinite rewards: a label that the policy masks has a log-probability of -infinity.

By the definition a pair's loss is (1 - smoothing) log(1 + exp(-z)) + smoothing log(1 + exp(z)), whose second part is not there without smoothing."""
import math

import pytest
import torch

import paper_2510_24061_amd as fq
from block_ops_common import F32_TOL, draw, gen
from test_gpu_preference import check_loss
from test_gpu_preference import loss_of as plain_loss

pytestmark = pytest.mark.gpu
INF = float("inf")


def loss_of(logp, offsets, smoothing, beta=0.1):
    T, P = logp.shape[0], (offsets.shape[0] - 1) // 2
    loss, rewards, d = (torch.full(s, float("nan"), device="cuda") for s in ((1,), (2, P), (T,)))
    ws = torch.full((fq.logprob_workspace_bytes(T, 1, P),), 0xFF, dtype=torch.uint8, device="cuda")
    fq.preference_loss(logp.cuda(), torch.zeros(T, device="cuda"), offsets.cuda(), loss, rewards, d, ws, beta=beta, smoothing=smoothing)
    return float(loss), rewards.cpu(), d.cpu()


# one workgroup for all pairs; a workgroup a pair (more than 16384 tokens)
@pytest.mark.parametrize("T", [64, 20000])
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("masked", ["rejected", "chosen"])
def test_a_masked_label(T, masked, smoothing):
    P, n = 2, T // 4
    offsets = torch.arange(5) * n
    logp = torch.zeros(T)
    logp[5 + (2 * n if masked == "rejected" else 0)] = -INF                     # of the first pair
    loss, rewards, d = loss_of(logp, offsets, smoothing)
    first = -1 if masked == "chosen" else 1
    want = {(1, 0.0): 0.5 * math.log(2.0)}.get((first, smoothing), INF)         # the second pair's z is 0
    assert loss == INF if want == INF else abs(loss - want) <= F32_TOL
    assert float(rewards[0 if first < 0 else 1, 0]) == -INF and not rewards[:, 1].any()
    # the loss by a chosen log-probability: beta / P (smoothing sigma(z) - (1 - smoothing) sigma(-z))
    slope = 0.1 / P * (smoothing if first > 0 else -(1.0 - smoothing))
    half = 0.1 / P * (smoothing - 0.5)
    want_d = torch.cat([torch.full((n,), slope), torch.full((n,), half), torch.full((n,), -slope), torch.full((n,), -half)])
    assert float((d - want_d).abs().max()) <= F32_TOL * 0.1


def launched(f):
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as p:
        f()
        torch.cuda.synchronize()
    return " ".join(e.name for e in p.events())


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("T,P", [(16384, 3), (16385, 3), (16385, 1), (50000, 4), (70000, 300), (4000, 32), (4000, 33), (4000, 1025), (20000, 1500), (1, 2000), (300000, 65536)])
def test_a_workgroup_a_pair(T, P, smoothing):
    """Beyond 16384 tokens or 32 pairs: a workgroup a pair and one for the mean.  Many pairs have empty sequences among them."""
    g = gen(T + P)
    offsets = torch.sort(torch.randint(T // 9, T - T // 7 + 1, (2 * P + 1,), generator=g))[0]     # tokens before and behind the sequences
    logp, ref = -3 + draw(g, T), -3 + draw(g, T)
    loss_of(logp, offsets, smoothing)
    names = launched(lambda: loss_of(logp, offsets, smoothing))
    pairs = T > 16384 or P > 32
    assert ("preference_pair_kernel" in names) == ("preference_mean_kernel" in names) == pairs and ("preference_one_kernel" in names) != pairs
    check_loss(logp, ref, offsets, 0.1, smoothing)


def test_a_workgroup_a_pair_with_bounds_outside():
    T = 17000
    g = gen(3)
    logp, ref = -3 + draw(g, T), -3 + draw(g, T)
    for outside, inside in (([-5, 6000, 90000], [0, 6000, T]), ([-9, -1, 8000, 8000, 1 << 40], [0, 0, 8000, 8000, T])):
        a, b = plain_loss(logp, ref, torch.tensor(outside), 0.1, 0.1), plain_loss(logp, ref, torch.tensor(inside), 0.1, 0.1)
        assert all(torch.equal(a[k], b[k]) for k in a)
        check_loss(logp, ref, torch.tensor(inside), 0.1, 0.1)


def test_the_two_forms_agree_across_their_line():
    """The same sequences with one token of none behind them: 16384 tokens in one workgroup, 16385 in a workgroup a pair."""
    g = gen(4)
    logp, ref = -3 + draw(g, 16385), -3 + draw(g, 16385)
    offsets = torch.tensor([0, 5000, 8000, 8001, 16384])
    one, many = plain_loss(logp[:16384], ref[:16384], offsets, 0.1, 0.1), plain_loss(logp, ref, offsets, 0.1, 0.1)
    # sums in 64 bits in another order, rounded once
    assert float((one["rewards"] - many["rewards"]).abs().max()) <= 2.0 ** -23 * float(one["rewards"].abs().max())
    assert float((one["d_logp"] - many["d_logp"][:16384]).abs().max()) <= F32_TOL * 0.1 * float(one["rewards"].abs().max()) and float(many["d_logp"][16384]) == 0.0
