"""Preference loss with infinite rewards: a label that the policy masks has a log-probability of -infinity.

By the definition a pair's loss is (1 - smoothing) log(1 + exp(-z)) + smoothing log(1 + exp(z)), whose second part is not there without smoothing."""
import math

import pytest
import torch

import paper_2510_24061_amd as fq
from block_ops_common import F32_TOL

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
