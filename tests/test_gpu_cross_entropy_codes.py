"""Random problems whose FP8 operands all are numbers, and problems in which one code is NaN."""
import math
import random

import pytest
import torch

from paper_2209_05433_b200 import api
from tests import test_gpu_cross_entropy as loss
from tests.test_gpu_fused import _guards_kept, _matrix

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4, E5, BF, F32 = api.E4M3, api.E5M2, torch.bfloat16, torch.float32
MOST = {E4: 448.0, E5: 57344.0}
_plain_operand = loss._operand


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("seed", range(40))
def test_random_problems_of_numbers(seed, monkeypatch):
    """with small scales the weights' codes reach the format's end: values beyond it are held there, and every problem is checked whole"""
    monkeypatch.setattr(loss, "_operand", lambda v, fmt: _plain_operand(v if fmt is None else v.clamp(-MOST[fmt], MOST[fmt]), fmt))
    rng = random.Random(5000 + seed)
    while True:
        T, K, V = _log(rng, 1, 4000), _log(rng, 1, 5000), _log(rng, 1, 30000)
        if T * V <= 6_000_000 and K * V <= 30_000_000:
            break
    fx, fw = rng.choice([(E4, E4), (E4, E4), (E4, E5), (E5, E4)])
    p = loss.Problem(T, K, V, fx, fw, seed=seed, ignored=rng.choice([0.0, 0.1, 0.9]), weighted=rng.random() < 0.5,
                     sx=2.0 ** rng.uniform(-10, 2), sw=2.0 ** rng.uniform(-10, 2))
    assert bool(torch.isfinite(p.w64).all()) and bool(torch.isfinite(p.x64).all())
    (dx, all_dx), (dw, all_dw) = _matrix(T, K, rng.choice([BF, F32])), _matrix(V, K, rng.choice([BF, F32]))
    p.forward()
    p.backward(dx, dw)
    loss._ok()
    p.check_forward()
    p.check_backward(dx, dw)
    assert _guards_kept(dx, all_dx) and _guards_kept(dw, all_dw)


def _run(p):
    dx, dw = torch.empty(p.T, p.K, device=DEV), torch.empty(p.V, p.K, device=DEV)
    p.forward()
    p.backward(dx, dw)
    loss._ok()
    return dx, dw


SHAPES = [(5, 64, 300), (200, 96, 1000)]


@pytest.mark.parametrize("T,K,V", SHAPES)
def test_a_nan_in_a_token_that_counts(T, K, V):
    """its row of everything, and the sums over tokens"""
    p = loss.Problem(T, K, V, E4, E4, ignored=0.0)
    clean, _ = _run(p)
    want = p.loss.clone(), p.lse.clone()
    p.x[2, 7] = 0x7F
    dx, dw = _run(p)
    others = torch.arange(T, device=DEV) != 2
    assert bool(torch.isnan(p.loss[2])) and bool(torch.isnan(p.lse[2])) and bool(torch.isnan(dx[2]).all()) and bool(torch.isnan(dw).all())
    assert torch.equal(p.loss[others], want[0][others]) and torch.equal(p.lse[others], want[1][others]) and torch.equal(dx[others], clean[others])


@pytest.mark.parametrize("T,K,V", SHAPES)
def test_a_nan_in_a_token_that_does_not_count(T, K, V):
    """its lse, and its column of dw, where a gradient of zero meets it"""
    p = loss.Problem(T, K, V, E4, E4, ignored=0.0)
    p.target[2] = -100
    p.dloss[2] = float("nan")
    clean, clean_w = _run(p)
    p.x[2, 7] = 0x7F
    dx, dw = _run(p)
    assert float(p.loss[2]) == 0.0 and bool(torch.isnan(p.lse[2]))
    assert torch.equal(dx, clean) and not dx[2].any()
    columns = torch.arange(K, device=DEV) != 7
    assert bool(torch.isnan(dw[:, 7]).all()) and torch.equal(dw[:, columns], clean_w[:, columns])


@pytest.mark.parametrize("T,K,V", SHAPES)
def test_a_nan_in_a_weight(T, K, V):
    """every token has that logit: all losses that count, their rows of dx and all sums over them; zero gradients meet it in its column"""
    p = loss.Problem(T, K, V, E4, E4, ignored=0.0)
    p.target[1::2] = V
    p.w[11, 3] = 0xFF
    dx, dw = _run(p)
    counts = torch.arange(T, device=DEV) % 2 == 0
    assert bool(torch.isnan(p.lse).all()) and bool(torch.isnan(p.loss[counts]).all()) and not p.loss[~counts].any()
    columns = torch.arange(K, device=DEV) != 3
    assert bool(torch.isnan(dx[counts]).all()) and bool(torch.isnan(dx[~counts][:, 3]).all()) and not dx[~counts][:, columns].any()
    assert bool(torch.isnan(dw).all())
    p.target.fill_(-1)                                            # nothing counts: dw is zero
    dx, dw = _run(p)
    assert not dw.any() and not p.loss.any()


@pytest.mark.parametrize("fmt", [E4, None], ids=["fp8", "bf16"])
@pytest.mark.parametrize("T,K,V", SHAPES)
def test_an_infinite_factor_leaves_nothing_finite_of_its_token(T, K, V, fmt):
    """a saturating conversion must not make numbers of it"""
    p = loss.Problem(T, K, V, fmt, fmt, ignored=0.0)
    for factor in (float("inf"), -float("inf"), float("nan")):
        p.dloss[2] = factor
        dx, dw = _run(p)
        others = torch.arange(T, device=DEV) != 2
        assert not torch.isfinite(dx[2]).any() and not torch.isfinite(dw).any() and bool(torch.isfinite(dx[others]).all())
    p.target[2] = -5                                              # it does not count: nothing of it is looked at
    dx, dw = _run(p)
    assert not dx[2].any() and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
