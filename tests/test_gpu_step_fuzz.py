"""Seeded random shapes, types, pitches and targets through the loss, its gradients and the AdamW step, against the same
definitions and tolerances as their own tests."""
import math
import random

import pytest
import torch

from paper_2209_05433_b200 import api
from tests import test_gpu_adamw as adamw
from tests import test_gpu_cross_entropy as loss
from tests.test_gpu_fused import _gen, _guards_kept, _matrix, _scalar

pytestmark = pytest.mark.gpu
E4, E5, BF, F32 = api.E4M3, api.E5M2, torch.bfloat16, torch.float32


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("seed", range(48))
def test_loss_and_gradients(seed):
    rng = random.Random(1000 + seed)
    while True:
        T, K, V = _log(rng, 1, 4000), _log(rng, 1, 5000), _log(rng, 1, 30000)
        if T * V <= 6_000_000 and K * V <= 30_000_000:
            break
    fx, fw = rng.choice([(E4, E4), (E4, E4), (E4, E5), (E5, E4), (None, None), (None, None)])
    p = loss.Problem(T, K, V, fx, fw, seed=seed, ignored=rng.choice([0.0, 0.1, 0.9]), weighted=rng.random() < 0.5,
                     sx=2.0 ** rng.uniform(-8, 2), sw=2.0 ** rng.uniform(-8, 2))
    (dx, all_dx), (dw, all_dw) = _matrix(T, K, rng.choice([BF, F32])), _matrix(V, K, rng.choice([BF, F32]))
    p.forward()
    p.backward(dx, dw)
    loss._ok()
    p.exact()
    counts = torch.zeros(T, dtype=torch.bool, device="cuda")
    counts[p.rows] = True
    if bool(torch.isnan(p.w64).any()):                            # weights beyond E4M3 became NaN codes: so does every logit's row
        assert bool(torch.isnan(p.lse64).all()) and bool(torch.isnan(p.lse).all())
        assert bool(torch.isnan(p.loss[counts]).all()) and not p.loss[~counts].any()
        clean = ~torch.isnan(p.w64).any(0)                        # elsewhere dx has the NaN of 0 * NaN
        assert bool(torch.isnan(dx[counts]).all()) and not dx[~counts][:, clean].any()
        assert _guards_kept(dx, all_dx) and _guards_kept(dw, all_dw)
        return
    p.check_forward()
    p.check_backward(dx, dw)
    assert _guards_kept(dx, all_dx) and _guards_kept(dw, all_dw)
    only, _ = _matrix(T, K, dx.dtype)
    p.backward(only, None)
    assert torch.equal(only, dx)


@pytest.mark.parametrize("seed", range(24))
def test_adamw(seed):
    rng = random.Random(2000 + seed)
    g = _gen(seed)
    copy = rng.choice([None, "bf16", E4, E5])
    ts = [adamw.Tensors(_log(rng, 1, 200000), rng.choice([F32, BF]), rng.choice([F32, BF]), rng.random() < 0.5, copy if rng.random() < 0.7 else None, g,
                        shift=rng.choice([0, 0, 1, 2, 4, 8]), decay=rng.choice([0.0, 0.1])) for _ in range(rng.randint(1, 12))]
    lr, step, b1, b2, eps = 10.0 ** rng.uniform(-5, -1), _log(rng, 1, 100000), rng.choice([0.0, 0.9, 0.95]), rng.choice([0.9, 0.99, 0.999]), 10.0 ** rng.uniform(-12, -6)
    norm, most, seed64 = 10.0 ** rng.uniform(-2, 2), 10.0 ** rng.uniform(-2, 2), rng.getrandbits(64)
    norm = float(_scalar(norm))
    api.fp8_adamw_step(adamw._plan(ts), lr, step, beta1=b1, beta2=b2, eps=eps, seed=seed64, norm=_scalar(norm), max_norm=most)
    adamw._ok()
    number = 0
    for t in ts:
        adamw._check_tensor(t, number, lr, step, b1, b2, eps, min(1.0, most / norm), seed64)
        number += -(-t.n // 256) * 256
