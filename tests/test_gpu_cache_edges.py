"""Calls of the receiver's side at their edges on MI355X: long sums, bytes that no call stores, pages that
are none, sizes and strides of one.  Plain 64-bit forms as in test_gpu_cache; tolerances are derived
beside each test.
"""
from __future__ import annotations

import itertools
import math

import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import U, UB, cache_with, dt, fill_cache, ints, model, randn, same_state, scratch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _torch

    assert _torch.cuda.is_available(), "GPU tests need a GPU"
    return _torch


@pytest.fixture(scope="module")
def cb():
    import paper_2609_32046_amd as _cb

    return _cb


# ---- attention: rounding over long sums -----------------------------------------


def rows_of(m, q, out, seqs, layer=0):
    """Every query row of a call without a causal mask: (got, want, weights, values, bound on a logit's
    error in units of 2^-24), all positions held."""
    L, n, Hq, Q, D = q.shape
    Hkv = m.pool.shape[2]
    qd, od = ref.to_f64(q), ref.to_f64(out)
    for l, i, h in itertools.product(range(L), range(n), range(Hkv)):
        k, v, there = m.read(seqs[i], layer + l, h)
        assert there.all()
        heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
        x = qd[l, i, heads].reshape(-1, D)
        z = x @ k.T / math.sqrt(D)
        w = np.exp(z - z.max(1, keepdims=True))
        p = w / w.sum(1, keepdims=True)
        err = ((D + 4) / math.sqrt(D) * (np.abs(x) @ np.abs(k).T) + 2 * np.abs(z)).max(1, keepdims=True)
        yield od[l, i, heads].reshape(-1, D), p @ v, p, v, err


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("D,P,G,m,lens", [(128, 64, 4, 1, [4000, 700]), (64, 16, 8, 2, [3000, 129]),
                                          (128, 32, 5, 3, [2500]), (64, 64, 16, 1, [1000, 4096])])
def test_few_bf16_rows_round_only_their_outputs(torch, cb, D, P, G, m, lens, cut):
    """Up to 16 rows a head: a weight loses 2^-16 of itself, so an output is off by its own rounding and
    2^-16 sum p|v|, beside what fp32 sums lose (as in check_attend: sums of 32 positions an instruction, the
    wave's steps, waves and chunks)."""
    c = cache_with(torch, cb, lens, H=2, D=D, P=P, width=8192 // P if cut else None)
    fill_cache(torch, cb, c, lens, 50 + D)
    q = randn(torch, 51, 1, len(lens), 2 * G, m, D).bfloat16().cuda()
    out = torch.empty_like(q)
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q), causal=False)
    for got, want, p, v, err in rows_of(model(c, D, P), q, out, range(len(lens))):
        size = p @ np.abs(v)
        tol = size * (2.0 ** -16 + (2 * err + len(p[0]) / 128 + 56) * U)
        tol = tol + UB * (np.abs(want) + tol)
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("D,P,G,m,lens", [(128, 64, 4, 40, [2500]), (64, 16, 8, 60, [3000, 129]), (128, 32, 5, 9, [2100])])
def test_many_bf16_rows_round_their_weights_apart(torch, cb, D, P, G, m, lens):
    """More rows: a weight loses up to 2^-8 of itself, each by itself, so the losses of a row add up as
    independent ones of mean zero: beyond x sqrt(sum (2^-8 p v)^2) with probability 2 exp(-x^2 / 2) at
    most (Hoeffding), 1e-12 at x = 7.5, over fewer than 1e5 outputs."""
    c = cache_with(torch, cb, lens, H=1, D=D, P=P)
    fill_cache(torch, cb, c, lens, 60 + D)
    q = randn(torch, 61, 1, len(lens), G, m, D).bfloat16().cuda()
    out = torch.empty_like(q)
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q), causal=False)
    for got, want, p, v, err in rows_of(model(c, D, P), q, out, range(len(lens))):
        tol = 7.5 * UB * np.sqrt((p * p) @ (v * v)) + p @ np.abs(v) * (2 * err + len(p[0]) / 128 + 56) * U
        tol = tol + UB * (np.abs(want) + tol)
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
