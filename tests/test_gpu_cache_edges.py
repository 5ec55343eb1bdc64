"""Calls of the receiver's side at their edges on MI355X: long sums, bytes that no call stores, pages that
are none, sizes and strides of one.  Plain 64-bit forms as in test_gpu_cache; tolerances are derived
beside each test.
"""
from __future__ import annotations

import itertools
import math
import os
import re

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


# ---- attention: what masked places hold ------------------------------------------


@pytest.mark.parametrize("rest,cut", [(0, False), (1198, False), (18, True)])
@pytest.mark.parametrize("dtype,D,P,G", [("bf16", 128, 32, 1), ("f32", 128, 16, 1), ("bf16", 64, 16, 3), ("f32", 64, 32, 3),
                                         ("bf16", 128, 64, 20), ("bf16", 64, 64, 30)])
def test_attend_rows_that_do_not_see_a_position_do_not_feel_it(torch, cb, dtype, D, P, G, rest, cut):
    """Room for eight positions, four of them not yet written, under a causal mask: the first four query tokens
    have the same bits whatever bytes the pages hold there."""
    lens, m = [75, 40], 8
    c = cache_with(torch, cb, lens, H=2, D=D, P=P, seed=70, width=8192 // P if cut else None)
    fill_cache(torch, cb, c, lens, 71)
    # rest: entries of no query token; beside many of them a workgroup is one wave
    seqs, q_lens = ints(torch, [0, 1] + [0] * rest), ints(torch, [m, m] + [0] * rest)
    q = randn(torch, 72, 1, 2 + rest, 2 * G, m, D).to(dt(torch, dtype)).cuda()
    ws = scratch(torch, cb, c, q)
    table, n, s = c.table.cpu().numpy(), P * D // 2, P * D // 32
    want = None
    for k, byte in [(127, 127), (127, 252), (127, 253), (127, 254), (127, 255), (253, 127), (254, 254), (255, 253)]:
        for i, length in enumerate(lens):
            for pos in range(length - 4, length):
                u, at = c.pool[int(table[i, pos // P]), 0], pos % P
                u[:, at * (D // 2):(at + 1) * (D // 2)] = 0x7F           # 6 and -6
                u[:, 2 * n + at * (D // 32):2 * n + (at + 1) * (D // 32)] = k
                u[:, n:2 * n].view(2, P // 4, 16, 4, D // 32)[:, at // 4, :, at % 4] = 0xF7
                u[:, 2 * n + s:].view(2, P // 4, D // 32, 4)[:, at // 4, :, at % 4] = byte
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:4], 7.0, device="cuda")
        cb.cb_cache_attend(c.desc, q, out, ws, lse, seqs, q_lens)
        got = out[:, :2, :, :4].clone(), lse[:, :2, :, :4].clone()
        if want is None:
            want = got
            assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (k, byte)


# ---- pages -----------------------------------------------------------------------


@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("n", [1, 3, 64, 65, 200, 1100])
@pytest.mark.parametrize("entry", [-1, -7, 10**6, 2**31 - 1])
def test_fork_of_a_parent_without_one_of_its_pages_changes_nothing(torch, cb, entry, n, copy):
    """A hole, or a number that is no page, anywhere in any parent's row: refused, and the children keep what
    they held; put right, the same call is done."""
    P, D = 16, 64
    lens = [7 * P + 5, 2 * P, 9] + [P + 3] * n
    c = cache_with(torch, cb, lens, L=1, H=1, D=D, P=P, extra=9 * n, width=9, seed=n)
    parents, children = ints(torch, [i % 3 for i in range(n)]), ints(torch, list(range(3, 3 + n)))
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, n), dtype=torch.uint8, device="cuda")
    for s, j in [(0, 0), (0, 7), (1, 1), (2, 0)]:
        if s >= n:   # no parent of this call
            continue
        before = c.table[s, j].item()
        c.table[s, j] = entry
        m = model(c, D, P)
        c.status.fill_(5)
        cb.cb_cache_fork(c.desc, parents, children, c.status, ws, copy)
        assert c.status.item() == -1 and cb.cb_cache_status(c.status) == -2
        same_state(c, m)
        c.table[s, j] = before
    m = model(c, D, P)
    cb.cb_cache_fork(c.desc, parents, children, c.status, ws, copy)
    assert c.status.item() == m.fork([i % 3 for i in range(n)], list(range(3, 3 + n)), copy) == 0
    same_state(c, m)


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64)])
def test_compact_of_positions_without_a_page(torch, cb, D, P):
    """Kept positions in a hole of the table, or behind an entry that is no page, are rows of zeros."""
    lens = [4 * P + 3, 10]
    c = cache_with(torch, cb, lens, L=1, H=2, D=D, P=P, extra=12, width=6)
    fill_cache(torch, cb, c, lens, 80)
    c.table[0, 1], c.table[0, 3] = -1, c.pool.shape[0]
    keep = 4 * P + 3
    idx = torch.arange(keep, dtype=torch.int32, device="cuda").reshape(1, 1, 1, keep)
    ws = torch.empty(cb.cb_cache_compact_workspace_bytes(c.desc, 1), dtype=torch.uint8, device="cuda")
    m = model(c, D, P)
    cb.cb_cache_compact(c.desc, ints(torch, [0]), ints(torch, [1]), idx, c.status, ws)
    assert cb.cb_cache_status(c.status) == 0
    got = model(c, D, P)
    for h in range(2):
        k, v, there = m.read(0, 0, h)
        kk, vv, _ = got.read(1, 0, h)
        assert np.array_equal(there, [t // P not in (1, 3) for t in range(keep)])
        assert np.array_equal(kk, k * there[:, None]) and np.array_equal(vv, v * there[:, None])


# ---- sizes and strides of one ------------------------------------------------------


@pytest.mark.parametrize("n,H", [(3, 2), (1, 4), (2, 1)])
def test_rows_of_unlike_strides_along_axes_of_one(torch, cb, n, H):
    """A decoding step's keys head-major and its values token-major: one token, so every row lies where the
    other's strides say; with two tokens, or heads apart, it does not, and the call is refused."""
    D, P = 128, 16
    c = cache_with(torch, cb, [20] * n, H=H, D=D, P=P)
    k = randn(torch, 90, 1, n, H, 1, D).bfloat16().cuda()
    v = randn(torch, 91, n, 1, H, D).bfloat16().cuda().transpose(1, 2)[None]
    v = v.as_strided(v.shape, (7, *v.stride()[1:3], 5 * D, 1))
    assert v.shape == k.shape and v.stride() != k.stride()
    cb.cb_cache_write(c.desc, k, v)
    ko = torch.zeros_like(k)
    vo = torch.zeros((n, 1, H, D), dtype=torch.bfloat16, device="cuda").transpose(1, 2)[None]
    vo = vo.as_strided(v.shape, v.stride())
    cb.cb_cache_read(c.desc, ko, vo, start=ints(torch, [19] * n))
    assert np.array_equal(ref.to_f64(ko), ref.values(*ref.quantise(ref.to_f64(k))))
    assert np.array_equal(ref.to_f64(vo), ref.values(*ref.quantise(ref.to_f64(v))))
    k2, v2 = torch.zeros((1, n, 2, 2, D), device="cuda"), torch.zeros((1, n, 2, 2, D), device="cuda").transpose(2, 3)
    c2 = cache_with(torch, cb, [20] * n, H=2, D=D, P=P)
    for fn in (cb.cb_cache_write, cb.cb_cache_read):
        with pytest.raises(cb.CBError, match="unlike strides"):
            fn(c2.desc, k2, v2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_in_pages_of_128(torch, cb, dtype, D):
    """Codes and scales byte for byte over the borders of pages of 128 positions, everything else as it was."""
    P, lens, start, T = 128, [300, 128, 5], [100, 0, 1], 150
    c = cache_with(torch, cb, lens, L=2, H=2, D=D, P=P, seed=D)
    m = model(c, D, P)
    counts = [T, 128, 4]
    k, v = (randn(torch, 95 + i, 1, 3, 2, T, D).to(dt(torch, dtype)).cuda() for i in range(2))
    cb.cb_cache_write(c.desc, k, v, start=ints(torch, start), counts=ints(torch, counts), layer=1)
    for x, which in ((k, 0), (v, 1)):
        code, scale = ref.quantise(ref.to_f64(x))
        for i, h in itertools.product(range(3), range(2)):
            for page in range(start[i] // P, (start[i] + counts[i] - 1) // P + 1):
                u = list(ref.unpack(m.pool[m.table[i, page], 1, h], P, D))
                a, b = max(start[i], page * P), min(start[i] + counts[i], (page + 1) * P)
                u[2 * which][a - page * P:b - page * P] = code[0, i, h, a - start[i]:b - start[i]]
                u[2 * which + 1][a - page * P:b - page * P] = scale[0, i, h, a - start[i]:b - start[i]]
                m.pool[m.table[i, page], 1, h] = ref.pack(*u)
    same_state(c, m)
    ko, vo = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    cb.cb_cache_read(c.desc, ko, vo, start=ints(torch, start), counts=ints(torch, counts), layer=1)
    for x, o in ((k, ko), (v, vo)):
        want = ref.values(*ref.quantise(ref.to_f64(x)))
        for i in range(3):
            assert np.array_equal(ref.to_f64(o[0, i, :, :counts[i]]), want[0, i, :, :counts[i]])
            assert (o[0, i, :, counts[i]:] == 3.0).all()


# ---- attention: large logits ---------------------------------------------------------


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P,G,m", [(128, 32, 4, 1), (64, 16, 5, 7), (64, 64, 8, 40)])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 24, 2.0 ** 28])
def test_attend_logits_of_any_size(torch, cb, size, D, P, G, m, dtype, cut):
    """Logits of 6000, of millions and of 2^24 * 12, exact by construction (one value of a key times a power of
    two), so that one position has all the weight: its values come out, rounded like any product with 1 / sum
    (2 U, the reciprocal and the product; three parts of a weight 2 U more) and to bf16, and the log-sum is its logit.
    2^28 * 12 is past the 2^28 that a call answers for: in units of log2 its reference has steps of 512, and half a
    step in an exponent is past 2^128.  Only rows that see no such logit are looked at."""
    lens = [333, 200, 40]
    c = cache_with(torch, cb, lens, H=1, D=D, P=P, width=8192 // P if cut else None)
    rng = np.random.default_rng(D + m)
    T = max(lens)
    k = np.zeros((1, 3, 1, T, D), np.float32)
    k[0, :2, 0, :, 5] = rng.choice([0.5, -1, 2, 3, -3, 4, -4], (2, T))
    k[0, 2, 0, :, 5] = rng.choice([-4, -6], T)                     # all logits below zero where size is above
    at = {0: (321, 17), 1: (3, 180), 2: (30, 11)}                  # of the largest and the smallest
    k[0, 0, 0, 321, 5], k[0, 0, 0, 17, 5] = 6, -6
    k[0, 1, 0, 3, 5], k[0, 1, 0, 180, 5] = 6, -6
    k[0, 2, 0, 30, 5], k[0, 2, 0, 11, 5] = -3, -12
    v = randn(torch, 96, 1, 3, 1, T, D)
    cb.cb_cache_write(c.desc, torch.from_numpy(k).cuda(), v.cuda(), start=ints(torch, [0] * 3), counts=ints(torch, lens))
    q = randn(torch, 97, 1, 3, G, m, D)                            # against zeros: no matter
    sign = torch.from_numpy(rng.choice([-1.0, 1.0], (1, 3, G, m))).float()
    q[..., 5] = size * sign
    q = q.to(dt(torch, dtype)).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device="cuda")
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q), lse, causal=False, scale=1.0)
    mm = model(c, D, P)
    for i in range(3):
        kk, vv, _ = mm.read(i, 0, 0)
        for g, r in itertools.product(range(G), range(m)):
            w = at[i][0 if sign[0, i, g, r] > 0 else 1]
            top = size * sign[0, i, g, r].item() * kk[w, 5]
            if abs(size * kk[:, 5]).max() > 2.0 ** 28:
                continue
            assert top == max(size * sign[0, i, g, r].item() * kk[:, 5]) and (kk[:, 5] == kk[w, 5]).sum() == 1
            want = vv[w]
            tol = np.abs(want) * (4 * U + (UB * 1.01 if dtype == "bf16" else 0))
            assert (np.abs(ref.to_f64(out[0, i, g, r]) - want) <= tol).all()
            # the logit in units of log2: c2, its product, the sum's logarithm, the way back: U each
            assert abs(lse[0, i, g, r].item() - top) <= 6 * U * abs(top)


# ---- pools past 2^32 bytes -------------------------------------------------------------


def test_forks_thinning_and_attention_in_a_large_pool(torch, cb):
    """Pages that lie beyond 4 GB are shared, copied, thinned and attended to as the same pages of a small pool."""
    L, H, D, P = 32, 8, 128, 256
    c = cb.Cache(L, H, D, P, 500, 4, 3)                            # 4.5 GB
    few = cb.Cache(L, H, D, P, 2, 4, 3)
    few.pool.random_(0, 256)
    few.pool[..., P * D:] = (few.pool[..., P * D:] & 3) + 124
    c.pool[485:499] = 1
    c.pool[[498, 485]] = few.pool
    few.table[:, :2] = ints(torch, [0, 1])
    few.lens.fill_(400)
    c.refs.fill_(1)
    c.refs[486:496] = 0
    c.table[0, :2] = ints(torch, [498, 485])
    c.lens[0] = 400
    page = c.pool[0].numel()
    assert 485 * page > 2 ** 32
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, 1), dtype=torch.uint8, device="cuda")
    zero = ints(torch, [0])
    words = [torch.full_like(c.status, 5) for _ in range(3)]
    cb.cb_cache_fork(c.desc, zero, ints(torch, [1]), words[0], ws, True)
    cb.cb_cache_fork(c.desc, zero, ints(torch, [2]), words[1], ws)
    idx = torch.sort(torch.rand((1, L, H, 400), device="cuda").topk(300, dim=-1)[1], dim=-1)[0].to(torch.int32)
    cw = torch.empty(cb.cb_cache_compact_workspace_bytes(c.desc, 1), dtype=torch.uint8, device="cuda")
    cb.cb_cache_compact(c.desc, zero, ints(torch, [3]), idx, words[2], cw)
    assert [w.item() for w in words] == [0, 0, 0]
    assert c.table.tolist() == [[498, 485, -1], [486, 487, -1], [498, 488, -1], [489, 490, -1]]
    assert torch.equal(c.pool[[486, 487]], few.pool) and torch.equal(c.pool[[498, 488]], few.pool)
    got = [torch.empty((L, 1, H, 300, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    all_ = [torch.empty((L, 1, H, 400, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cb.cb_cache_read(c.desc, *got, ints(torch, [3]))
    cb.cb_cache_read(few.desc, *all_, zero)
    for x, y in zip(got, all_):
        assert torch.equal(x[:, 0], y[:, 0].gather(2, idx[0].long().unsqueeze(-1).expand(L, H, 300, D)))
    for m in (1, 30):
        q = randn(torch, 98, L, 3, 2 * H, m, D).bfloat16().cuda()
        outs = []
        for x in (c, few):
            out = torch.empty_like(q)
            cb.cb_cache_attend(x.desc, q, out, scratch(torch, cb, x, q), seqs=ints(torch, [0, 1, 2]))
            outs.append(out)
        assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


# ---- the smallest and the largest calls ------------------------------------------------


def test_counts_beyond_the_rows_that_are_given(torch, cb):
    """More rows named than there are: all of them, the sequence's last; fewer than none: none."""
    D, P = 64, 16
    c = cache_with(torch, cb, [40, 33, 20], D=D, P=P)
    m = model(c, D, P)
    k = randn(torch, 100, 1, 3, 2, 5, D).cuda()
    counts = ints(torch, [5, 2**31 - 1, -2**31])
    cb.cb_cache_write(c.desc, k, k, counts=counts)
    after = model(c, D, P)
    want = ref.values(*ref.quantise(ref.to_f64(k)))
    for s, n in ((0, 40), (1, 33), (2, 20)):
        for h in range(2):
            kk, vv, _ = after.read(s, 0, h)
            ko, vo, _ = m.read(s, 0, h)
            if s < 2:
                ko[n - 5:], vo[n - 5:] = want[0, s, h], want[0, s, h]
            assert np.array_equal(kk, ko, equal_nan=True) and np.array_equal(vv, vo, equal_nan=True)
    ko, vo = torch.full_like(k, 3.0), torch.full_like(k, 3.0)
    cb.cb_cache_read(c.desc, ko, vo, counts=counts)
    assert np.array_equal(ref.to_f64(ko[:, :2]), want[:, :2]) and (ko[:, 2] == 3.0).all() and torch.equal(ko, vo)


@pytest.mark.parametrize("D", [64, 128])
def test_a_cache_of_one_page(torch, cb, D):
    """One page, one sequence, one layer and head: filled, read, attended to, refused more, given back."""
    c = cb.Cache(1, 1, D, 16, 1, 1, 1)
    zero, one = ints(torch, [0]), ints(torch, [1])
    ws = torch.empty(max(cb.cb_cache_fork_workspace_bytes(c.desc, 1), cb.cb_cache_compact_workspace_bytes(c.desc, 1)),
                     dtype=torch.uint8, device="cuda")
    for t in range(16):
        cb.cb_cache_extend(c.desc, zero, one, c.status)
        assert c.status.item() == 0 and c.lens.tolist() == [t + 1] and c.refs.tolist() == [1]
        k, v = randn(torch, 101 + t, 1, 1, 1, 1, D).cuda(), randn(torch, 131 + t, 1, 1, 1, 1, D).cuda()
        cb.cb_cache_write(c.desc, k, v)
        q = randn(torch, 161 + t, 1, 1, 1, 1, D).cuda()
        out = torch.empty_like(q)
        cb.cb_cache_attend(c.desc, q, out)
        for got, want, p, vv, err in rows_of(model(c, D, 16), q, out, [0]):
            assert (np.abs(got - want) <= p @ np.abs(vv) * (2 * err + 56) * U).all()
    cb.cb_cache_extend(c.desc, zero, one, c.status)
    assert cb.cb_cache_status(c.status) == -2          # longer than the table
    idx = torch.zeros((1, 1, 1, 1), dtype=torch.int32, device="cuda")
    cb.cb_cache_compact(c.desc, zero, zero, idx, c.status, ws)
    assert c.status.item() == 1 and c.lens.tolist() == [16] and c.refs.tolist() == [1]
    cb.cb_cache_fork(c.desc, zero, zero, c.status, ws)
    assert c.status.item() == -1
    cb.cb_cache_free(c.desc, zero)
    assert c.lens.tolist() == [0] and c.refs.tolist() == [0] and c.table.tolist() == [[-1]]


def test_a_cache_of_the_most_sequences(torch, cb):
    """2^17 sequences and calls of 2048 entries: the last of each."""
    n, seqs, P, D = 2048, 1 << 17, 16, 64
    c = cb.Cache(1, 1, D, P, 3 * n, seqs, 2)
    m = ref.Model(np.zeros((3 * n, 0)), c.refs.cpu().numpy(), c.table.cpu().numpy(), c.lens.cpu().numpy(), D, P)
    a, b = list(range(seqs - n, seqs)), list(range(n))
    add = [1 + i % 17 for i in range(n)]
    cb.cb_cache_extend(c.desc, ints(torch, a), ints(torch, add), c.status)
    assert c.status.item() == m.extend(a, add) == 0
    same_state(c, m, pool=False)
    for bad in (a[:-1] + [a[0]], a[:-1] + [seqs]):
        cb.cb_cache_extend(c.desc, ints(torch, bad), ints(torch, add), c.status)
        assert c.status.item() == -1
    same_state(c, m, pool=False)
    m.pool = c.pool.cpu().numpy()
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, n), dtype=torch.uint8, device="cuda")
    cb.cb_cache_fork(c.desc, ints(torch, a), ints(torch, b), c.status, ws)
    assert c.status.item() == m.fork(a, b, False) == 0
    same_state(c, m)
    cb.cb_cache_free(c.desc, ints(torch, a + b + a))
    assert not c.refs.any() and not c.lens.any() and int(c.table.max()) == -1


def test_a_pool_of_the_most_pages(torch, cb):
    """2^24 pages of which only the last few are free: found, taken and given back."""
    pages = 1 << 24
    c = cb.Cache(1, 1, 64, 16, pages, 3, 8)
    c.refs.fill_(1)
    c.refs[pages - 7:] = 0
    c.refs[pages - 3] = 1
    cb.cb_cache_extend(c.desc, ints(torch, [2, 0]), ints(torch, [40, 33]), c.status)
    assert c.status.item() == 0
    free = [pages - 7, pages - 6, pages - 5, pages - 4, pages - 2, pages - 1]
    assert c.table[[2, 0], :4].tolist() == [[*free[:3], -1], [*free[3:], -1]] and int(c.refs.min()) == 1
    k = randn(torch, 102, 1, 1, 1, 9, 64).cuda()
    cb.cb_cache_write(c.desc, k, k, ints(torch, [0]))
    out = torch.empty_like(k)
    cb.cb_cache_read(c.desc, out, k.clone(), ints(torch, [0]))
    assert np.array_equal(ref.to_f64(out), ref.values(*ref.quantise(ref.to_f64(k))))
    cb.cb_cache_extend(c.desc, ints(torch, [1]), ints(torch, [1]), c.status)
    assert c.status.item() == 1
    cb.cb_cache_free(c.desc, ints(torch, [0, 2]))
    assert c.refs[pages - 7:].tolist() == [0, 0, 0, 0, 1, 0, 0]


@pytest.mark.parametrize("dtype,causal,G,m", [("f32", True, 2, 1), ("bf16", False, 4, 1), ("bf16", True, 8, 3)])
def test_a_sequence_of_nearly_2_to_the_31_positions(torch, cb, dtype, causal, G, m):
    """As long as a table allows, most of its entries one page: the row's weights are those of the page and of
    the last positions, many times over.  Its sums have 2^26 / (runs * waves) terms a wave, each rounded: at most half
    a step, and so many of them below 2^18 with 64 runs of four waves; the values of the page's positions
    add up to nearly nothing against those of the end, which makes the limit seen."""
    D, P = 64, 256
    width = ((1 << 31) - (1 << 16)) // P
    c = cb.Cache(1, 1, D, P, 3, 2, width)
    length = width * P - 77
    c.table[0] = 0
    c.table[0, width - 1] = 2
    c.lens[0] = length
    k = 0.3 * randn(torch, 103, 1, 1, 1, P, D)
    v = randn(torch, 104, 1, 1, 1, P, D)
    cb.cb_cache_write(c.desc, k.cuda(), v.cuda(), ints(torch, [0]), ints(torch, [0]))
    k2, v2 = 0.3 * randn(torch, 105, 1, 1, 1, P - 77, D), randn(torch, 106, 1, 1, 1, P - 77, D)
    k2[..., 3] = 40.0                                        # the last page's positions weigh as much as all others
    q = randn(torch, 107, 1, 1, G, m, D)
    q[..., 3] = 4.3
    cb.cb_cache_write(c.desc, k2.cuda(), v2.cuda(), ints(torch, [0]), ints(torch, [(width - 1) * P]))
    got = torch.zeros((1, 1, 1, P - 77, D), device="cuda")
    cb.cb_cache_read(c.desc, got, torch.empty_like(got), ints(torch, [0]))   # the last P - 77 positions
    assert np.array_equal(ref.to_f64(got), ref.values(*ref.quantise(ref.to_f64(k2))))
    q = q.to(dt(torch, dtype)).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device="cuda")
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q), lse, ints(torch, [0]), causal=causal)
    kk, vv = (ref.values(*ref.quantise(ref.to_f64(x[0, 0, 0]))) for x in (k, v))
    ke, ve = (ref.values(*ref.quantise(ref.to_f64(x[0, 0, 0]))) for x in (k2, v2))
    many = width - 1
    for g, r in itertools.product(range(G), range(m)):
        x = ref.to_f64(q[0, 0, g, r])
        end = P - 77 - (m - 1 - r if causal else 0)
        za, zb = kk @ x / math.sqrt(D), ke[:end] @ x / math.sqrt(D)
        top = max(za.max(), zb.max())
        wa, wb = many * np.exp(za - top), np.exp(zb - top)
        z = wa.sum() + wb.sum()
        want = (wa @ vv + wb @ ve[:end]) / z
        size = (wa @ np.abs(vv) + wb @ np.abs(ve[:end])) / z
        err = ((D + 4) / math.sqrt(D) * (np.abs(np.concatenate([kk, ke])) @ np.abs(x)).max() + 2 * abs(top)) * U
        lost = 2 * err + 2.0 ** 18 * U + (2.0 ** -16 + 0 if dtype == "bf16" and G * m <= 16 else UB if dtype == "bf16" else 0)
        tol = size * lost + (UB * (np.abs(want) + size * lost) if dtype == "bf16" else 0)
        assert (np.abs(ref.to_f64(out[0, 0, g, r]) - want) <= tol).all()
        assert abs(lse[0, 0, g, r].item() - (top + math.log(z))) <= err + 2.0 ** 18 * U + 8 * U * abs(top + math.log(z))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,G,m,lens", [(64, 1, 3001, [4000]), (128, 128, 1, [700, 50]), (128, 71, 9, [500]), (64, 2, 1500, [1, 900])])
def test_attend_wide_groups_and_thousands_of_tokens(torch, cb, dtype, D, G, m, lens):
    """128 query heads a KV head, a group that is no power of two, 3001 query tokens; every row against 64 bits.
    Tolerances as in check_attend."""
    c = cache_with(torch, cb, lens, H=1, D=D, P=64)
    fill_cache(torch, cb, c, lens, 110)
    q = randn(torch, 111, 1, len(lens), G, m, D).to(dt(torch, dtype)).cuda()
    out = torch.empty_like(q)
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q))
    mm, qd, od = model(c, D, 64), ref.to_f64(q), ref.to_f64(out)
    for i, T in enumerate(lens):
        k, v, _ = mm.read(i, 0, 0)
        for g in range(G):
            z = qd[0, i, g] @ k.T / math.sqrt(D)
            err = ((D + 4) / math.sqrt(D) * (np.abs(qd[0, i, g]) @ np.abs(k).T) + 2 * np.abs(z)).max(1, keepdims=True)
            limit = T - m + np.arange(m)[:, None] + 1
            z = np.where(np.arange(T) < limit, z, -np.inf)
            w = np.exp(z - np.where(limit > 0, z.max(1, keepdims=True), 0.0))
            p = w / np.where(limit > 0, w.sum(1, keepdims=True), 1.0)
            want, size = p @ v, p @ np.abs(v)
            tol = size * (2 * err + T / 128 + 56) * U + 2.0 ** -126 * np.abs(v).sum(0)
            if dtype == "bf16":
                tol = tol + UB * (size + np.abs(want))
            assert (np.abs(od[0, i, g] - want) <= tol).all()


# ---- the documents' example ----------------------------------------------------------


def readme_example():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "README.md")).read()
    blocks = [b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "cb_cache_fork" in b]
    assert len(blocks) == 1
    return blocks[0]


def test_the_example_of_the_readme(torch, cb):
    got = {}
    exec(readme_example(), got)
    c, q, out = got["c"], got["q"], got["out"]
    assert c.lens.tolist() == [1000, 1000, 1000, 0]
    m = model(c, got["D"], 64)
    for l, i, h in [(0, 0, 0), (1, 1, 31)]:
        k, v, there = m.read(1 + i, l, h // 4)
        x = ref.to_f64(q[l, i, h, 0])
        want, _, err, size, _ = ref.attend(x, k, v, 1000, there, 1 / math.sqrt(got["D"]))
        tol = size * (2.0 ** -16 + (2 * err + 64) * U) + UB * (np.abs(want) + size * 2.0 ** -15)
        assert (np.abs(ref.to_f64(out[l, i, h, 0]) - want) <= tol).all()


def test_the_example_of_the_readme_says_when_pages_lack(torch, cb):
    """A message of 16 pages and room for 8: nothing is held, so nothing may be answered from it."""
    text = readme_example()
    assert "pages=64" in text
    with pytest.raises(AssertionError):
        exec(text.replace("pages=64", "pages=8"), {})
