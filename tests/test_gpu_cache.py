"""Rotary positions, the paged four-bit cache and attention over it on MI355X, through the public calls,
against the plain 64-bit forms of cache_ref.

Tolerances are derived from the arithmetic: u = 2^-24 is half a step of fp32 (relative), 2^-8 of bf16.
"""
from __future__ import annotations

import itertools
import math

import numpy as np
import pytest

import cache_ref as ref

pytestmark = pytest.mark.gpu

U, UB = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def torch():
    import torch as _torch

    assert _torch.cuda.is_available(), "GPU tests need a GPU"
    return _torch


@pytest.fixture(scope="module")
def cb():
    import paper_2609_32046_amd as _cb

    return _cb


def dt(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def ints(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def randn(torch, seed, *shape):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(shape, generator=g)


# ---- rotary -------------------------------------------------------------------


def check_rotary(torch, y, x, freq, delta, amp, interleaved, transpose, dtype):
    x = ref.to_f64(x)
    want = ref.rotate(x, freq, delta, amp, interleaved, transpose)
    # the turn's remainder in fp32 is off by 2^-26 of a turn at most (2 pi 2^-26 < 1.6 u), sine and cosine
    # by 4 u (two units in the last place), amplitude, two products and a sum by u each
    tol = 12 * U * abs(amp) * ref.pair_size(x, 2 * len(freq), interleaved)
    if dtype == "bf16":
        tol += UB * np.abs(want) * 1.01
    err = np.abs(ref.to_f64(y) - want)
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(64, 64), (128, 128), (128, 64), (128, 70), (64, 2), (8, 8), (72, 16), (256, 128)])
def test_rotary(torch, cb, dtype, interleaved, D, R):
    """Queries and keys of one call: shared positions, part of the head, both directions, heads that do
    not divide by the rows a thread takes."""
    freq, amp = cb.cb_rotary_frequencies(R, 1e6, "yarn", 4.0, 4096)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    q = randn(torch, 1, 2, 5, 7, D).to(dt(torch, dtype)).cuda()
    k = randn(torch, 2, 2, 3, 7, D).to(dt(torch, dtype)).cuda()
    pos = ints(torch, [[[0, 1, 2, 31999, 2**20 + 7, 2**31 - 1, 5]], [[9, 8, 7, 6, 5, 4, -3]]])
    for transpose in (False, True):
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        cb.cb_rotary([cb.rows(q, qo, pos), cb.rows(k, ko, pos)], fd, amp, interleaved, transpose)
        qi, ki = q.clone(), k.clone()   # in place: the same bits
        cb.cb_rotary([cb.rows(qi, qi, pos), cb.rows(ki, ki, pos)], fd, amp, interleaved, transpose)
        assert torch.equal(qi, qo) and torch.equal(ki, ko)
        for x, y in ((q, qo), (k, ko)):
            d = pos.cpu().numpy().astype(np.float64) * np.ones((2, x.shape[1], 7))
            check_rotary(torch, y, x, freq, d, amp, interleaved, transpose, dtype)


def test_rotary_move_in_place_of_strided_rows(torch, cb):
    """Kept keys of every head from their own old positions, in place, in a [token][head] layout
    within a wider buffer; what lies around the rows stays."""
    D, H, T = 128, 6, 45
    freq, _ = cb.cb_rotary_frequencies(D, 1e4)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    buf = randn(torch, 3, 1, T, H + 2, D + 16).bfloat16().cuda()
    before = buf.clone()
    x = buf[:, :, 1:H + 1, 8:D + 8].transpose(1, 2)         # [1][H][T][D]
    old = torch.sort(torch.randint(0, 50000, (H, T), dtype=torch.int32), 1)[0].cuda()
    new = torch.arange(T, dtype=torch.int32, device="cuda")
    cb.cb_rotary(cb.rows(x, x, new, old.reshape(1, H, T)), fd)
    src = before[:, :, 1:H + 1, 8:D + 8].transpose(1, 2)
    d = (new.cpu().numpy() - old.cpu().numpy().astype(np.int64)).reshape(1, H, T)
    check_rotary(torch, x, src, freq, d, 1.0, False, False, "bf16")
    x.copy_(src)
    assert torch.equal(buf.view(torch.int16), before.view(torch.int16))


def test_rotary_gradient(torch, cb):
    """transpose is the gradient: against the formula by autograd in 64 bits, and against differences
    of the forward pass."""
    D, R = 64, 32
    freq, amp = cb.cb_rotary_frequencies(R, 1e4, "yarn", 2.0, 512)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    pos = torch.arange(900, 911, dtype=torch.int32, device="cuda")
    x, dy = randn(torch, 4, 1, 2, 11, D).cuda(), randn(torch, 5, 1, 2, 11, D).cuda()
    dx, y = torch.empty_like(x), torch.empty_like(x)
    cb.cb_rotary(cb.rows(dy, dx, pos), fd, amp, transpose=True)
    xx = x.double().cpu().requires_grad_()
    ang = 2 * math.pi * pos.cpu().double()[:, None] * torch.tensor(freq, dtype=torch.float64)
    a, b = xx[..., :R // 2], xx[..., R // 2:R]
    yy = torch.cat([amp * (a * ang.cos() - b * ang.sin()), amp * (b * ang.cos() + a * ang.sin()), xx[..., R:]], -1)
    (yy * dy.cpu().double()).sum().backward()
    tol = 12 * U * amp * ref.pair_size(ref.to_f64(dy), R, False) + 1e-12
    assert (np.abs(ref.to_f64(dx) - xx.grad.numpy()) <= tol).all()
    # the map is linear: <A(x + h) - A(x), dy> = <h, dx>, up to the two passes' rounding
    h = randn(torch, 6, 1, 2, 11, D).cuda()
    y2 = torch.empty_like(x)
    cb.cb_rotary(cb.rows(x, y, pos), fd, amp)
    cb.cb_rotary(cb.rows(x + h, y2, pos), fd, amp)
    lhs = ((y2.double() - y.double()) * dy.double()).sum().item()
    moved = (x + h).double() - x.double()
    rhs = (moved * dx.double()).sum().item()
    bound = 2 * 12 * U * amp * ((x.abs() + h.abs()).double().amax().item() * 4) * dy.abs().double().sum().item()
    assert abs(lhs - rhs) <= bound


def test_rotary_sizes(torch, cb):
    """No rows, one row, more rows along the outer axes than a grid has, 64-bit offsets."""
    freq, _ = cb.cb_rotary_frequencies(8, 1e4)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    one = ints(torch, [3])
    for shape in [(0, 2, 3, 8), (2, 0, 3, 8), (2, 2, 0, 8)]:
        x = torch.empty(shape, device="cuda")
        cb.cb_rotary(cb.rows(x, x, one), fd)
    x = randn(torch, 7, 70000, 1, 1, 8).cuda()
    y = torch.empty_like(x)
    pos = torch.arange(70000, dtype=torch.int32, device="cuda").reshape(-1, 1, 1)
    cb.cb_rotary(cb.rows(x, y, pos), fd)
    check_rotary(torch, y, x, freq, np.arange(70000).reshape(-1, 1, 1), 1.0, False, False, "f32")
    big = torch.zeros((1, 1, 3, 1 << 31), dtype=torch.bfloat16, device="cuda")[..., :8]   # rows 4 GB apart
    big.copy_(randn(torch, 8, 1, 1, 3, 8).bfloat16())
    want = big.clone()
    cb.cb_rotary(cb.rows(big, big, ints(torch, [1, 2, 3])), fd)
    check_rotary(torch, big, want, freq, np.array([[[1, 2, 3]]]), 1.0, False, False, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R,T", [(1024, 8, 5), (1024, 1022, 40), (1024, 512, 9), (64, 16, 700), (64, 38, 301), (128, 70, 130),
                                     (72, 72, 257), (8, 2, 1000), (128, 64, 1)])
def test_rotary_parts_of_many_rows(torch, cb, dtype, D, R, T):
    """Rows over several workgroups, of one row and of many, with more turned or more copied pieces."""
    freq, amp = cb.cb_rotary_frequencies(R, 1e4)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    x = randn(torch, D + R, 1, 2, T, D).to(dt(torch, dtype)).cuda()
    y, pos = torch.full_like(x, 7.0), torch.arange(T, dtype=torch.int32, device="cuda")
    cb.cb_rotary(cb.rows(x, y, pos), fd, amp)
    check_rotary(torch, y, x, freq, np.arange(T) * np.ones((1, 2, T)), amp, False, False, dtype)
    assert torch.equal(y[..., R:], x[..., R:])


def test_rotary_refuses_tensors(torch, cb):
    x, p = torch.zeros((1, 1, 2, 8), device="cuda"), ints(torch, [0, 1])
    f = torch.zeros(4, dtype=torch.float64, device="cuda")
    for bad in [lambda: cb.rows(x.half(), x.half(), p), lambda: cb.rows(x, x.bfloat16(), p),
                lambda: cb.rows(x, x, p.long()), lambda: cb.rows(x, x, ints(torch, [1, 2, 3])),
                lambda: cb.rows(x.cpu(), x.cpu(), p), lambda: cb.rows(x[0], x[0], p),
                lambda: cb.rows(x.transpose(2, 3), x.transpose(2, 3), p),
                lambda: cb.cb_rotary(cb.rows(x, x, p), f.float()),
                lambda: cb.cb_rotary(cb.rows(x, x, p), f.repeat(2)),
                lambda: cb.cb_rotary([cb.rows(x, x, p), cb.rows(x.bfloat16(), x.bfloat16(), p)], f)]:
        with pytest.raises(cb.CBError):
            bad()


# ---- the cache: rows in and out -------------------------------------------------


def cache_with(torch, cb, lens, L=1, H=2, D=64, P=16, extra=3, width=None, seed=0, holes=()):
    """A cache whose sequences have `lens` positions in scattered pages; pool bytes random everywhere."""
    rng = np.random.default_rng(seed)
    need = [-(-n // P) for n in lens]
    width = max(max(need), 1) + 1 if width is None else width
    pages = sum(need) + extra
    c = cb.Cache(L, H, D, P, pages, len(lens), width)
    c.pool.copy_(torch.from_numpy(rng.integers(0, 256, c.pool.shape).astype(np.uint8)))
    order, at = rng.permutation(pages), 0
    table, refs = np.full((len(lens), width), -1, np.int32), np.zeros(pages, np.int32)
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        refs[order[at:at + n]] = 1
        at += n
    for s, j in holes:
        table[s, j] = -1
    c.table.copy_(torch.from_numpy(table))
    c.refs.copy_(torch.from_numpy(refs))
    c.lens.copy_(ints(torch, lens))
    return c


def model(c, D, P):
    return ref.Model(c.pool.cpu().numpy(), c.refs.cpu().numpy(), c.table.cpu().numpy(), c.lens.cpu().numpy(), D, P)


def same_state(c, m, pool=True):
    assert np.array_equal(c.refs.cpu().numpy(), m.refs)
    assert np.array_equal(c.lens.cpu().numpy(), m.lens)
    assert np.array_equal(c.table.cpu().numpy(), m.table)
    if pool:
        assert np.array_equal(c.pool.cpu().numpy(), m.pool)


def hard_rows(torch, seed, *shape):
    """Rows of every size, with zeros, ties, the largest and smallest magnitudes, NaN and infinities."""
    x = randn(torch, seed, *shape)
    g = x.view(*shape[:-1], shape[-1] // 32, 32).flatten(0, -2)
    n = g.shape[0]
    rng = np.random.default_rng(seed)
    g *= torch.from_numpy(np.exp2(rng.integers(-20, 20, (n, 1))).astype(np.float32))
    kinds = [lambda r: r.zero_(), lambda r: r.copy_(torch.tensor([7, 5, 3.5, 2.5, 1.75, 1.25, .75, .25] * 4)),
             lambda r: r.mul_(3e38 / r.abs().max()), lambda r: r.mul_(1e-37 / r.abs().max()),
             lambda r: r.mul_(2e-39 / r.abs().max()), lambda r: r[3:4].fill_(math.nan),
             lambda r: r[31:].fill_(math.inf), lambda r: r[:1].fill_(-math.inf),
             lambda r: r.copy_(torch.tensor([-0.0, 0.0] * 16)), lambda r: r.mul_(7.0 / r.abs().max())]
    for i, f in enumerate(kinds):
        if i < n:
            f(g[(i * 7 + 1) % n])
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (64, 64), (128, 32), (128, 256)])
def test_write_and_read(torch, cb, dtype, D, P):
    """Codes and scales bit for bit, positions in the middle of pages, counts of none, a sequence that
    is named out of order, layers from the second on, everything else left as it was."""
    lens = [5, 70, 0, 33]
    c = cache_with(torch, cb, lens, L=3, H=3, D=D, P=P, seed=P + D)
    m = model(c, D, P)
    seqs, start, counts, T = [3, 1, 0], [2, 13, 0], [31, 40, 0], 41
    k, v = (hard_rows(torch, s + D, 2, 3, 3, T, D).to(dt(torch, dtype)).cuda() for s in (1, 2))
    cb.cb_cache_write(c.desc, k, v, ints(torch, seqs), ints(torch, start), ints(torch, counts), layer=1)
    for x, which in ((k, 0), (v, 1)):
        code, scale = ref.quantise(ref.to_f64(x))
        for l, i, h in itertools.product(range(2), range(3), range(3)):
            for t in range(counts[i]):
                pos = start[i] + t
                page = m.table[seqs[i], pos // P]
                u = list(ref.unpack(m.pool[page, 1 + l, h], P, D))
                u[2 * which][pos % P], u[2 * which + 1][pos % P] = code[l, i, h, t], scale[l, i, h, t]
                m.pool[page, 1 + l, h] = ref.pack(*u)
    same_state(c, m)
    ko, vo = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    cb.cb_cache_read(c.desc, ko, vo, ints(torch, seqs), ints(torch, start), ints(torch, counts), layer=1)
    for x, which in ((ko, 0), (vo, 1)):
        want = np.full(x.shape, 3.0)
        for l, i, h in itertools.product(range(2), range(3), range(3)):
            full = m.read(seqs[i], 1 + l, h)[which]
            want[l, i, h, :counts[i]] = full[start[i]:start[i] + counts[i]]
        assert np.array_equal(ref.to_f64(x), want, equal_nan=True)


def test_write_by_default_goes_behind(torch, cb):
    """Without starts and lists: the last positions of sequences 0, 1, ..: a decoding step's append."""
    D, P = 128, 16
    c = cache_with(torch, cb, [16, 17, 40], H=2, D=D, P=P)
    k, v = randn(torch, 1, 1, 3, 2, 1, D).bfloat16().cuda(), randn(torch, 2, 1, 3, 2, 1, D).bfloat16().cuda()
    cb.cb_cache_write(c.desc, k, v)
    m = model(c, D, P)
    for s, n in enumerate([16, 17, 40]):
        for h in range(2):
            kk, vv, _ = m.read(s, 0, h)
            assert np.array_equal(kk[n - 1], ref.values(*ref.quantise(ref.to_f64(k[0, s, h, 0]))))
            assert np.array_equal(vv[n - 1], ref.values(*ref.quantise(ref.to_f64(v[0, s, h, 0]))))


def test_write_passes_over_what_has_no_page(torch, cb):
    """Positions before the sequence, behind its pages, in a hole of the table, of unknown
    sequences: nothing is written; reads of them are zeros."""
    D, P = 64, 16
    c = cache_with(torch, cb, [40, 20], D=D, P=P, holes=[(0, 1)])
    before = c.pool.clone()
    k = randn(torch, 1, 1, 5, 2, 4, D).cuda()
    seqs, start = ints(torch, [0, 0, 1, 7, -1]), ints(torch, [-4, 20, 32, 0, 0])
    cb.cb_cache_write(c.desc, k, k, seqs, start)
    assert torch.equal(c.pool, before)
    ko, vo = torch.ones_like(k), torch.ones_like(k)
    cb.cb_cache_read(c.desc, ko, vo, seqs, start)
    assert not ko.any() and not vo.any()
    # beyond the table, where position * width passes 32 bits
    far = ints(torch, [2**31 - 100] * 5)
    cb.cb_cache_write(c.desc, k, k, seqs, far)
    cb.cb_cache_read(c.desc, ko.fill_(1), vo.fill_(1), seqs, far)
    assert torch.equal(c.pool, before) and not ko.any()


def test_write_and_read_strided(torch, cb):
    """Rows of a fused [token][q, k, v heads][D] buffer; none of it but the rows changes."""
    D, P, n, T, H = 128, 32, 2, 9, 2
    c = cache_with(torch, cb, [50, 60], H=H, D=D, P=P)
    buf = randn(torch, 1, n, T, 3 * H, D).bfloat16().cuda()
    k = buf[:, :, H:2 * H].transpose(1, 2)[None]
    v = buf[:, :, 2 * H:].transpose(1, 2)[None]
    cb.cb_cache_write(c.desc, k, v, start=ints(torch, [3, 30]))
    out = torch.full_like(buf, 9.0)
    ko, vo = out[:, :, :H].transpose(1, 2)[None], out[:, :, H:2 * H].transpose(1, 2)[None]
    cb.cb_cache_read(c.desc, ko, vo, start=ints(torch, [3, 30]))
    assert np.array_equal(ref.to_f64(ko), ref.values(*ref.quantise(ref.to_f64(k))))
    assert np.array_equal(ref.to_f64(vo), ref.values(*ref.quantise(ref.to_f64(v))))
    assert (out[:, :, 2 * H:] == 9.0).all()


def test_rows_of_a_large_pool(torch, cb):
    """Pages whose bytes lie beyond 32 bits."""
    D, P = 128, 256
    c = cb.Cache(32, 8, D, P, 500, 1, 2)          # 4.4 GB
    c.table[0] = ints(torch, [499, 480])
    c.lens[0] = 400
    c.pool[[480, 499]] = 0
    k = randn(torch, 1, 32, 1, 8, 300, D).bfloat16().cuda()
    cb.cb_cache_write(c.desc, k, k, start=ints(torch, [90]))
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    cb.cb_cache_read(c.desc, ko, vo, start=ints(torch, [90]))
    want = ref.values(*ref.quantise(ref.to_f64(k[31, :, :, :40])))
    assert torch.equal(ko.view(torch.int16), vo.view(torch.int16))
    assert np.array_equal(ref.to_f64(ko[31, :, :, :40]), want)


# ---- pages ----------------------------------------------------------------------


def test_extend(torch, cb):
    D, P = 64, 16
    c = cache_with(torch, cb, [0, 15, 16, 33, 48], D=D, P=P, extra=9, width=6)
    m = model(c, D, P)
    for seqs, add in [([4, 0, 2], [1, 33, 16]), ([1], [1]), ([1, 3], [0, 0]), ([], []),
                      ([0], [1000]), ([0, 0], [1, 1]), ([5], [1]), ([-1], [1]), ([1], [-1]),
                      ([1, 2, 3], [40, 40, 40]), ([1], [64])]:
        cb.cb_cache_extend(c.desc, ints(torch, seqs), ints(torch, add), c.status)
        want = m.extend(seqs, add)
        assert c.status.item() == want, (seqs, add)
        assert cb.cb_cache_status(c.status) == (0 if want == 0 else -2 if want < 0 else -9)
        same_state(c, m)


def test_needs_of_more_than_32_bits(torch, cb):
    """A thousand rows of two million pages: what they ask for together passes 2^31 pages."""
    n, width, P = 1024, 1 << 21, 16
    c = cb.Cache(1, 1, 64, P, 64, n, width)
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    cb.cb_cache_extend(c.desc, seqs, torch.full((n,), width * P, dtype=torch.int32, device="cuda"), c.status)
    assert c.status.item() == n * width - 64
    idx = torch.zeros(width * P, dtype=torch.int32, device="cuda").expand(n, 1, 1, width * P)
    ws = torch.empty(cb.cb_cache_compact_workspace_bytes(c.desc, n), dtype=torch.uint8, device="cuda")
    cb.cb_cache_compact(c.desc, seqs, seqs, idx, c.status, ws)
    assert c.status.item() == n * width - 64
    assert not c.lens.any() and not c.refs.any() and int(c.table.max()) == -1


def test_free(torch, cb):
    """Shared pages stay with their other holders; repeated and unknown entries pass."""
    D, P = 64, 16
    c = cache_with(torch, cb, [40, 20, 0, 100], D=D, P=P)
    c.table[2, :2] = c.table[0, :2]
    c.refs[c.table[0, :2].long()] = 2
    c.lens[2] = 32
    m = model(c, D, P)
    for seqs in ([], [0, 0, 9, -3], [2, 1], [2], [3, 0]):
        cb.cb_cache_free(c.desc, ints(torch, seqs))
        m.free(seqs)
        same_state(c, m)
    assert not c.refs.any()


@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("D,P,L", [(64, 16, 1), (128, 64, 3)])
def test_fork(torch, cb, copy, D, P, L):
    lens = [3 * P + 5, 2 * P, 0, 1, 40, 7, 2 * P + 1, 0, 5]
    c = cache_with(torch, cb, lens, L=L, D=D, P=P, extra=24, width=6)
    m = model(c, D, P)
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, 16), dtype=torch.uint8, device="cuda")
    for parents, children in [([0, 1], [4, 5]), ([0, 0, 1, 2, 3], [5, 6, 4, 7, 8]), ([], []), ([4], [0]),
                              ([0], [0]), ([1, 2], [3, 3]), ([0, 5], [5, 6]), ([9], [1]), ([1], [-1]),
                              ([6, 6, 6], [1, 2, 3])]:
        for _ in range(2):   # once more: the same pages come back
            cb.cb_cache_fork(c.desc, ints(torch, parents), ints(torch, children), c.status, ws, copy)
            assert c.status.item() == m.fork(parents, children, copy), (parents, children)
            same_state(c, m)


def test_fork_without_room_changes_nothing(torch, cb):
    c = cache_with(torch, cb, [40, 30, 20], D=64, P=16, extra=2)
    m = model(c, 64, 16)
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, 4), dtype=torch.uint8, device="cuda")
    cb.cb_cache_fork(c.desc, ints(torch, [0, 0]), ints(torch, [1, 2]), c.status, ws, True)
    assert m.fork([0, 0], [1, 2], True) == 0 and c.status.item() == 0   # the children's own four help
    same_state(c, m)
    c = cache_with(torch, cb, [40, 30, 20], D=64, P=16, extra=1)
    m = model(c, 64, 16)
    cb.cb_cache_fork(c.desc, ints(torch, [0, 0]), ints(torch, [1, 2]), c.status, ws, True)
    assert c.status.item() == m.fork([0, 0], [1, 2], True) == 1
    assert cb.cb_cache_status(c.status) == -9
    same_state(c, m)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("D,P,L,H", [(64, 16, 2, 3), (128, 32, 1, 2), (128, 64, 2, 1)])
def test_compact(torch, cb, shared, D, P, L, H):
    """Into other sequences and in place, ragged counts, lists out of order with repeats and
    positions that do not exist, dst that held pages before, a shared source."""
    lens = [3 * P + 9, 2 * P, 0, 50, 20]
    c = cache_with(torch, cb, lens, L=L, H=H, D=D, P=P, extra=14, width=8)
    c.table[2, :2] = c.table[0, :2]
    c.refs[c.table[0, :2].long()] += 1
    c.lens[2] = 2 * P
    m = model(c, D, P)
    ws = torch.empty(cb.cb_cache_compact_workspace_bytes(c.desc, 8), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(D + P)
    for src, dst, keep, counts in [([0, 3], [4, 3], 37, None), ([0, 0], [1, 3], 2 * P, [2 * P, 1]),
                                   ([2], [2], P + 1, None), ([1, 2], [1, 2], 5, [0, 5]), ([0], [0], 9, None),
                                   ([], [], 3, None), ([0, 1], [1, 1], 3, None), ([0, 1], [1, 2], 3, None),
                                   ([5], [0], 3, None), ([0], [-1], 3, None), ([0], [1], 3, [4]), ([0], [1], 3, [-1]),
                                   ([0], [1], 8 * P, None)]:
        shape = (max(len(src), 1), 1 if shared else L, 1 if shared else H, keep)
        idx = np.sort(rng.integers(0, 3 * P + 12, shape), -1).astype(np.int32)
        idx[..., keep // 2] = [-5, 2**31 - 1][keep % 2]
        idx[..., 0] = idx[..., -1]
        got = torch.from_numpy(idx)[:len(src)].cuda()
        cb.cb_cache_compact(c.desc, ints(torch, src), ints(torch, dst), got, c.status, ws,
                            None if counts is None else ints(torch, counts))
        want = m.compact(src, dst, lambda i, l, h: idx[i, 0 if shared else l, 0 if shared else h], counts)
        assert c.status.item() == want, (src, dst)
        same_state(c, m)


def test_pages_of_a_large_pool(torch, cb):
    """More pages than one sweep of the planning workgroup, nearly all of them held; lists of a
    thousand entries."""
    D, P, pages, n = 64, 16, 70001, 1500
    c = cb.Cache(1, 1, D, P, pages, 2 * n, 4)
    c.refs.fill_(1)
    free = np.sort(np.random.default_rng(0).choice(pages, 2 * n + 3, replace=False))
    c.refs[torch.from_numpy(free).cuda()] = 0
    m = ref.Model(np.zeros((pages, 0)), c.refs.cpu().numpy(), c.table.cpu().numpy(), c.lens.cpu().numpy(), D, P)
    first, second = list(range(n)), list(range(n, 2 * n))
    cb.cb_cache_extend(c.desc, ints(torch, first), ints(torch, [5] * n), c.status)
    assert c.status.item() == m.extend(first, [5] * n) == 0
    same_state(c, m, pool=False)
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, n), dtype=torch.uint8, device="cuda")
    c.pool.random_(0, 256)
    before = c.pool.cpu().numpy()
    m.pool = before.copy()
    cb.cb_cache_fork(c.desc, ints(torch, first), ints(torch, second), c.status, ws)
    assert c.status.item() == m.fork(first, second, False) == 0
    same_state(c, m)
    cb.cb_cache_extend(c.desc, ints(torch, first), ints(torch, [20] * n), c.status)
    assert c.status.item() == m.extend(first, [20] * n) == n - 3   # three are left of 2n + 3
    same_state(c, m)
    cb.cb_cache_free(c.desc, ints(torch, second + first))
    m.free(second + first)
    same_state(c, m)


# ---- attention --------------------------------------------------------------------


def check_attend(torch, m, q, out, lse, seqs, q_lens, causal, scale, layer0, dtype, fill=7.0):
    """Every row against the plain form.  The bound: a logit's error e (of D products in fp32) moves
    the output by at most 2 e sum p|v| and the log-sum by e; the sums run over 32 positions within an
    instruction and over the wave's steps, then over waves and chunks; weights lose 2^-24 and the
    exponential 2 units; with bf16 rows weights and outputs are rounded to 2^-8 once each.  A weight relative to the largest (whose own
    is 1 or more) that lies below 2^-126 is lost to fp32's range: 2^-126 |v| a position."""
    Lq, n, Hq, Q, D = q.shape
    G, qd, od = Hq // m.pool.shape[2], ref.to_f64(q), ref.to_f64(out)
    ld = ref.to_f64(lse) if lse is not None else None
    scale = scale or 1.0 / math.sqrt(D)
    for l, i in itertools.product(range(Lq), range(n)):
        s, T = seqs[i], q_lens[i]
        if T <= 0:
            assert (od[l, i] == fill).all()
            continue
        length = int(m.lens[s])
        for h in range(m.pool.shape[2]):
            k, v, there = m.read(s, layer0 + l, h)
            for g, r in itertools.product(range(G), range(Q)):
                got = od[l, i, h * G + g, r]
                if r >= T:
                    assert (got == fill).all()
                    continue
                limit = length - T + r + 1 if causal else length
                want, z, err, size, lost = ref.attend(qd[l, i, h * G + g, r], k, v, limit, there, scale)
                steps = length / 128 + 48
                tol = size * (2 * err + steps + 8) * U + lost
                if dtype == "bf16":
                    tol = tol + UB * (size + np.abs(want))
                bad = np.isnan(want)
                assert np.array_equal(np.isnan(got), bad), (l, i, h, g, r)
                diff = np.abs(got - want)[~bad]
                assert (diff <= tol[~bad] if np.ndim(tol) else diff <= tol).all(), \
                    (l, i, h, g, r, float((diff - tol[~bad]).max()))
                if ld is not None:
                    zg = ld[l, i, h * G + g, r]
                    if math.isinf(z) or math.isnan(z):
                        assert zg == z or (math.isnan(z) and math.isnan(zg))
                    else:
                        assert abs(zg - z) <= (err + steps + 8 + 4 * abs(z)) * U, (l, i, h, g, r)


def fill_cache(torch, cb, c, lens, seed, layers=1, start=None):
    """Real rows at every position (channels of unlike size)."""
    n, H, D = len(lens), c.pool.shape[2], c.desc.head_dim
    T = max(max(lens), 1)
    k = randn(torch, seed, layers, n, H, T, D) * (0.5 + 1.5 * randn(torch, seed + 1, 1, 1, H, 1, D).abs())
    v = randn(torch, seed + 2, layers, n, H, T, D)
    cb.cb_cache_write(c.desc, k.cuda(), v.cuda(), start=ints(torch, [0] * n), counts=ints(torch, lens))


def scratch(torch, cb, c, q):
    """Scratch of an attention call, of any contents."""
    n = cb.cb_cache_attend_workspace_bytes(c.desc, q.shape[0], q.shape[1], q.shape[2], q.shape[3])
    return torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda") if n else None


def attend_case(torch, cb, lens, Hkv, G, D, P, m, dtype, causal, seqs=None, q_lens=None, layers=1, layer0=0,
                scale=0.0, seed=0, holes=(), prepare=None, extra=3, cut=False):
    """cut: a table of more than 4096 positions, whose sequences are cut into runs, however short they are."""
    c = cache_with(torch, cb, lens, L=layers + layer0, H=Hkv, D=D, P=P, seed=seed, extra=extra,
                   width=8192 // P if cut else None)
    fill_cache(torch, cb, c, lens, seed, layers + layer0)
    for s, j in holes:
        c.table[s, j] = -1
    if prepare:
        prepare(c)
    seqs_ = list(range(len(lens))) if seqs is None else seqs
    n = len(seqs_)
    q = randn(torch, seed + 5, layers, n, Hkv * G, m, D).to(dt(torch, dtype)).cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:4], 7.0, device="cuda")
    ws = scratch(torch, cb, c, q)
    cb.cb_cache_attend(c.desc, q, out, ws, lse, None if seqs is None else ints(torch, seqs),
                       None if q_lens is None else ints(torch, q_lens), causal, scale, layer0)
    clipped = [m] * n if q_lens is None else [max(0, min(x, m)) for x in q_lens]
    check_attend(torch, model(c, D, P), q, out, lse, seqs_, clipped, causal, scale, layer0, dtype)
    for i, x in enumerate(clipped):
        assert (lse[:, i, :, x:] == 7.0).all()
    return c, q, out, lse, ws


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P,Hkv,G", [(128, 64, 2, 4), (64, 16, 2, 2), (128, 16, 1, 5), (64, 128, 3, 1),
                                       (128, 256, 1, 8), (64, 32, 1, 17)])
def test_attend_single_tokens(torch, cb, dtype, D, P, Hkv, G, cut):
    """Decoding: one query token a sequence, every length around the tiles and pages."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]
    attend_case(torch, cb, lens, Hkv, G, D, P, 1, dtype, True, seed=D + P + G, cut=cut)


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P,G,m", [(128, 32, 4, 5), (64, 16, 3, 7), (128, 16, 1, 33), (64, 64, 8, 20), (128, 128, 5, 50),
                                       (64, 16, 7, 40), (128, 32, 8, 65), (64, 16, 8, 65)])
def test_attend_several_tokens(torch, cb, causal, dtype, D, P, G, m, cut):
    """Prompts' parts: more query tokens than positions (rows of no position), ragged query counts, one
    of none, sequences named out of order and twice, the second layer."""
    lens = [40, 3, 0, 150, m]
    attend_case(torch, cb, lens, 2, G, D, P, m, dtype, causal, seqs=[3, 0, 4, 1, 3, 2, 0],
                q_lens=[m, max(1, m // 2), m + 9, m, 0, m, -1], layers=1, layer0=1, seed=m + G, cut=cut)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_long_sequences_in_chunks(torch, cb, dtype):
    """Rows cut into many chunks beside short and empty ones; the second kernel joins them."""
    attend_case(torch, cb, [5000, 0, 1, 700, 2049], 1, 4, 128, 64, 1, dtype, True, seed=3)
    attend_case(torch, cb, [3001, 1300], 1, 6, 64, 16, 7, dtype, True, seed=4)
    attend_case(torch, cb, [2600], 2, 2, 128, 32, 3, dtype, False, layers=2, seed=5)
    attend_case(torch, cb, [2100, 0, 900], 1, 4, 128, 64, 60, dtype, True, seed=16)
    attend_case(torch, cb, [2100, 300], 1, 5, 64, 16, 50, dtype, False, seed=17, holes=[(0, 3), (0, 130), (1, 0)])


def test_attend_many_sequences(torch, cb):
    """More sequences than lanes, so that the search for a chunk takes several rounds."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 90, 150)] + [1200]
    attend_case(torch, cb, lens, 1, 2, 64, 16, 1, "bf16", True, seed=6, cut=True)
    attend_case(torch, cb, lens, 1, 2, 64, 16, 1, "bf16", True, seed=6)


def test_attend_told_the_longest(torch, cb):
    """A bound on the lengths spares the scratch of a wide table and changes nothing of a bound that holds; a longer
    sequence is taken to be as long as it says."""
    lens, D, P, m = [0, 17, 1000, 130], 128, 16, 3
    c, q, out, _, _ = attend_case(torch, cb, lens, 2, 3, D, P, m, "bf16", True, seed=33, cut=True)
    for longest in (1000, 1001, 130, 1):
        assert cb.cb_cache_attend_workspace_bytes(c.desc, 1, 4, 6, m, longest) == 0
        out.fill_(7.0)
        cb.cb_cache_attend(c.desc, q, out, longest=longest)
        got = model(c, D, P)
        got.lens = np.minimum(got.lens, longest)
        check_attend(torch, got, q, out, None, [0, 1, 2, 3], [m] * 4, True, 0.0, 0, "bf16")
    with pytest.raises(cb.CBError):
        cb.cb_cache_attend(c.desc, q, out, longest=5000)   # cut after all: it needs scratch
    with pytest.raises(cb.CBError):
        cb.cb_cache_attend(c.desc, q, out, longest=-1)


def test_attend_scale_and_large_logits(torch, cb):
    """A scale of its own; logits of several hundred; equal logits."""
    attend_case(torch, cb, [100, 400], 1, 2, 64, 16, 3, "f32", True, scale=0.31, seed=7)
    attend_case(torch, cb, [100, 400], 1, 2, 64, 16, 3, "f32", True, scale=9.0, seed=8)
    attend_case(torch, cb, [100, 400], 1, 2, 128, 16, 3, "bf16", True, scale=9.0, seed=9)
    attend_case(torch, cb, [100, 400], 1, 2, 128, 16, 3, "bf16", True, scale=1e-30, seed=10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,P,G,m", [(128, 32, 4, 1), (64, 16, 2, 8), (128, 16, 3, 9), (64, 64, 8, 4), (128, 64, 4, 16),
                                       (64, 32, 5, 25), (128, 128, 8, 17)])
def test_attend_hundreds_of_short_sequences(torch, cb, dtype, D, P, G, m):
    """So many that each wave takes rows of its own: 400 entries over eight sequences."""
    crowd(torch, cb, dtype, D, P, G, m, 400, [0, 1, 16, 17, 33, 100, 128, 64])


@pytest.mark.parametrize("D,P,G,m,n,longest", [(128, 64, 4, 16, 6400, 128), (64, 32, 5, 25, 3200, 128),
                                                 (128, 64, 4, 16, 400, 2000), (64, 16, 8, 9, 300, 2000)])
def test_attend_crowds_in_tiles_of_64_rows(torch, cb, D, P, G, m, n, longest):
    """Enough steps for four blocks a wave: one wave a workgroup, and four over whole sequences."""
    crowd(torch, cb, "bf16", D, P, G, m, n, [0, 1, 16, 17, 33, 100, longest, 64])


def crowd(torch, cb, dtype, D, P, G, m, n, lens):
    """n entries over eight sequences, most of no or one query token, some of all."""
    rng = np.random.default_rng(m)
    q_lens = [int(x) for x in rng.choice([0, 1], n, p=[0.9, 0.1])]
    for i in range(8):
        q_lens[n // 8 * i + i] = [m, m + 3, (m + 1) // 2][i % 3]
    attend_case(torch, cb, lens, 1, G, D, P, m, dtype, True, seqs=[i % 8 for i in range(n)], q_lens=q_lens,
                seed=m + G + D)


@pytest.mark.parametrize("rest,cut", [(0, False), (1198, False), (18, True)])
@pytest.mark.parametrize("dtype,G", [("bf16", 3), ("f32", 3), ("bf16", 20), ("bf16", 30)])
def test_attend_masked_places_hold_anything(torch, cb, dtype, G, rest, cut):
    """Positions behind the limit with NaN groups, infinite values and any bytes: rows that do not see
    them stay as they are, rows that do are NaN in the group's values (or wholly, for a key)."""
    D, P, lens, m = 128, 32, [75, 40], 12

    def spoil(c):
        n, s = P * D // 2, P * D // 32
        pages = c.table.cpu().numpy()
        for q in range(75 - 64, P):               # behind the end: scale bytes of NaN and of overflow
            u = c.pool[int(pages[0, 2]), 0]
            u[:, 2 * n + q * 4:2 * n + q * 4 + 4] = 255
            for g in range(4):
                u[:, 2 * n + s + (q // 4 * 4 + g) * 4 + q % 4] = 254 + g % 2
        # position 70 of sequence 0: the second value group is NaN; rows 7.. of its 12 see it
        q = 70 - 64
        c.pool[int(pages[0, 2]), 0, :, 2 * n + s + (q // 4 * 4 + 1) * 4 + q % 4] = 255
        # position 38 of sequence 1: a key group is NaN; rows 10 and 11 see it
        q = 38 - 32
        c.pool[int(pages[1, 1]), 0, :, 2 * n + q * 4 + 2] = 255

    # rest: entries of no query token; beside many of them a workgroup is one wave
    _, _, out, _, _ = attend_case(torch, cb, lens, 1, G, D, P, m, dtype, True, seed=11, prepare=spoil,
                                  seqs=[0, 1] + [0] * rest, q_lens=[m, m] + [0] * rest, cut=cut)
    nan = torch.isnan(out[0, 0])                  # [heads][rows][D]
    assert nan[:, 7:, 32:64].all() and not nan[:, :7].any() and not nan[:, 7:, :32].any()
    nan = torch.isnan(out[0, 1])
    assert nan[:, 10:].all() and not nan[:, :10].any()


@pytest.mark.parametrize("dtype,m", [("f32", 1), ("bf16", 1), ("bf16", 110)])
def test_attend_nan_in_the_open(torch, cb, dtype, m):
    """A NaN value group far from any mask reaches every row, in its group only."""
    D, P = 64, 16

    def spoil(c):
        n, s = P * D // 2, P * D // 32
        c.pool[int(c.table[0, 3]), 0, 0, 2 * n + s + (5 // 4 * 2 + 1) * 4 + 5 % 4] = 255

    _, _, out, _, _ = attend_case(torch, cb, [1000], 1, 2, D, P, m, dtype, True, seed=12, prepare=spoil)
    assert torch.isnan(out[..., 32:]).all() and not torch.isnan(out[..., :32]).any()


def test_attend_positions_without_a_page(torch, cb):
    """Holes in the table count for nothing, a sequence of holes only is an empty one; entries behind the pool and unknown
    sequences do no harm."""
    attend_case(torch, cb, [100, 30, 500], 1, 2, 64, 16, 2, "f32", False, seed=13,
                holes=[(0, 2), (1, 0), (1, 1), (2, 0), (2, 31), (2, 7)])
    c = cache_with(torch, cb, [40, 20], D=64, P=16)
    fill_cache(torch, cb, c, [40, 20], 1)
    c.table[0, 1] = c.pool.shape[0] + 5
    q = randn(torch, 1, 1, 3, 2, 1, 64).cuda()
    out, lse = torch.ones_like(q), torch.ones(q.shape[:4], device="cuda")
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q), lse, seqs=ints(torch, [0, 99, -1]))
    assert not out[:, 1:].any() and (lse[:, 1:] == -math.inf).all()
    m = model(c, 64, 16)
    check_attend(torch, m, q[:, :1], out[:, :1], lse[:, :1], [0], [1], True, 0.0, 0, "f32")


def test_attend_strided_rows(torch, cb):
    """q within a fused [token][heads][D] buffer, out token-major; the rest of both is left."""
    D, P, lens, m, Hkv, G = 128, 16, [50, 90], 4, 2, 2
    c = cache_with(torch, cb, lens, H=Hkv, D=D, P=P)
    fill_cache(torch, cb, c, lens, 2)
    buf = randn(torch, 3, 2, m, 3 * Hkv * G, D).bfloat16().cuda()
    q = buf[:, :, :Hkv * G].transpose(1, 2)[None]
    room = torch.full((2, m, Hkv * G + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, :, 1:].transpose(1, 2)[None]
    cb.cb_cache_attend(c.desc, q, out, scratch(torch, cb, c, q))
    check_attend(torch, model(c, D, P), q, out, None, [0, 1], [m, m], True, 0.0, 0, "bf16")
    assert (room[:, :, 0] == 7.0).all()


def test_attend_is_deterministic_and_composes(torch, cb):
    """The same bits on a second run, on another stream, and from a captured graph replayed between eager
    work; two halves of a sequence joined by their log-sums give the whole."""
    c, q, out, lse, ws = attend_case(torch, cb, [4000, 900], 2, 4, 128, 64, 1, "f32", False, seed=14)
    first, flse = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cb.cb_cache_attend(c.desc, q, out.zero_(), ws, lse, causal=False)
    side.synchronize()
    assert torch.equal(out, first) and torch.equal(lse, flse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cb.cb_cache_attend(c.desc, q, out, ws, lse, causal=False)
    for i in range(3):
        out.zero_()
        q.copy_(randn(torch, 20 + i, *q.shape).cuda())
        g.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        cb.cb_cache_attend(c.desc, q, want, ws, lse, causal=False)
        assert torch.equal(out, want)


def test_attend_two_calls_at_once(torch, cb):
    """Two streams, each with its own scratch, on one cache."""
    c, q, out, lse, ws = attend_case(torch, cb, [3000, 2000], 2, 4, 64, 32, 1, "bf16", True, seed=15)
    want = out.clone()
    outs = [torch.empty_like(out) for _ in range(2)]
    wss = [torch.empty_like(ws) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s, o, w in zip(streams, outs, wss):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                cb.cb_cache_attend(c.desc, q, o, w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_calls_refuse_tensors(torch, cb):
    c = cache_with(torch, cb, [20], D=64, P=16)
    k = torch.zeros((1, 1, 2, 3, 64), device="cuda")
    one = ints(torch, [0])
    for bad in [lambda: cb.cb_cache_write(c.desc, k, k.bfloat16()), lambda: cb.cb_cache_write(c.desc, k.half(), k.half()),
                lambda: cb.cb_cache_write(c.desc, k[:, :, :1], k[:, :, :1]), lambda: cb.cb_cache_write(c.desc, k.cpu(), k),
                lambda: cb.cb_cache_write(c.desc, k, k, one.long()), lambda: cb.cb_cache_write(c.desc, k, k, ints(torch, [0, 0])),
                lambda: cb.cb_cache_read(c.desc, k, k[..., :32]), lambda: cb.cb_cache_read(c.desc, k, k, layer=1),
                lambda: cb.cb_cache_attend(c.desc, k, k[:, :, :1]), lambda: cb.cb_cache_attend(c.desc, k.half(), k.half()),
                lambda: cb.cb_cache_attend(c.desc, k[:, :, :, :, :32], k[:, :, :, :, :32]),
                lambda: cb.cb_cache_attend(c.desc, k, k.clone(), lse=torch.zeros((1, 1, 2, 3), device="cuda").half()),
                lambda: cb.cb_cache_extend(c.desc, one, ints(torch, [1, 2]), c.status),
                lambda: cb.cb_cache_fork(c.desc, one, one, c.status, None),
                lambda: cb.cb_cache_compact(c.desc, one, one, torch.zeros((1, 2, 2, 4), dtype=torch.int32, device="cuda"),
                                            c.status, None),
                lambda: cb.cache(c.pool, c.refs, c.table, c.lens, 128, 16), lambda: cb.cache(c.pool[0], c.refs, c.table, c.lens, 64, 16),
                lambda: cb.cache(c.pool, c.refs[1:], c.table, c.lens, 64, 16)]:
        with pytest.raises(cb.CBError):
            bad()


def test_calls_refuse_other_devices_and_wide_sizes(torch, cb):
    """A cache or rows described on another device than the current one; sizes that C takes in 32 bits."""
    c = cache_with(torch, cb, [20], D=64, P=16)
    k = torch.zeros((1, 1, 2, 3, 64), device="cuda")
    one, wide = ints(torch, [0]), k[:, :, :, :1].expand(1, 2**32 + 1, 2, 1, 64)
    freq = torch.zeros(2**10, dtype=torch.float64, device="cuda")
    moved = cb.rows(k[0], k[0], one)
    moved.dev = 1   # as if made there
    for bad in [lambda: cb.cb_rotary(moved, freq[:32]), lambda: cb.cb_rotary(cb.rows(k[0], k[0], one), freq),
                lambda: cb.cb_cache_write(c.desc, wide, wide), lambda: cb.cb_cache_read(c.desc, k, k.clone(), layer=2**32),
                lambda: cb.cb_cache_attend(c.desc, k, k.clone(), layer=2**32),
                lambda: cb.cb_cache_attend(c.desc, wide, wide),
                lambda: cb.cb_rotary_frequencies(2**32 + 64)]:
        with pytest.raises(cb.CBError):
            bad()
    c.desc.dev = 1
    ws = torch.zeros(1 << 12, dtype=torch.uint8, device="cuda")
    idx = torch.zeros((1, 1, 1, 4), dtype=torch.int32, device="cuda")
    for bad in [lambda: cb.cb_cache_write(c.desc, k, k), lambda: cb.cb_cache_read(c.desc, k, k.clone()),
                lambda: cb.cb_cache_attend(c.desc, k, k.clone()), lambda: cb.cb_cache_extend(c.desc, one, one, c.status),
                lambda: cb.cb_cache_free(c.desc, one), lambda: cb.cb_cache_fork(c.desc, one, one, c.status, ws),
                lambda: cb.cb_cache_compact(c.desc, one, one, idx, c.status, ws)]:
        with pytest.raises(cb.CBError, match="current one is 0"):
            bad()


# ---- all of it together -----------------------------------------------------------


def test_a_round_of_answers_in_a_graph(torch, cb):
    """Free, fork, extend, rotate, write, attend and thin, captured once and replayed on inputs that change, with eager
    work and synchronisation between: every replay as the same calls run eagerly on a second cache."""
    D, P, Hkv, G, kids = 64, 16, 2, 2, 3
    lens = [203, 0, 0, 0, 0]
    a, b = (cache_with(torch, cb, lens, H=Hkv, D=D, P=P, extra=40, width=15, seed=5) for _ in range(2))
    for c in (a, b):
        fill_cache(torch, cb, c, lens, 6)
    par, chi, one, thin = ints(torch, [0] * kids), ints(torch, [1, 2, 3]), ints(torch, [1] * kids), ints(torch, [4])
    src = ints(torch, [2])
    freq = torch.tensor(cb.cb_rotary_frequencies(D, 1e4)[0], dtype=torch.float64, device="cuda")
    k, v = (torch.empty((1, kids, Hkv, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.empty((1, kids, Hkv * G, 1, D), dtype=torch.bfloat16, device="cuda")
    idx = torch.empty((1, 1, 1, 50), dtype=torch.int32, device="cuda")
    pos = ints(torch, [203])

    def scratches(c):
        return [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (
            cb.cb_cache_fork_workspace_bytes(c.desc, kids), cb.cb_cache_compact_workspace_bytes(c.desc, 1))]

    def step(c, ws, kk, qq, out, lse, aw):
        cb.cb_cache_free(c.desc, chi)
        cb.cb_cache_fork(c.desc, par, chi, c.status, ws[0])
        cb.cb_cache_extend(c.desc, chi, one, c.status)
        cb.cb_rotary([cb.rows(q[0], qq[0], pos), cb.rows(k[0], kk[0], pos)], freq)
        cb.cb_cache_write(c.desc, kk, v, chi)
        cb.cb_cache_attend(c.desc, qq, out, aw, lse, chi)
        cb.cb_cache_compact(c.desc, src, thin, idx, c.status, ws[1])

    def fresh(i):
        for x, n in ((k, 0), (v, 1), (q, 2)):
            x.copy_(randn(torch, 100 + 10 * i + n, *x.shape))
        idx.copy_(torch.sort(torch.randperm(204, generator=torch.Generator().manual_seed(i))[:50])[0].reshape(1, 1, 1, 50))

    bufs = []
    for c in (a, b):
        qq = torch.empty_like(q)
        bufs.append((scratches(c), torch.empty_like(k), qq, torch.empty_like(q),
                     torch.empty(q.shape[:4], device="cuda"), scratch(torch, cb, c, q)))
    fresh(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, *bufs[0])
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, *bufs[0])
    step(b, *bufs[1])
    for i in range(4):
        fresh(i)
        bufs[0][3].zero_()
        g.replay()
        torch.cuda.synchronize()
        step(b, *bufs[1])
        assert a.status.item() == b.status.item() == 0
        for x, y in ((a.pool, b.pool), (a.refs, b.refs), (a.table, b.table), (a.lens, b.lens),
                     (bufs[0][3], bufs[1][3]), (bufs[0][4], bufs[1][4])):
            assert torch.equal(x, y)
        m = model(a, D, P)
        check_attend(torch, m, bufs[0][2], bufs[0][3], bufs[0][4], [1, 2, 3], [1] * kids, True, 0.0, 0, "bf16")
        assert m.lens.tolist() == [203, 204, 204, 204, 50]


def test_scratch_on_the_wrong_device_is_refused(torch, cb):
    c = cache_with(torch, cb, [20], D=64, P=16)
    one, ws = ints(torch, [0]), torch.empty(1 << 16, dtype=torch.uint8)
    with pytest.raises(cb.CBError):
        cb.cb_cache_fork(c.desc, one, one, c.status, ws)
    with pytest.raises(cb.CBError):
        cb.cb_cache_fork(c.desc, one, one, c.status, ws[::2].cuda()[::2])


def test_a_message_from_selection_to_answers(torch, cb, oracle):
    """The receiver's path: select and compact two senders' caches, move the kept keys, store them, fork two
    answers, append a token to each, attend, thin one answer, attend again."""
    L, Hq, Hkv, D, T, m, S, P = 2, 4, 2, 64, 512, 16, 2, 16
    lay = cb.layout(L, Hq, Hkv, D, m, T, senders=S)
    q = randn(torch, 1, L, Hq, m, D).bfloat16().cuda()
    k, v = randn(torch, 2, S, L, Hkv, T, D).bfloat16().cuda(), randn(torch, 3, S, L, Hkv, T, D).bfloat16().cuda()
    buf = cb.Buffers(lay, 0.25)
    cb.run_pipeline(q, k, v, buf)
    n, kept = buf.keep, S * buf.keep
    # move: row s * keep + j of (l, g) comes from idx[s][l][g][j] and goes to position s * keep + j
    freq, _ = cb.cb_rotary_frequencies(D, 1e6)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    new = torch.arange(kept, dtype=torch.int32, device="cuda").reshape(S, 1, n)
    x = buf.k_out.reshape(L * Hkv, S, n, D).transpose(0, 1)
    kk = buf.k_out.clone()
    cb.cb_rotary(cb.rows(x, x, new, buf.idx.reshape(S, L * Hkv, n)), fd)
    d = new.cpu().numpy().astype(np.int64) - buf.idx.reshape(S, L * Hkv, n).cpu().numpy()
    check_rotary(torch, x, kk.reshape(L * Hkv, S, n, D).transpose(0, 1), freq, d, 1.0, False, False, "bf16")
    # store
    c = cb.Cache(L, Hkv, D, P, 64, 4, 20)
    zero = ints(torch, [0])
    cb.cb_cache_extend(c.desc, zero, ints(torch, [kept]), c.status)
    cb.cb_cache_write(c.desc, buf.k_out.reshape(L, 1, Hkv, kept, D), buf.v_out.reshape(L, 1, Hkv, kept, D), zero)
    mm = model(c, D, P)
    for l, h in itertools.product(range(L), range(Hkv)):
        a, b, _ = mm.read(0, l, h)
        assert np.array_equal(a, ref.values(*ref.quantise(ref.to_f64(buf.k_out[l, h]))))
        assert np.array_equal(b, ref.values(*ref.quantise(ref.to_f64(buf.v_out[l, h]))))
    # two answers, a token each
    kids = ints(torch, [1, 2])
    ws = torch.empty(cb.cb_cache_fork_workspace_bytes(c.desc, 2), dtype=torch.uint8, device="cuda")
    cb.cb_cache_fork(c.desc, ints(torch, [0, 0]), kids, c.status, ws)
    cb.cb_cache_extend(c.desc, kids, ints(torch, [1, 1]), c.status)
    row = randn(torch, 4, L, 2, Hkv, 1, D).bfloat16().cuda()
    cb.cb_cache_write(c.desc, row, row, kids)
    aw = torch.empty(cb.cb_cache_attend_workspace_bytes(c.desc, L, 2, Hq, 1), dtype=torch.uint8, device="cuda")
    qq = randn(torch, 5, L, 2, Hq, 1, D).bfloat16().cuda()
    out, lse = torch.empty_like(qq), torch.empty(qq.shape[:4], device="cuda")
    cb.cb_cache_attend(c.desc, qq, out, aw, lse, kids)
    mm = model(c, D, P)
    assert int(mm.refs[mm.table[0, 0]]) == 3 and mm.lens.tolist() == [kept, kept + 1, kept + 1, 0]
    check_attend(torch, mm, qq, out, lse, [1, 2], [1, 1], True, 0.0, 0, "bf16")
    for s in (1, 2):   # the message below, each answer's own token on top
        a, _, _ = mm.read(s, 0, 0)
        assert np.array_equal(a[:kept], mm.read(0, 0, 0)[0])
        assert np.array_equal(a[kept], ref.values(*ref.quantise(ref.to_f64(row[0, s - 1, 0, 0]))))
    # the next reader thins answer 1 by a ranking of its keys
    ko = torch.empty((L, 1, Hkv, kept + 1, D), dtype=torch.bfloat16, device="cuda")
    vo = torch.empty_like(ko)
    cb.cb_cache_read(c.desc, ko, vo, ints(torch, [1]))
    lay2 = cb.layout(L, Hq, Hkv, D, m, kept + 1)
    buf2 = cb.Buffers(lay2, 0.5)
    cb.run_steps(q, ko.reshape(1, L, Hkv, kept + 1, D), vo, buf2)
    cw = torch.empty(cb.cb_cache_compact_workspace_bytes(c.desc, 1), dtype=torch.uint8, device="cuda")
    one = ints(torch, [1])
    cb.cb_cache_compact(c.desc, one, one, buf2.idx, c.status, cw)
    assert cb.cb_cache_status(c.status) == 0
    assert mm.compact([1], [1], lambda i, l, h: buf2.idx[0, l, h].cpu().numpy(), None) == 0
    same_state(c, mm)
    cb.cb_cache_attend(c.desc, qq, out, aw, lse, kids)
    check_attend(torch, mm, qq, out, lse, [1, 2], [1, 1], True, 0.0, 0, "bf16")
    cb.cb_cache_free(c.desc, ints(torch, [0, 1, 2]))
    assert not c.refs.any() and not c.lens.any() and (c.table == -1).all()
