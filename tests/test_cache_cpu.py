"""The receiver's side on a host without a GPU: header, exports, frequencies, and every
refusal that returns before any launch."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

import cache_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cacheback_cache.h")
FAKE = 1 << 20   # never dereferenced: every call below fails validation first
L = ctypes.byref


@pytest.fixture(scope="module")
def cb():
    import paper_2609_32046_amd as cb

    return cb


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(cb_[a-z_]+)\s*\(", text)))


def test_header_and_exports(cb):
    want = ["cb_rotary", "cb_rotary_frequencies", "cb_cache_page_bytes", "cb_cache_status",
            "cb_cache_extend", "cb_cache_free", "cb_cache_fork", "cb_cache_fork_workspace_bytes",
            "cb_cache_compact", "cb_cache_compact_workspace_bytes", "cb_cache_write",
            "cb_cache_read", "cb_cache_attend", "cb_cache_attend_workspace_bytes"]
    assert declared() == sorted(want)
    out = subprocess.run(["nm", "-D", "--defined-only", cb.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if line.strip()}
    for name in want:
        assert name in exported and hasattr(cb, name) and name in cb.__all__
    assert cb.cb_status_string(-9) != "unknown status"


def test_headers_compile_as_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "cacheback_cache.h"\nint main(void) { cb_cache c; cb_rows r; cb_rope p; '
                   'return (int)(sizeof c + sizeof r + sizeof p) == 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src),
                    "-o", str(tmp_path / "t.o")], check=True)


@pytest.mark.parametrize("R", [2, 16, 64, 70, 128])
def test_frequencies(cb, R):
    i = np.arange(R // 2)
    f = 1e6 ** (-2.0 * i / R) / (2 * math.pi)
    got, amp = cb.cb_rotary_frequencies(R, 1e6)
    assert np.allclose(got, f, rtol=1e-14, atol=0) and amp == 1.0
    got, amp = cb.cb_rotary_frequencies(R, 1e6, "linear", 4.0)
    assert np.allclose(got, f / 4, rtol=1e-14, atol=0) and amp == 1.0
    got, amp = cb.cb_rotary_frequencies(R, 1e6, "yarn", 4.0, 32768)
    got = np.array(got)
    assert amp == pytest.approx(0.1 * math.log(4.0) + 1.0, rel=1e-15)
    assert (got <= f * (1 + 1e-14)).all() and (got >= f / 4 * (1 - 1e-14)).all()
    # by the definition: pairs of 32 turns in the original length stay, of one turn and fewer slow down
    turns = f * 32768
    lo, hi = (R * math.log(32768 / (t * 2 * math.pi)) / (2 * math.log(1e6)) for t in (32.0, 1.0))
    assert np.allclose(got[i <= math.floor(lo)], f[i <= math.floor(lo)], rtol=1e-13, atol=0)
    slow = i >= math.ceil(hi)
    assert np.allclose(got[slow], f[slow] / 4, rtol=1e-13, atol=0)
    assert (np.diff(got) <= 0).all() and (turns[slow] <= 1.0 + 1e-9).all()


def test_frequencies_refuse(cb):
    for kw in [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=1026), dict(base=1.0),
               dict(base=math.inf), dict(scaling="linear", factor=0.5),
               dict(scaling="yarn", factor=4.0), dict(scaling="yarn", factor=math.nan, original_len=9),
               dict(scaling="yarn", factor=4.0, original_len=9, fast_turns=1, slow_turns=2),
               dict(scaling="yarn", factor=4.0, original_len=9, slow_turns=-1), dict(scaling="other")]:
        with pytest.raises(cb.CBError) as e:
            cb.cb_rotary_frequencies(**{"rotary_dim": 64, **kw})
        assert e.value.status == -2, kw


def rows(cb, **kw):
    r = cb.cb_rows(x=FAKE, out=FAKE, pos=FAKE, size=(ctypes.c_int64 * 3)(2, 3, 4))
    for name in ("in_stride", "out_stride"):
        setattr(r, name, (ctypes.c_int64 * 3)(12 * 64, 4 * 64, 64))
    for name in ("pos_stride", "from_stride"):
        setattr(r, name, (ctypes.c_int64 * 3)(12, 4, 1))
    for k, v in kw.items():
        setattr(r, k, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return r


def test_rotary_refuses(cb):
    def call(r, parts=1, D=64, freq=FAKE, R=64, amp=1.0, dtype=1):
        return cb._lib.cb_rotary(L(r) if r is not None else None, parts, D, freq, R, amp, 0, 0, dtype,
                                 None)

    ok = rows(cb)
    assert call(None) == -1 and call(ok, freq=None) == -1
    assert call(ok, parts=0) == -2 and call(ok, parts=3) == -2
    assert call(ok, dtype=2) == -3
    for D in (0, 4, 60, 1032):
        assert call(ok, D=D, R=2) == -2
    for R in (0, 1, 63, 66, -2):
        assert call(ok, R=R) == -2
    assert call(ok, amp=math.nan) == -2 and call(ok, amp=1e300) == -2
    assert call(ok, freq=FAKE + 4) == -6
    for bad in (dict(x=None), dict(out=None), dict(pos=None)):
        assert call(rows(cb, **bad)) == -1
    for bad in (dict(x=FAKE + 8), dict(out=FAKE + 2), dict(pos=FAKE + 2), dict(frm=FAKE + 1),
                dict(in_stride=(768, 256, 60)), dict(out_stride=(768, 252, 64))):
        assert call(rows(cb, **bad)) == -6, bad
    for bad in (dict(size=(-1, 3, 4)), dict(size=(2**31, 3, 4)), dict(size=(2**30, 2**20, 4)),
                dict(out_stride=(768, 0, 64))):
        assert call(rows(cb, **bad)) == -2, bad


def desc(cb, **kw):
    f = dict(layers=2, kv_heads=2, head_dim=64, page_len=16, pages=8, seqs=3, width=4, reserved=0,
             pool=FAKE, refs=FAKE, table=FAKE, lens=FAKE)
    f.update(kw)
    return cb.cb_cache(**f)


BAD_SIZES = [dict(layers=0), dict(kv_heads=0), dict(head_dim=96), dict(head_dim=256), dict(page_len=8),
             dict(page_len=48), dict(page_len=512), dict(pages=0), dict(pages=2**24 + 1), dict(seqs=0),
             dict(seqs=2**17 + 1), dict(width=0), dict(width=2**27), dict(layers=5000)]


def calls(cb):
    """Every call on a cache with arguments that are fine: name -> f(descriptor, **changes)."""
    lib = cb._lib
    s4 = (ctypes.c_int64 * 4)(4096, 2048, 1024, 64)
    s3 = (ctypes.c_int64 * 3)(8, 4, 2)

    def extend(c, seqs=FAKE, add=FAKE, n=2, status=FAKE):
        return lib.cb_cache_extend(c, seqs, add, n, status, None)

    def free(c, seqs=FAKE, n=2):
        return lib.cb_cache_free(c, seqs, n, None)

    def fork(c, parents=FAKE, children=FAKE, n=2, status=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return lib.cb_cache_fork(c, parents, children, n, 0, status, ws, ws_bytes, None)

    def compact(c, src=FAKE, dst=FAKE, n=2, idx=FAKE, stride=s3, keep=8, counts=None, status=FAKE,
                ws=FAKE, ws_bytes=1 << 30):
        return lib.cb_cache_compact(c, src, dst, n, idx, stride, keep, counts, status, ws, ws_bytes,
                                    None)

    def moved(fn):
        def f(c, layer=0, layers=2, seqs=None, n=2, start=None, counts=None, most=4, k=FAKE, v=FAKE,
              stride=s4, dtype=1):
            return fn(c, layer, layers, seqs, n, start, counts, most, k, v, stride, dtype, None)
        return f

    def attend(c, layer=0, layers=2, seqs=None, n=2, q=FAKE, qs=s4, heads=4, q_lens=None, m=4,
               longest=0, scale=0.0, out=FAKE, os_=s4, lse=None, dtype=1, ws=FAKE, ws_bytes=1 << 40):
        return lib.cb_cache_attend(c, layer, layers, seqs, n, q, qs, heads, q_lens, m, 1, longest, scale, out,
                                   os_, lse, dtype, ws, ws_bytes, None)

    return {"extend": extend, "free": free, "fork": fork, "compact": compact,
            "write": moved(lib.cb_cache_write), "read": moved(lib.cb_cache_read), "attend": attend}


@pytest.mark.parametrize("name", ["extend", "free", "fork", "compact", "write", "read", "attend"])
def test_cache_calls_refuse_bad_caches(cb, name):
    f = calls(cb)[name]
    assert f(None) == -1
    for bad in BAD_SIZES:
        assert f(L(desc(cb, **bad))) == -2, bad
        assert cb._lib.cb_cache_page_bytes(L(desc(cb, **bad))) == 0
    for p in ("pool", "refs", "table", "lens"):
        assert f(L(desc(cb, **{p: None}))) == -1
        assert f(L(desc(cb, **{p: FAKE + 8}))) == -6


def test_cache_calls_refuse_bad_arguments(cb):
    f, c = calls(cb), L(desc(cb))
    wrong4 = (ctypes.c_int64 * 4)(4096, 2048, 1020, 64)
    zero4 = (ctypes.c_int64 * 4)(4096, 2048, 0, 64)
    for name, bad, code in [
            ("extend", dict(seqs=None), -1), ("extend", dict(add=None), -1), ("extend", dict(status=None), -1),
            ("extend", dict(n=-1), -2), ("extend", dict(n=2049), -2), ("extend", dict(add=FAKE + 2), -6),
            ("free", dict(seqs=None), -1), ("free", dict(n=-1), -2), ("free", dict(seqs=FAKE + 1), -6),
            ("fork", dict(parents=None), -1), ("fork", dict(children=None), -1), ("fork", dict(status=None), -1),
            ("fork", dict(n=2049), -2), ("fork", dict(ws=None), -5), ("fork", dict(ws_bytes=16 + 2 * 4 * 8 - 1), -5),
            ("fork", dict(ws=FAKE + 8), -6), ("fork", dict(status=FAKE + 2), -6),
            ("compact", dict(src=None), -1), ("compact", dict(dst=None), -1), ("compact", dict(idx=None), -1),
            ("compact", dict(stride=None), -1), ("compact", dict(keep=0), -2), ("compact", dict(keep=65), -2),
            ("compact", dict(n=-1), -2), ("compact", dict(ws=None), -5), ("compact", dict(ws_bytes=2 * 5 * 4 - 1), -5),
            ("compact", dict(counts=FAKE + 2), -6), ("compact", dict(idx=FAKE + 2), -6)]:
        assert f[name](c, **bad) == code, (name, bad)
    for name in ("write", "read"):
        for bad, code in [(dict(layer=-1), -2), (dict(layer=1), -2), (dict(layers=3), -2), (dict(layers=-1), -2),
                          (dict(n=-1), -2), (dict(n=4), -2), (dict(most=-1), -2), (dict(most=2**31), -2),
                          (dict(k=None), -1), (dict(v=None), -1), (dict(stride=None), -1), (dict(dtype=2), -3),
                          (dict(k=FAKE + 8), -6), (dict(v=FAKE + 4), -6), (dict(stride=wrong4), -6),
                          (dict(start=FAKE + 2), -6), (dict(counts=FAKE + 1), -6), (dict(seqs=FAKE + 3), -6)]:
            assert f[name](c, **bad) == code, (name, bad)
    assert f["read"](c, stride=zero4) == -2
    for bad, code in [(dict(layer=-1), -2), (dict(layers=3), -2), (dict(n=-1), -2), (dict(n=4), -2),
                      (dict(heads=3), -2), (dict(heads=0), -2), (dict(m=-1), -2), (dict(m=2**27), -2), (dict(longest=-1), -2),
                      (dict(scale=-1.0), -2), (dict(scale=math.nan), -2), (dict(scale=math.inf), -2),
                      (dict(q=None), -1), (dict(out=None), -1), (dict(qs=None), -1), (dict(os_=None), -1),
                      (dict(dtype=7), -3), (dict(q=FAKE + 8), -6), (dict(out=FAKE + 8), -6),
                      (dict(lse=FAKE + 2), -6), (dict(qs=wrong4), -6), (dict(os_=wrong4), -6),
                      (dict(os_=zero4), -2), (dict(q_lens=FAKE + 2), -6)]:
        assert f["attend"](c, **bad) == code, bad
    big = L(desc(cb, width=65))   # long enough to be cut into chunks
    need = cb._lib.cb_cache_attend_workspace_bytes(big, 2, 2, 4, 4, 0)
    assert need > 0
    assert f["attend"](big, ws=None, ws_bytes=0) == -5 and f["attend"](big, dtype=0, ws_bytes=15) == -5
    assert f["attend"](big, ws=FAKE + 8) == -6


def test_calls_refuse_sizes_past_a_launch(cb):
    """A grid holds 2^32 - 1 threads along an axis; a scale that fp32 holds, but not times log2(e)."""
    f, c = calls(cb), L(desc(cb))
    for name in ("write", "read"):                       # 8 units of 8 threads a row
        assert f[name](c, most=(2**32 - 256) // 64 + 1) == -2
    assert f["free"](c, n=2**24) == -2
    for size in ((1, 1, 2**29), (2**10, 2**10, 2**30)):
        assert cb._lib.cb_rotary(L(rows(cb, size=size)), 1, 64, FAKE, 64, 1.0, 0, 0, 1, None) == -2
    long = L(desc(cb, width=4096))
    assert f["attend"](long, seqs=FAKE, n=2**20, m=64) == -2   # 2^26 workgroups of the join
    many = L(desc(cb, layers=4096, kv_heads=4096))
    assert f["attend"](many, layers=4096, heads=4096, seqs=FAKE, n=2**20) == -2
    need = cb._lib.cb_cache_attend_workspace_bytes
    assert need(many, 4096, 2**20, 4096, 2**26, 0) == need(long, 2, 2**20, 4, 64, 0) == 0
    assert f["attend"](c, scale=3e38) == -2
    far = L(desc(cb, width=2**27 - 4096))                      # 2^24 rounds of 128 positions
    assert f["attend"](far, seqs=FAKE, n=200, m=1) == -2 and need(far, 2, 200, 4, 1, 0) == 0
    assert need(far, 2, 200, 4, 1, 2**20) > 0


def test_status_refuses(cb):
    assert cb._lib.cb_cache_status(None, None) == -1
    assert cb._lib.cb_cache_status(FAKE + 2, None) == -6


def test_sizes(cb):
    assert cb._lib.cb_cache_page_bytes(L(desc(cb))) == 2 * 2 * 16 * 68
    assert cb._lib.cb_cache_page_bytes(L(desc(cb, head_dim=128, page_len=64))) == 2 * 2 * 64 * 136
    for fn in (cb._lib.cb_cache_fork_workspace_bytes, cb._lib.cb_cache_compact_workspace_bytes):
        assert fn(L(desc(cb)), 3) > 0 and fn(L(desc(cb)), -1) == 0 and fn(L(desc(cb)), 2049) == 0
        assert fn(L(desc(cb, width=0)), 3) == 0
    n = cb._lib.cb_cache_attend_workspace_bytes
    assert n(L(desc(cb)), 1, 1, 4, 1, 0) == 0                     # 64 positions: no split
    assert n(L(desc(cb, width=64)), 1, 3, 4, 1, 0) == 0           # 1024 neither
    assert n(L(desc(cb, width=65)), 1, 3, 4, 1, 0) > 0
    assert n(L(desc(cb, width=4096)), 1, 1, 4, 1, 0) > 0
    assert n(L(desc(cb, width=4096)), 1, 1, 4, 1, 1024) == 0     # told that none is longer
    assert n(L(desc(cb, width=4096)), 1, 1, 4, 1, -1) == 0       # refused by the call
    assert n(L(desc(cb, width=4096)), 1, 1, 3, 1, 0) == 0         # refused by the call


# ---- the reference itself -----------------------------------------------------


def test_reference_quantiser_by_hand():
    x = np.zeros((3, 32))
    x[0, :8] = [7.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25]      # scale 1: every tie to the even code
    x[1, :3] = [7.0000001, -14.0, 0.5]                           # scale 2
    code, scale = ref.quantise(x)
    assert scale.ravel().tolist() == [127, 128, 3]
    assert code[0, :8].tolist() == [7, 6, 6, 4, 4, 2, 2, 0]
    assert code[1, :3].tolist() == [6, 15, 0]   # 3.5 to 4, -7 to -6, 0.25 to 0
    v = ref.values(code, scale)
    assert v[0, :8].tolist() == [6, 4, 4, 2, 2, 1, 1, 0] and v[1, :3].tolist() == [8, -12, 0]
    rng = np.random.default_rng(0)
    y = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-30, 30, (200, 1)))
    code, scale = ref.quantise(y)
    step = 2.0 ** (scale.astype(float) - 127)
    err = np.abs(ref.values(code, scale) - y).reshape(200, 2, 32).max(-1)
    assert (err <= step).all()                                   # half a step of the largest levels
    assert (np.abs(y).reshape(200, 2, 32).max(-1) > 3.5 * step).all()   # and no larger scale than needed


@pytest.mark.parametrize("D,P", [(64, 16), (128, 32)])
def test_reference_layout_round_trip(D, P):
    rng = np.random.default_rng(1)
    unit = rng.integers(0, 256, P * (D + D // 16)).astype(np.uint8)
    assert np.array_equal(ref.pack(*ref.unpack(unit, P, D)), unit)
