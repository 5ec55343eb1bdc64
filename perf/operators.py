"""The receiver's side of a message, as measured cases.

What the receiver does with the rows that a sender kept: it moves their keys to
new positions, holds them in pages of a cache of four bits a value, lets several
answers share those pages, thins them again, and attends to them.

  rope    cb_rotary: the query and key rows of a step, or kept keys moved from
          their old positions to new ones
  attend  cb_cache_attend: attention of query rows over the pages of a batch of
          sequences
  store   cb_cache_write and cb_cache_read: rows into the cache's four bits,
          and the values they stand for back, as the next ranking reads them
  fork    cb_cache_free, cb_cache_fork and cb_cache_extend: earlier answers give
          their pages back, new ones share (or copy) a message and take room
          for their next position
  thin    cb_cache_compact: new pages with the selected positions of a sequence

Sizes are those of this repository's workloads and of its tests' ranges: 1 to 48
layers, 1 to 8 query heads per KV head, head width 64 or 128, 1 to 512 query
tokens, 1 to 131072 positions, 1 to 64 sequences, pages of 16 to 128 positions.

The cache: ``pool`` [pages][layers][kv_heads][unit] bytes.  A unit holds, for
its P positions and D values a row, the key codes [P][D/2], the value codes
[P/4][16][4][D/32], the key scales [P][D/32] and the value scales
[P/4][D/32][4].  A code is a sign and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or
6, the even value of a pair in the low half of its byte; a scale byte b stands
for 2^(b - 127) and covers 32 values of one row.  ``refs`` [pages] counts the
holders of a page, ``table`` [seqs][width] lists the pages of a sequence (-1
behind the last) and ``lens`` [seqs] its positions.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
BLOCK = 32


def _rope(name, L, n, Hq, Hkv, T, D, R, interleaved, dtype, scaling, far, transpose=False,
          move=False):
    return {"name": name, "kind": "rope", "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "T": T, "D": D,
            "R": R, "interleaved": interleaved, "dtype": dtype, "scaling": scaling, "far": far,
            "transpose": transpose, "move": move}


def _attend(name, L, n, Hq, Hkv, D, T, m, P, dtype="bf16", causal=True, ragged=True):
    return {"name": name, "kind": "attend", "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T,
            "m": m, "P": P, "dtype": dtype, "causal": causal, "ragged": ragged}


def _store(name, L, n, Hkv, D, T, new, P, dtype="bf16"):
    return {"name": name, "kind": "store", "L": L, "n": n, "Hkv": Hkv, "D": D, "T": T, "new": new,
            "P": P, "dtype": dtype}


def _fork(name, L, parents, each, Hkv, D, T, P, copy):
    return {"name": name, "kind": "fork", "L": L, "parents": parents, "each": each, "Hkv": Hkv,
            "D": D, "T": T, "P": P, "copy": copy}


def _thin(name, L, n, Hkv, D, T, keep, P, shared):
    return {"name": name, "kind": "thin", "L": L, "n": n, "Hkv": Hkv, "D": D, "T": T,
            "keep": keep, "P": P, "shared": shared}


def listed():
    return [
        # One decoding step's queries and keys of 16 answers, fp32, adjacent
        # pairs in half of the head: latency.
        _rope("rope-step", 1, 16, 32, 8, 1, 128, 64, True, "f32", "linear", 32768),
        # The message of the 8B shape takes its place at the receiver: 2048 kept
        # keys of every layer and head, each from its own old position.
        _rope("rope-move", 36, 1, 0, 8, 2048, 128, 128, False, "bf16", "yarn", 8192, move=True),
        # The smallest configuration's query (16 tokens, fp32) over 512
        # positions: latency.
        _attend("attend-tiny", 1, 1, 4, 2, 64, 512, 16, 16, "f32", causal=False, ragged=False),
        # One answer decoding over a very long context: few rows, a long axis.
        _attend("attend-long", 1, 1, 32, 8, 128, 131072, 1, 64, ragged=False),
        # 64 answers decoding together, lengths up to 16384 as they come.
        _attend("attend-batch", 1, 64, 32, 8, 128, 16384, 1, 64),
        # A prompt's part of 500 tokens behind 32768 positions, five query heads
        # per KV head.
        _attend("attend-prompt", 1, 1, 40, 8, 128, 32768, 500, 128),
        # One new token of 32 answers, all layers of a narrow-headed model.
        _store("store-step", 24, 32, 8, 64, 2048, 1, 16),
        # A message of 2048 positions of the 8B shape.
        _store("store-message", 36, 1, 8, 128, 4096, 2048, 64),
        # 16 answers to each of four messages of odd length: shared pages.
        _fork("fork-share", 36, 4, 16, 8, 128, 2001, 64, False),
        # A message copied for a receiver that will change it.
        _fork("fork-copy", 36, 1, 2, 8, 128, 8192, 64, True),
        # A chain's next reader ranks 900 positions and keeps a third of them:
        # one list of positions for all layers of a small model.
        _thin("thin-chain", 8, 1, 8, 64, 900, 300, 16, True),
        # Three messages thinned to a quarter, each layer and head by its own
        # list.
        _thin("thin-units", 36, 3, 8, 128, 8192, 2048, 64, False),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rope", "attend", "attend", "attend", "store", "fork", "thin"])
    D = rng.choice([64, 128, 128])
    P = rng.choice([16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    L = log_int(1, 48)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rope":
        move = rng.random() < 0.4
        T = log_int(1, 8192)
        Hq = 0 if move else Hkv * rng.choice([1, 2, 4, 5, 8])
        c = _rope("", L if move else 1, log_int(1, 64), Hq, Hkv, T, D,
                  rng.choice([D, D, D // 2, D // 4, D // 2 + 6]), rng.random() < 0.5, dtype,
                  rng.choice(["none", "linear", "yarn"]), log_int(T, 2**20),
                  rng.random() < 0.3, move)
    elif kind == "attend":
        m = rng.choice([1, 1, log_int(1, 16), log_int(1, 512)])
        c = _attend("", rng.choice([1, 1, 1, 2, 3]), log_int(1, 64),
                    Hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), Hkv, D, log_int(1, 131072), m, P,
                    dtype, rng.random() < 0.8, rng.random() < 0.8)
    elif kind == "store":
        T = log_int(1, 16384)
        c = _store("", L, log_int(1, 64), Hkv, D, T, rng.choice([1, log_int(1, T)]), P, dtype)
    elif kind == "fork":
        c = _fork("", L, log_int(1, 8), log_int(1, 16), Hkv, D, log_int(1, 16384), P,
                  rng.random() < 0.3)
    else:
        T = log_int(1, 16384)
        c = _thin("", L, log_int(1, 8), Hkv, D, T, log_int(1, T), P, rng.random() < 0.5)
    del c["name"]
    # no dearer than the dearest listed case of its kind, and a pool of at most 1.4 GB
    most = max(_cost(x) for x in listed() if x["kind"] == kind)
    while _cost(c) > most or _pool_bytes(c) > 1.4e9:
        if c["L"] > 1:
            c["L"] = (c["L"] + 1) // 2
        elif c.get("n", 1) > 1:
            c["n"] = (c["n"] + 1) // 2
        elif c.get("each", 1) > 1:
            c["each"] = (c["each"] + 1) // 2
        else:
            c["T"] = (c["T"] + 1) // 2
            for k in ("new", "keep"):
                if k in c:
                    c[k] = min(c[k], c["T"])
    return c


# ---------------------------------------------------------------------------
# sizes


def _unit(c):
    return c["P"] * (c["D"] + c["D"] // 16)


def _page(c):
    return c["L"] * c["Hkv"] * _unit(c)


def _pages_of(positions, c):
    return -(-positions // c["P"])


def _sizes(c):
    """(rows of the table, entries a row, pages): room for every sequence, and an
    eighth more pages."""
    if c["kind"] == "fork":
        seqs, held = c["parents"] * (1 + c["each"]), c["parents"] * _pages_of(c["T"], c)
        held += c["parents"] * c["each"] * (_pages_of(c["T"] + 1, c) if c["copy"] else 2)
        width = _pages_of(c["T"] + 1, c)
    elif c["kind"] == "thin":
        seqs, width = 2 * c["n"], _pages_of(c["T"], c)
        held = c["n"] * (width + _pages_of(c["keep"], c))
    else:
        seqs, width = c["n"], _pages_of(c["T"], c)
        held = seqs * width
    return seqs, width, held + held // 8 + 1


def _pool_bytes(c):
    return 0 if c["kind"] == "rope" else _sizes(c)[2] * _page(c)


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lens(c, seed):
    """Lengths of the sequences: the first has T positions; ragged ones go down
    to none."""
    n, T = c["n"], c["T"]
    if not c.get("ragged", c["kind"] == "store"):
        return [T] * n
    gen = torch.Generator()
    gen.manual_seed(1000 + n)   # the work of a case does not hang on the seed
    low = c.get("new", 0)
    rest = torch.rand(n, generator=gen) * (T + 1 - low)
    return [T] + [min(T, low + int(x)) for x in rest[1:]]


def work(case):
    c = case
    es = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "rope":
        rows = (c["Hq"] + c["Hkv"]) * c["L"] * c["n"] * c["T"]
        pos = c["n"] * c["T"] * 4
        if c["move"]:
            pos += rows * 4
        return {"bytes": 2 * rows * c["D"] * es + pos, "flops": 3 * rows * c["R"]}
    row = c["D"] + c["D"] // 16   # key and value of one position and head
    if c["kind"] == "attend":
        lens = _lens(c, 0)
        rows = c["L"] * c["n"] * c["Hq"] * c["m"]
        pairs = 0
        for T in lens:
            if c["causal"]:   # the last m positions are the query tokens' own
                seen = sum(max(0, T - c["m"] + r + 1) for r in range(c["m"]))
            else:
                seen = T * c["m"]
            pairs += seen * c["L"] * c["Hq"]
        return {"bytes": c["L"] * c["Hkv"] * sum(lens) * row + rows * (2 * c["D"] * es + 4),
                "flops": 4 * pairs * c["D"]}
    U = c["L"] * c["Hkv"]
    if c["kind"] == "store":
        rows = U * c["n"] * c["new"]
        # written once, read again: the caller's rows in and out, the four bits in and out
        return {"bytes": rows * (2 * 2 * c["D"] * es + 2 * row), "flops": 0}
    if c["kind"] == "fork":
        kids = c["parents"] * c["each"]
        pages = _pages_of(c["T"], c)
        copied = pages if c["copy"] else int(c["T"] % c["P"] != 0)
        return {"bytes": kids * (2 * copied * _page(c) + 3 * 4 * pages) + 4 * _sizes(c)[2],
                "flops": 0}
    lists = 1 if c["shared"] else U
    return {"bytes": c["n"] * c["keep"] * (2 * U * row + 4 * lists) + 4 * _sizes(c)[2], "flops": 0}


# ---------------------------------------------------------------------------
# four bits in the plain form


_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _quantise(x):
    """Codes [..., D] and scale bytes [..., D/32] of rows x [..., D]."""
    y = x.float().unflatten(-1, (-1, BLOCK))
    bits = y.abs().amax(-1).view(torch.int32)     # 1.f * 2^(b - 127): exponent, then fraction
    e = (bits >> 23) - 129 + ((bits & 0x7FFFFF) > 0x600000).int()   # least with amax <= 7 * 2^e
    e = e.clamp(-124, 125)
    z = (y.double() * torch.exp2((-e).double()).unsqueeze(-1)).abs()
    code = ((z > 0.25).to(torch.uint8) + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5)
            + (z >= 3.5) + (z > 5.0))
    code = code + 8 * torch.signbit(y).to(torch.uint8)
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _values(code, scale):
    """What codes [..., D] and scale bytes [..., D/32] stand for, in 32 bits."""
    lut = torch.tensor(_LEVELS + [-x for x in _LEVELS], device=code.device)
    s = torch.exp2(scale.float() - 127.0)
    return (lut[code.int()].unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _pairs(code):
    """Bytes [..., D/2] of codes [..., D]."""
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpairs(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _pack(k, v):
    """Units [..., unit] of keys and values [..., P, D]."""
    kc, ks = _quantise(k)
    vc, vs = _quantise(v)
    kb, vb = _pairs(kc), _pairs(vc)
    lead, P, D = k.shape[:-2], k.shape[-2], k.shape[-1]
    vb = vb.reshape(*lead, P // 4, 4, 16, D // 32).transpose(-3, -2)
    vs = vs.reshape(*lead, P // 4, 4, D // 32).transpose(-2, -1)
    return torch.cat([x.reshape(*lead, -1) for x in (kb, vb, ks, vs)], -1)


def _fields(units, P, D):
    """Key bytes [..., P, D/2], value bytes alike, key scales [..., P, D/32],
    value scales alike, of units [..., unit]: views in order of positions."""
    lead, n, s = units.shape[:-1], P * D // 2, P * D // 32
    kb = units[..., :n].unflatten(-1, (P, D // 2))
    vb = units[..., n:2 * n].unflatten(-1, (P // 4, 16, 4, D // 32)).transpose(-3, -2)
    ks = units[..., 2 * n:2 * n + s].unflatten(-1, (P, D // 32))
    vs = units[..., 2 * n + s:].unflatten(-1, (P // 4, D // 32, 4)).transpose(-2, -1)
    return (kb, vb.reshape(*lead, P, D // 2), ks, vs.reshape(*lead, P, D // 32))


def _unpack(units, P, D):
    """Keys and values [..., P, D] in 32 bits of units [..., unit]."""
    kb, vb, ks, vs = _fields(units, P, D)
    return _values(_unpairs(kb), ks), _values(_unpairs(vb), vs)


# ---------------------------------------------------------------------------
# inputs


def _frequencies(R, scaling):
    """Turns per position of each pair, and the amplitude: base 1e6, for four
    times the 32768 positions of the original length."""
    i = torch.arange(R // 2, dtype=torch.float64)
    f = 1e6 ** (-2.0 * i / R) / (2.0 * math.pi)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "yarn":
        # whole turns within the original length: 32 and more stay, one and
        # fewer slow down by the factor, the pairs between go from one to the other
        def pair(turns):
            return R * math.log(32768.0 / (turns * 2.0 * math.pi)) / (2.0 * math.log(1e6))

        lo = max(math.floor(pair(32.0)), 0)
        hi = min(math.ceil(pair(1.0)), R - 1)
        keep = 1.0 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        return f / 4.0 * (1.0 - keep) + f * keep, 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _rope_inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    parts = [torch.randn((c["L"] * c["n"], h, c["T"], c["D"]), generator=gen, device=DEV)
             .to(_dtype(c)) for h in (c["Hq"], c["Hkv"]) if h]
    n, T, far = c["n"], c["T"], c["far"]
    if c["move"]:
        # kept positions of a cache of `far`, per row of heads; new ones in order
        rows = c["L"] * n * c["Hkv"]
        frm = torch.sort(torch.randint(0, far, (rows, T), generator=gen, device=DEV), 1)[0]
        frm = frm.to(torch.int32).reshape(c["L"] * n, c["Hkv"], T)
        pos = torch.arange(T, dtype=torch.int32, device=DEV).reshape(1, 1, T)
        return parts, pos, frm
    first = torch.randint(0, max(1, far - T + 1), (n, 1, 1), generator=gen, device=DEV)
    pos = (first + torch.arange(T, device=DEV)).to(torch.int32)
    return parts, pos, None


def _fill(c, gen, pool):
    """Random keys (channels of unlike size) and values in every page."""
    L, H, P, D = c["L"], c["Hkv"], c["P"], c["D"]
    size = torch.rand((L, H, 1, D), generator=gen, device=DEV) * 1.5 + 0.5
    step = max(1, (1 << 27) // (L * H * P * D))
    for part in pool.split(step):
        shape = (part.shape[0], L, H, P, D)
        k = torch.randn(shape, generator=gen, device=DEV) * size
        part.copy_(_pack(k, torch.randn(shape, generator=gen, device=DEV)))


def _random_bytes(c, gen, pool):
    """Pages whose contents are only moved: random codes, scales near one."""
    P, D = c["P"], c["D"]
    pool.random_(0, 256, generator=gen)
    pool[..., P * D:] = (pool[..., P * D:] & 3) + 124


def _cache(c, seed, lens, fill):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed + 77)
    seqs, width, pages = _sizes(c)
    pool = torch.empty((pages, c["L"], c["Hkv"], _unit(c)), dtype=torch.uint8, device=DEV)
    fill(c, gen, pool)
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device=DEV)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(lens):
        k = _pages_of(n, c)
        table[b, :k] = order[at:at + k]
        at += k
    refs[order[:at].long()] = 1
    full = torch.zeros(seqs, dtype=torch.int32)
    full[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    return {"pool": pool, "refs": refs, "table": table, "lens": full.to(DEV)}


def _queries(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed + 5)
    return torch.randn((c["L"], c["n"], c["Hq"], c["m"], c["D"]), generator=gen,
                       device=DEV).to(_dtype(c))


def _new_rows(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed + 9)
    shape = (c["L"], c["n"], c["Hkv"], c["new"], c["D"])
    k = torch.randn(shape, generator=gen, device=DEV)
    k *= torch.rand((c["L"], 1, c["Hkv"], 1, c["D"]), generator=gen, device=DEV) * 1.5 + 0.5
    v = torch.randn(shape, generator=gen, device=DEV)
    return k.to(_dtype(c)), v.to(_dtype(c))


def _lists(c, seed):
    """Ascending positions [n][L or 1][Hkv or 1][keep], drawn without repeats."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed + 13)
    shape = (c["n"], 1, 1) if c["shared"] else (c["n"], c["L"], c["Hkv"])
    x = torch.rand((*shape, c["T"]), generator=gen, device=DEV)
    return torch.sort(x.topk(c["keep"], dim=-1)[1], dim=-1)[0].to(torch.int32)


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c = dict(case)
    st = {"c": c}
    if c["kind"] == "rope":
        st["parts"], st["pos"], st["from"] = _rope_inputs(c, seed)
        f, st["amplitude"] = _frequencies(c["R"], c["scaling"])
        if c["move"]:
            st["amplitude"] = 1.0   # the kept keys have it already
        st["freq"] = f.to(DEV)
        st["out"] = [torch.empty_like(x) for x in st["parts"]]
        return st
    if c["kind"] == "attend":
        st.update(_cache(c, seed, _lens(c, seed), _fill))
        st["q"] = _queries(c, seed)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:-1], dtype=torch.float32, device=DEV)
    elif c["kind"] == "store":
        lens = _lens(c, seed)
        st.update(_cache(c, seed, lens, _random_bytes))
        st["k"], st["v"] = _new_rows(c, seed)
        st["k_out"], st["v_out"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
        st["start"] = _ints(*[x - c["new"] for x in lens])
    elif c["kind"] == "fork":
        st.update(_cache(c, seed, [c["T"]] * c["parents"], _random_bytes))
        kids = c["parents"] * c["each"]
        st["parents"] = _ints(*range(c["parents"])).repeat_interleave(c["each"]).contiguous()
        st["children"] = _ints(*range(c["parents"], c["parents"] + kids))
        st["add"] = torch.ones(kids, dtype=torch.int32, device=DEV)
    else:
        st.update(_cache(c, seed, [c["T"]] * c["n"], _random_bytes))
        st["src"], st["dst"] = _ints(*range(c["n"])), _ints(*range(c["n"], 2 * c["n"]))
        st["idx"] = _lists(c, seed)
    st["status"] = torch.empty(1, dtype=torch.int32, device=DEV)
    return st


# ---------------------------------------------------------------------------
# the plain forms


def _plain_rope(st):
    c = st["c"]
    R, sign = c["R"], -1.0 if c["transpose"] else 1.0
    outs = []
    for x in st["parts"]:
        pos = st["pos"] if c["move"] else st["pos"].repeat(c["L"], 1, 1)
        delta = pos.double() - (st["from"].double() if c["move"] else 0.0)
        turn = delta.unsqueeze(-1) * st["freq"]
        angle = 2.0 * math.pi * (turn - torch.floor(turn))
        cos = (torch.cos(angle) * st["amplitude"]).float()
        sin = (torch.sin(angle) * (st["amplitude"] * sign)).float()
        y = x.float().clone()
        if c["interleaved"]:
            a, b = x[..., 0:R:2].float(), x[..., 1:R:2].float()
            y[..., 0:R:2] = a * cos - b * sin
            y[..., 1:R:2] = b * cos + a * sin
        else:
            a, b = x[..., :R // 2].float(), x[..., R // 2:R].float()
            y[..., :R // 2] = a * cos - b * sin
            y[..., R // 2:R] = b * cos + a * sin
        outs.append(y.to(x.dtype))
    return outs


def _plain_attend(st):
    c = st["c"]
    L, n, Hq, Hkv, m, D, P = (c[x] for x in ("L", "n", "Hq", "Hkv", "m", "D", "P"))
    units = st["pool"][st["table"].clamp(min=0).long()]            # [n][width][L][H][unit]
    k, v = _unpack(units, P, D)                                    # [n][width][L][H][P][D]
    k, v = (x.permute(2, 0, 3, 1, 4, 5).flatten(3, 4) for x in (k, v))   # [L][n][H][T][D]
    T = k.shape[3]
    t = torch.arange(T, device=DEV)
    lens = st["lens"][:n].reshape(n, 1, 1, 1)
    limit = lens.expand(n, 1, m, 1)
    if c["causal"]:
        limit = lens - m + torch.arange(m, device=DEV).reshape(m, 1) + 1
    seen = (t < limit).repeat(1, 1, Hq // Hkv, 1)                  # [n][1][G*m][T]
    v = v * (t.reshape(T, 1) < lens)
    q = st["q"].float().reshape(L, n, Hkv, Hq // Hkv * m, D)
    x = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = torch.log(total) + torch.where(top > -math.inf, top, 0.0)
    return (out.to(st["q"].dtype).reshape(L, n, Hq, m, D), lse.reshape(L, n, Hq, m))


def _plain_store(st):
    c = st["c"]
    L, n, Hkv, D, P, new = (c[x] for x in ("L", "n", "Hkv", "D", "P", "new"))
    t = st["start"].reshape(n, 1).long() + torch.arange(new, device=DEV)
    page, at = st["table"].gather(1, t // P).long(), t % P         # [n][new]
    pool, out = st["pool"], []
    half, sc = P * D // 2, P * D // 32
    byte = torch.arange(D // 2, device=DEV)
    block = torch.arange(D // 32, device=DEV)
    at = at.unsqueeze(-1)
    # byte offsets of a position's codes and scales within a unit
    per = D // 32
    kpos = at * (D // 2) + byte
    vpos = half + ((at // 4 * 16 + byte // per) * 4 + at % 4) * per + byte % per
    kscale = 2 * half + at * per + block
    vscale = 2 * half + sc + (at // 4 * per + block) * 4 + at % 4
    p = page.unsqueeze(-1)
    for x, cpos, spos in ((st["k"], kpos, kscale), (st["v"], vpos, vscale)):
        code, scale = _quantise(x)
        pool[p, :, :, cpos] = _pairs(code).permute(1, 3, 4, 0, 2)
        pool[p, :, :, spos] = scale.permute(1, 3, 4, 0, 2)
    for cpos, spos in ((kpos, kscale), (vpos, vscale)):
        code = _unpairs(pool[p, :, :, cpos].permute(3, 0, 4, 1, 2))
        scale = pool[p, :, :, spos].permute(3, 0, 4, 1, 2)
        out.append(_values(code, scale).to(st["k"].dtype))
    return out


def _held(st, seqs):
    """Pages of the sequences [n][width], and which entries are pages."""
    rows = st["table"][seqs.long()]
    return rows, rows >= 0


def _give_back(st, seqs):
    rows, held = _held(st, seqs)
    gone = torch.bincount(rows[held].long(), minlength=st["refs"].numel())
    st["refs"] -= gone.to(torch.int32)
    st["table"][seqs.long()] = -1
    st["lens"][seqs.long()] = 0


def _take(st, count):
    """The lowest `count` free pages, taken."""
    new = torch.nonzero(st["refs"] == 0).flatten()[:count]
    st["refs"][new] = 1
    return new.to(torch.int32)


def _plain_fork(st):
    c = st["c"]
    P, table, lens = c["P"], st["table"], st["lens"]
    kids, par = st["children"].long(), st["parents"].long()
    _give_back(st, kids)
    rows, held = _held(st, par)
    col = torch.arange(rows.shape[1], device=DEV)
    size = lens[par].reshape(-1, 1)
    own_page = held if c["copy"] else held & (col >= size // P)    # the part page, or all
    old = rows[own_page].long()
    new = _take(st, old.numel())
    st["pool"][new.long()] = st["pool"][old]
    rows = rows.clone()
    rows[own_page] = new
    share = rows[held & ~own_page].long()
    st["refs"] += torch.bincount(share, minlength=st["refs"].numel()).to(torch.int32)
    table[kids] = rows
    lens[kids] = lens[par]
    # room for the next position of each child
    size = lens[kids] + st["add"]
    need = (col * P < size.reshape(-1, 1)) & (rows < 0)
    rows[need] = _take(st, int(need.sum()))
    table[kids] = rows
    lens[kids] = size
    return {k: st[k] for k in ("pool", "refs", "table", "lens")}


def _plain_thin(st):
    c = st["c"]
    n, L, H, D, P, keep = (c[x] for x in ("n", "L", "Hkv", "D", "P", "keep"))
    _give_back(st, st["dst"])
    pages = _pages_of(keep, c)
    new = _take(st, n * pages).reshape(n, pages)
    room = pages * P
    idx = torch.nn.functional.pad(st["idx"].long(), (0, room - keep), value=-1)
    idx = idx.expand(n, L, H, room)
    src = st["table"][st["src"].long()].long()                     # [n][width]
    page = src.gather(1, (idx.clamp(min=0) // P).reshape(n, -1)).reshape(idx.shape)
    at = idx.clamp(min=0) % P
    kept = (idx >= 0).unsqueeze(-1)
    half, sc, per = P * D // 2, P * D // 32, D // 32
    flat = st["pool"].flatten()
    unit = (page * L + torch.arange(L, device=DEV).reshape(L, 1, 1)) * H
    base = ((unit + torch.arange(H, device=DEV).reshape(H, 1)) * _unit(c)).unsqueeze(-1)
    at = at.unsqueeze(-1)
    byte, block = torch.arange(D // 2, device=DEV), torch.arange(per, device=DEV)
    kb = flat[base + at * (D // 2) + byte]
    vb = flat[base + half + ((at // 4 * 16 + byte // per) * 4 + at % 4) * per + byte % per]
    ks = flat[base + 2 * half + at * per + block]
    vs = flat[base + 2 * half + sc + (at // 4 * per + block) * 4 + at % 4]
    # positions behind the last kept one: codes of zero, the least scale
    kb, vb = (torch.where(kept, x, 0) for x in (kb, vb))
    ks, vs = (torch.where(kept, x, 3) for x in (ks, vs))
    vb = vb.reshape(n, L, H, room // 4, 4, 16, per).transpose(-3, -2)
    vs = vs.reshape(n, L, H, room // 4, 4, per).transpose(-2, -1)
    units = torch.cat([x.reshape(n, L, H, pages, -1) for x in (kb, vb, ks, vs)], -1)
    st["pool"][new.long()] = units.permute(0, 3, 1, 2, 4)
    dst = st["dst"].long()
    st["table"][dst, :pages] = new
    st["lens"][dst] = keep
    return {k: st[k] for k in ("pool", "refs", "table", "lens")}


# ---------------------------------------------------------------------------
# the framework's calls


def _handle(st):
    """What a serving program keeps beside its buffers: the cache's descriptor
    and the scratch of its calls."""
    import paper_2609_32046_amd as cb

    if "cache" not in st:
        c = st["c"]
        h = st["cache"] = cb.cache(st["pool"], st["refs"], st["table"], st["lens"],
                                   head_dim=c["D"], page_len=c["P"])
        n = 0
        if c["kind"] == "attend":
            n = cb.cb_cache_attend_workspace_bytes(h, c["L"], c["n"], c["Hq"], c["m"])
        elif c["kind"] == "fork":
            n = cb.cb_cache_fork_workspace_bytes(h, c["parents"] * c["each"])
            st["forked"] = torch.empty_like(st["status"])   # the extension has a word of its own
        elif c["kind"] == "thin":
            n = cb.cb_cache_compact_workspace_bytes(h, c["n"])
        st["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return cb, st["cache"]


def _own(st):
    c = st["c"]
    if c["kind"] == "rope":
        import paper_2609_32046_amd as cb

        if "rows" not in st:
            st["rows"] = []
            for x, y in zip(st["parts"], st["out"]):
                st["rows"].append(cb.rows(x, y, st["pos"], st["from"]))
        cb.cb_rotary(st["rows"], st["freq"], amplitude=st["amplitude"],
                     interleaved=c["interleaved"], transpose=c["transpose"])
        return st["out"]
    cb, h = _handle(st)
    if c["kind"] == "attend":
        cb.cb_cache_attend(h, st["q"], st["out"], lse=st["lse"], causal=c["causal"], ws=st["ws"])
        return st["out"], st["lse"]
    if c["kind"] == "store":
        cb.cb_cache_write(h, st["k"], st["v"], start=st["start"])
        cb.cb_cache_read(h, st["k_out"], st["v_out"], start=st["start"])
        return [st["k_out"], st["v_out"]]
    if c["kind"] == "fork":
        cb.cb_cache_free(h, st["children"])
        cb.cb_cache_fork(h, st["parents"], st["children"], st["forked"], st["ws"], copy=c["copy"])
        cb.cb_cache_extend(h, st["children"], st["add"], st["status"])
    else:
        cb.cb_cache_compact(h, st["src"], st["dst"], st["idx"], st["status"], st["ws"])
    return {k: st[k] for k in ("pool", "refs", "table", "lens")}


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "attend": _plain_attend, "store": _plain_store,
            "fork": _plain_fork, "thin": _plain_thin}[state["c"]["kind"]](state)


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions


def _exact_rope(c, seed):
    parts, pos, frm = _rope_inputs(c, seed)
    f, amp = _frequencies(c["R"], c["scaling"])
    if c["move"]:
        amp = 1.0
    got = []
    for x in parts:
        y = x.double()
        for a in range(x.shape[0]):
            p = pos[0 if c["move"] else a].double()
            if frm is not None:
                p = p - frm[a].double()
            turns = torch.remainder(p.unsqueeze(-1) * f.to(DEV), 1.0)
            w = torch.polar(torch.full_like(turns, amp), 2.0 * math.pi * turns)
            if c["transpose"]:
                w = w.conj()
            z = y[a, ..., :c["R"]]
            if c["interleaved"]:
                z = torch.view_as_complex(z.unflatten(-1, (-1, 2)).contiguous()) * w
                y[a, ..., :c["R"]] = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(z[..., :c["R"] // 2].contiguous(),
                                  z[..., c["R"] // 2:].contiguous()) * w
                y[a, ..., :c["R"]] = torch.cat([z.real, z.imag], -1)
        got.append(y)
    return got


def _read64(units, P, D):
    """Keys and values [P, D] of one page's unit, byte by byte of its layout."""
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=units.device)

    def row(b):   # [..., bytes] to [..., 2 * bytes]
        lo, hi = b % 16, b // 16
        x = torch.stack([lo, hi], -1).flatten(-2)
        return level[x % 8] * (1 - 2 * (x // 8))

    u = units.long()
    n = P * D // 2
    k = row(u[:, :n].reshape(-1, P, D // 2))
    ks = 2.0 ** (u[:, 2 * n:2 * n + P * D // 32].reshape(-1, P, D // 32) - 127).double()
    v = row(u[:, n:2 * n].reshape(-1, P // 4, 16, 4, D // 32)).permute(0, 1, 3, 2, 4)
    vs = 2.0 ** (u[:, 2 * n + P * D // 32:].reshape(-1, P // 4, D // 32, 4) - 127).double()
    vs = vs.permute(0, 1, 3, 2).reshape(-1, P, D // 32)
    k = k.reshape(-1, D) * ks.reshape(-1, D // 32).repeat_interleave(32, dim=1)
    v = v.reshape(-1, D) * vs.reshape(-1, D // 32).repeat_interleave(32, dim=1)
    return k, v


def _exact_attend(c, seed):
    lens = _lens(c, seed)
    st = _cache(c, seed, lens, _fill)
    q = _queries(c, seed)
    G, m, D = c["Hq"] // c["Hkv"], c["m"], c["D"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:-1], -math.inf, dtype=torch.float64, device=DEV)
    for b, T in enumerate(lens):
        if T == 0:
            continue
        pages = st["table"][b, :_pages_of(T, c)].long()
        for l in range(c["L"]):
            for h in range(c["Hkv"]):
                k, v = _read64(st["pool"][pages, l, h], c["P"], D)
                k, v = k[:T], v[:T]
                rows = q[l, b, h * G:(h + 1) * G].double().reshape(G * m, D)
                x = rows @ k.t().contiguous() / math.sqrt(D)
                if c["causal"] and m > 1:
                    r = torch.arange(m, device=DEV).repeat(G).reshape(-1, 1)
                    x.masked_fill_(torch.arange(T, device=DEV) > T - m + r, -math.inf)
                z = torch.logsumexp(x, -1, keepdim=True)
                w = torch.exp(x - torch.nan_to_num(z, neginf=0.0))
                out[l, b, h * G:(h + 1) * G] = (w @ v).reshape(G, m, D)
                lse[l, b, h * G:(h + 1) * G] = z.reshape(G, m)
    return out, lse


def _exact_store(c, seed):
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=DEV)
    border = (level[1:] + level[:-1]) / 2
    got = []
    for x in _new_rows(c, seed):
        out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
        for l in range(c["L"]):
            y = x[l].double().unflatten(-1, (-1, 32))
            top = y.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(top / 7.0)).clamp(-124, 125)
            e = torch.where(top > 7.0 * 2.0 ** e, e + 1, e)        # log2's own rounding
            e = torch.where(top <= 7.0 * 2.0 ** (e - 1), e - 1, e).clamp(-124, 125)
            z = y.abs() * 2.0 ** -e
            # the nearest level; half way between two, the one of even number
            lo = torch.bucketize(z, border)                        # border[lo-1] < z <= border[lo]
            tie = (lo < 7) & (z == border[lo.clamp(max=6)])
            lo = torch.where(tie & (lo % 2 == 1), lo + 1, lo)
            out[l] = (torch.sign(y) * level[lo] * 2.0 ** e).flatten(-2)
        got.append(out)
    return got


def exact(case, seed):
    c = dict(case)
    if c["kind"] == "rope":
        return _exact_rope(c, seed)
    if c["kind"] == "attend":
        return _exact_attend(c, seed)
    if c["kind"] == "store":
        return _exact_store(c, seed)
    return None   # pages and counts: whole numbers
