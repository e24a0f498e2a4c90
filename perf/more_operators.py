"""A cache of keys and values in pages, as measurable cases.

Tokens that are served one after another keep their keys and values.  Sequences
of different lengths share one pool of pages; a table names the pages of each
sequence.  Three operators work on it:

``write``   the keys and values of new tokens into their places, as they are or
            in 8 or 4 bits with a power of two for each 32 neighbours of a head;
``read``    the last tokens of each sequence back from it;
``attend``  attention of new tokens, one or a chunk for each sequence, over what
            the cache holds, within a window and the first keys.

The rows of all sequences stand one behind another; ``offsets`` says where each
sequence's begin.  ``own`` False computes them by elementary torch operations in
32 bits, True by the library's kernels.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BITS = {"plain": 0, "e4m3": 8, "e2m1": 4}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _move(name, op, dtype, fmt, B, rows, longest, Hkv, D, page, ragged):
    return {"name": name, "op": op, "dtype": dtype, "fmt": fmt, "B": B, "rows": rows, "longest": longest,
            "Hkv": Hkv, "D": D, "page": page, "ragged": ragged}


def _attend(name, dtype, fmt, B, rows, longest, Hq, Hkv, D, page, left, sinks, ragged):
    return {**_move(name, "attend", dtype, fmt, B, rows, longest, Hkv, D, page, ragged), "Hq": Hq,
            "left": left, "sinks": sinks}


def listed():
    return [
        # A serving step: the keys and values of one new token for each of 32
        # sequences; latency is all.
        _move("write_token_e4m3", "write", "bf16", "e4m3", 32, 1, 8192, 8, 128, 64, True),
        # Prompts that arrive in chunks, of different lengths; the most bytes
        # that are written.
        _move("write_prompt_e4m3", "write", "bf16", "e4m3", 16, 4096, 8192, 8, 128, 64, True),
        # The tokens of images cut to an odd size, as they are: a head that is
        # no power of two, pages that are not either.
        _move("write_odd_plain_f32", "write", "f32", "plain", 3, 1001, 1500, 6, 80, 24, True),
        # Whole sequences back for a pass over all their tokens (and the most
        # bytes that are read back).
        _move("read_all_e4m3", "read", "bf16", "e4m3", 8, 8192, 8192, 8, 128, 64, False),
        # The last chunk of each sequence back from the smallest cache.
        _move("read_chunk_e2m1_f16", "read", "f16", "e2m1", 8, 500, 3000, 4, 64, 32, True),
        # One new token over the tokens of a 14 x 14 map, one sequence: the
        # smallest call of attention.
        _attend("token_map14_f32", "f32", "plain", 1, 1, 196, 8, 8, 64, 16, -1, 0, False),
        # Serving steps: one new token for each of many sequences of different
        # lengths, shared heads; bound by memory.
        _attend("token_long_bf16", "bf16", "plain", 32, 1, 16384, 32, 8, 128, 64, -1, 0, True),
        _attend("token_long_e4m3", "bf16", "e4m3", 64, 1, 16384, 32, 4, 128, 64, -1, 0, True),
        # One sequence with a very long cache of 4 bits, five drafted tokens.
        _attend("draft_longest_e2m1_f16", "f16", "e2m1", 1, 5, 131072, 32, 8, 128, 128, -1, 0, False),
        # Chunks of prompts over what is cached of them; bound by arithmetic.
        _attend("chunk_bf16", "bf16", "plain", 4, 512, 8192, 32, 8, 128, 64, -1, 0, True),
        # A step that takes chunks of some sequences and single tokens of the
        # others, within a window and the first tokens.
        _attend("mixed_window_e4m3", "bf16", "e4m3", 16, 700, 12000, 16, 2, 128, 32, 4095, 4, True),
        # The tokens of images cut to an odd size, in the library's own type.
        _attend("chunk_odd_f32", "f32", "plain", 3, 57, 1001, 6, 2, 80, 24, 300, 1, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most:
            del case["name"]
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _drawn(rng):
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    fmt = rng.choice(["plain", "e4m3", "e2m1"])
    D = rng.choice([40, 64, 80, 96, 128, 128, 256] if fmt == "plain" else [32, 64, 96, 128, 128, 256])
    page = rng.choice([8, 16, 24, 32, 64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    ragged = rng.random() < 0.7
    op = rng.choice(["write", "read", "token", "token", "chunk", "chunk"])
    if op in ("write", "read"):
        rows = rng.choice([1, _log(rng, 2, 4096)])
        return _move(None, op, dtype, fmt, _log(rng, 1, 48), rows, rows + _log(rng, 1, 8192), Hkv, D, page, ragged)
    left = rng.choice([-1, _log(rng, 16, 4096)])
    sinks = 0 if left < 0 else rng.randrange(6)
    Hq = Hkv * rng.choice([1, 2, 4, 7, 8])
    if op == "token":
        rows = rng.choice([1, 1, 1, 2, 5])
        return _attend(None, dtype, fmt, _log(rng, 1, 64), rows, rows + _log(rng, 16, 32768), Hq, Hkv, D, page,
                       left, sinks, ragged)
    rows = _log(rng, 6, 1500)
    return _attend(None, dtype, fmt, rng.randrange(1, 17), rows, rows + _log(rng, 1, 6000), Hq, Hkv, D, page,
                   left, sinks, ragged)


def _rows(case):
    """New tokens of each sequence.  In a ragged batch of chunks every fourth
    sequence brings a chunk (of its own length), one nothing and the others one
    token each; a batch of four or less brings chunks only."""
    B, rows = case["B"], case["rows"]
    if not case["ragged"] or rows == 1:
        return [rows] * B
    n = []
    for b in range(B):
        chunk = max(1, rows - (b * 37) % max(1, rows // 2))
        n.append(chunk if B <= 4 or case["op"] != "attend" or b % 4 == 0 else 0 if b == 3 else 1)
    return n


def _lengths(case):
    """Tokens of each sequence, the new ones among them.  Ragged batches step
    down from the longest."""
    B, most = case["B"], case["longest"]
    if not case["ragged"]:
        return [most] * B
    return [max(r, most - b * (most // (B + 1)) - (b * 37) % max(1, most // (2 * B + 2)))
            for b, r in enumerate(_rows(case))]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    N, Hkv, D, bits = sum(_rows(case)), case["Hkv"], case["D"], _BITS[case["fmt"]]
    stored = 2 * Hkv * (D * bits // 8 + D // 32 if bits else D * es)     # bytes of a token's keys and values
    if case["op"] == "write" or case["op"] == "read":
        return {"bytes": N * (stored + 2 * Hkv * D * es), "flops": 2 * 4 * N * Hkv * D}
    pairs = keys = 0
    for n, r in zip(_lengths(case), _rows(case)):
        if r == 0:
            continue
        pos = np.arange(n - r, n, dtype=np.int64)
        lo = np.zeros_like(pos) if case["left"] < 0 else np.clip(pos - case["left"], 0, None)
        pairs += int((pos + 1 - lo + np.minimum(case["sinks"], lo)).sum())
        keys += int(n - lo[0] + min(case["sinks"], lo[0]))
    return {"bytes": 2 * es * N * case["Hq"] * D + keys * stored, "flops": 4 * pairs * case["Hq"] * D}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
#: Largest code of a format, and the largest value whose code reads back as finite, by type.
_LARGEST = {"e4m3": 448.0, "e2m1": 6.0}
_LIMIT = {("e4m3", "f16"): 61440.0, ("e2m1", "f16"): 49152.0, ("e4m3", "bf16"): 1.875 * 2.0 ** 127,
          ("e2m1", "bf16"): 1.5 * 2.0 ** 127, ("e4m3", "f32"): 1.875 * 2.0 ** 127,
          ("e2m1", "f32"): 1.5 * 2.0 ** 127}


def _encode(x, fmt, dtype):
    """x [..., D] as its stored form: codes and exponents, each of the stored type.
    A scale is the smallest power of two with which the largest of 32 neighbours
    has a code; dividing by it is exact."""
    if fmt == "plain":
        return x, None
    limit = _LIMIT[fmt, dtype]
    x = x.float().reshape(*x.shape[:-1], -1, 32).clamp(-limit, limit)
    top, largest = x.abs().amax(-1, keepdim=True), _LARGEST[fmt]
    m, e = torch.frexp(top / largest)      # m in [0.5, 1), and the quotient is rounded
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(top.double() > largest * torch.exp2(e.double()), e + 1, e)
    e = torch.where(top == 0, -127, e).clamp(min=-127)
    y = torch.ldexp(x.double(), -e).float().flatten(-2)
    scale = (e.squeeze(-1) + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn), scale
    a = y.abs()
    # halves up to 2, ones up to 4, then 4 and 6; ties to the even code
    q = torch.where(a <= 2, torch.round(a * 2), torch.where(a <= 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    code = q.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _decode(code, scale, fmt):
    """The values in 32 bits."""
    if fmt == "plain":
        return code.float()
    if fmt == "e2m1":
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=code.device)
        table = torch.cat([table, -table])
        code = torch.stack([table[(code & 15).long()], table[(code >> 4).long()]], -1).flatten(-2)
    return code.float() * torch.exp2(scale.view(torch.uint8).float() - 127).repeat_interleave(32, -1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    B, Hkv, D, page, fmt = (case[n] for n in ("B", "Hkv", "D", "page", "fmt"))
    st = {"case": case, "rows": _rows(case), "long": _lengths(case)}
    # Sequences hold whole pages, in any order; a table is as wide as the longest
    # needs, and names no page behind a sequence's last.
    held = [-(-n // page) for n in st["long"]]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((B, max(held)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    st["table"] = table
    st["lengths"] = torch.tensor(st["long"], dtype=torch.int32, device=dev)
    even = len(set(st["rows"])) == 1
    st["offsets"] = None if even else torch.tensor([0] + list(np.cumsum(st["rows"])), dtype=torch.int32, device=dev)
    N = sum(st["rows"])

    # Keys have a few channels that are larger than the others, values have not.
    loud = 1.0 + 5.0 * (torch.rand(Hkv, D, generator=g, device=dev) < 0.04).float()

    def tokens(*lead):
        return (torch.randn((*lead, Hkv, D), generator=g, device=dev) * loud).to(dt), \
            torch.randn((*lead, Hkv, D), generator=g, device=dev).to(dt)

    # A page holds the tokens of one head after another.
    shape = (pages, Hkv, page, D)
    store = {"plain": dt, "e4m3": torch.float8_e4m3fn, "e2m1": torch.uint8}[fmt]
    names = ("k", "v", "k_scale", "v_scale")
    if case["op"] == "write":
        kept = [torch.zeros(*shape[:3], D // 2 if fmt == "e2m1" else D, device=dev).to(store) for _ in range(2)]
        kept += [torch.zeros(*shape[:3], D // 32, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
                 for _ in range(2)] if fmt != "plain" else [None, None]
        qkv = torch.randn(N, 3 * Hkv, D, generator=g, device=dev)     # heads of one fused projection
        qkv[:, Hkv:2 * Hkv] *= loud
        qkv = qkv.to(dt)
        st["k_new"], st["v_new"] = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:]
    else:
        kept = [None] * 4
        step = max(1, (1 << 26) // (Hkv * page * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            for i, x in enumerate(tokens(n, page)):
                for j, part in ((i, 0), (i + 2, 1)):
                    y = _encode(x.transpose(1, 2), fmt, case["dtype"])[part]
                    if y is None:
                        continue
                    if kept[j] is None:
                        kept[j] = torch.empty((pages, *y.shape[1:]), dtype=y.dtype, device=dev)
                    kept[j][p:p + n] = y
        if case["op"] == "attend":
            st["q"] = torch.randn(N, case["Hq"], D, generator=g, device=dev).to(dt)
    # [pages, page, heads, D]
    st["kept"] = {n: None if t is None else t.transpose(1, 2) for n, t in zip(names, kept)}
    if own:
        import paper_2212_00404_amd as dc
        st["cache"] = dc.Cache(**st["kept"])
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _stored(st):
    """What a written cache holds, as the values that its bits stand for: of the
    smallest format as the new tokens read back."""
    return {n: t for n, t in st["kept"].items() if t is not None}


def _own_write(st):
    import paper_2212_00404_amd as dc
    where = (st["table"], st["lengths"], st["offsets"])
    dc.cache_write(st["cache"], st["k_new"], st["v_new"], *where)
    if st["case"]["fmt"] == "e2m1":
        k, v = dc.cache_read(st["cache"], st["k_new"].shape[0], *where, dtype=st["k_new"].dtype)
        return {"k": k, "v": v}
    return _stored(st)


def _own_read(st):
    import paper_2212_00404_amd as dc
    c = st["case"]
    k, v = dc.cache_read(st["cache"], sum(st["rows"]), st["table"], st["lengths"], st["offsets"],
                         dtype=_TYPES[c["dtype"]])
    return {"k": k, "v": v}


def _own_attend(st):
    import paper_2212_00404_amd as dc
    c = st["case"]
    return dc.attend_cache(st["q"], st["cache"], st["table"], st["lengths"], st["offsets"], left=c["left"],
                           sinks=c["sinks"])


# ---------------------------------------------------------------------------
# Plain forms: elementary operations in 32 bits, rounded once at the end
# ---------------------------------------------------------------------------
def _places(st):
    """Page and slot of each row."""
    page = st["case"]["page"]
    pages, slots = [], []
    for b, (n, r) in enumerate(zip(st["long"], st["rows"])):
        i = torch.arange(n - r, n, device=st["table"].device)
        pages.append(st["table"][b, i // page].long())
        slots.append(i % page)
    return torch.cat(pages), torch.cat(slots)


def _plain_write(st):
    c = st["case"]
    at = _places(st)
    for n, x in (("k", st["k_new"]), ("v", st["v_new"])):
        code, scale = _encode(x, c["fmt"], c["dtype"])
        kept = st["kept"][n]
        if c["fmt"] == "e4m3":
            kept, code = kept.view(torch.uint8), code.view(torch.uint8)
        kept[at] = code
        if scale is not None:
            st["kept"][n + "_scale"].view(torch.uint8)[at] = scale.view(torch.uint8)
    return _plain_read(st) if c["fmt"] == "e2m1" else _stored(st)


def _rows_of(kept, name, at, fmt):
    """The tokens at the places `at` in 32 bits."""
    if fmt == "plain":
        return kept[name][at].float()
    code = kept[name].view(torch.uint8)[at]
    if fmt == "e4m3":
        code = code.view(torch.float8_e4m3fn)
    return _decode(code, kept[name + "_scale"].view(torch.uint8)[at].view(torch.float8_e8m0fnu), fmt)


def _plain_read(st):
    c, at = st["case"], _places(st)
    return {n: _rows_of(st["kept"], n, at, c["fmt"]).to(_TYPES[c["dtype"]]) for n in ("k", "v")}


def _plain_attend(st):
    c = st["case"]
    q = st["q"]
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]
    G = Hq // Hkv
    out = torch.zeros(q.shape, device=q.device)
    at = 0
    for b, (n, r) in enumerate(zip(st["long"], st["rows"])):
        first = max(0, n - r - c["left"]) if c["left"] >= 0 else 0      # the keys that the window leaves
        first = first // page * page
        j = torch.arange(first, n, device=q.device)
        sinks = min(c["sinks"], first)
        j = torch.cat([torch.arange(sinks, device=q.device), j])
        where = (st["table"][b, j // page].long(), j % page)
        k = _rows_of(st["kept"], "k", where, c["fmt"]).permute(1, 0, 2)
        v = _rows_of(st["kept"], "v", where, c["fmt"]).permute(1, 0, 2)
        for t0 in range(0, r, 128):
            t1 = min(r, t0 + 128)
            i = n - r + torch.arange(t0, t1, device=q.device)
            seen = j[None] <= i[:, None]
            if c["left"] >= 0:
                seen = seen & ((j[None] >= i[:, None] - c["left"]) | (j[None] < c["sinks"]))
            seen = seen.repeat_interleave(G, 0)                         # rows: query, then head of the group
            x = q[at + t0:at + t1].float().reshape(t1 - t0, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
            s = (x @ k.transpose(1, 2) / math.sqrt(D)).masked_fill(~seen, -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = p @ v / p.sum(-1, keepdim=True)
            out[at + t0:at + t1] = o.reshape(Hkv, t1 - t0, G, D).permute(1, 0, 2, 3).reshape(t1 - t0, Hq, D)
        at += r
    return out.to(q.dtype)


_own = {"write": _own_write, "read": _own_read, "attend": _own_attend}
_plain = {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["op"]](case, st)


def _grid(fmt):
    """The values of a format's codes that are not negative, in order."""
    if fmt == "e2m1":
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    sub = [m / 8 * 2.0 ** -6 for m in range(8)]
    return torch.tensor(sub + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1],
                        dtype=torch.float64)


def _nearest(x, fmt):
    """The nearest value of the grid, the one at an even place between two."""
    grid = _grid(fmt).to(x.device)
    a = x.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    take = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(grid[take], x)


def _exact_write(c, st):
    """Each block of 32 by its own: the scale by trying the next power of two."""
    out = {}
    for n, x in (("k", st["k_new"]), ("v", st["v_new"])):
        x = x.double()
        page = torch.full(st["kept"][n].shape[:3], -1, dtype=torch.int64, device=x.device)
        row = 0
        for b in range(c["B"]):
            for t in range(0, st["rows"][b]):
                i = st["long"][b] - st["rows"][b] + t
                if t == 0 or i % c["page"] == 0:
                    upto = min(st["rows"][b], t + c["page"] - i % c["page"])
                    s = i % c["page"]
                    page[st["table"][b, i // c["page"]], s:s + upto - t] = torch.arange(
                        row + t, row + upto, device=x.device)[:, None]
            row += st["rows"][b]
        new = page >= 0
        take = page.clamp(min=0)
        head = torch.arange(c["Hkv"], device=x.device).expand_as(take)
        if c["fmt"] == "plain":
            out[n] = torch.where(new[..., None], x[take, head], 0.0)
            continue
        blocks = x.clamp(-_LIMIT[c["fmt"], c["dtype"]], _LIMIT[c["fmt"], c["dtype"]]).reshape(*x.shape[:2], -1, 32)
        top = blocks.abs().amax(-1)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -120))) - 9      # too small
        for _ in range(10):
            e = torch.where(torch.exp2(e) * _LARGEST[c["fmt"]] < top, e + 1, e)
        s = torch.exp2(torch.where(top == 0, -127.0, e).clamp(min=-127))
        value = _nearest(blocks / s[..., None], c["fmt"]).flatten(-2)
        if c["fmt"] == "e2m1":
            out[n] = (value.reshape(blocks.shape) * s[..., None]).flatten(-2)
            continue
        out[n] = torch.where(new[..., None], value[take, head], 0.0)
        out[n + "_scale"] = torch.where(new[..., None], s[take, head], 2.0 ** -127)
    if c["fmt"] == "e4m3":
        return {n: out[n] for n in ("k", "v", "k_scale", "v_scale")}
    return out


def _bits(code, scale, fmt):
    """Values by the meaning of the bits, in 64."""
    if fmt == "plain":
        return code.double()
    if fmt == "e4m3":
        bits = code.view(torch.uint8).long()
        sign, e, m = 1.0 - 2.0 * (bits >> 7).double(), bits >> 3 & 15, (bits & 7).double()
        x = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7)) * sign
    else:
        two = torch.stack([code % 16, code // 16], -1).long().flatten(-2)
        e, m = two >> 1 & 3, (two & 1).double()
        x = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1)) * (1.0 - 2.0 * (two >> 3).double())
    s = torch.exp2(scale.view(torch.uint8).double() - 127)
    return (x.reshape(*s.shape, 32) * s[..., None]).flatten(-2)


def _sequence(c, st, name, b, j):
    """Tokens j of sequence b, in 64 bits: [tokens, heads, D]."""
    page, slot = st["table"][b].long()[j // c["page"]], j % c["page"]
    code = st["kept"][name]
    if c["fmt"] == "e4m3":
        code = code.view(torch.uint8)
    scale = st["kept"][name + "_scale"]
    return _bits(code[page, slot], None if scale is None else scale.view(torch.uint8)[page, slot], c["fmt"])


def _exact_read(c, st):
    dev = st["table"].device
    return {n: torch.cat([_sequence(c, st, n, b, torch.arange(L - r, L, device=dev))
                          for b, (L, r) in enumerate(zip(st["long"], st["rows"]))]) for n in ("k", "v")}


def _exact_attend(c, st):
    """Each head's whole matrix of probabilities."""
    q = st["q"].double()
    out = torch.zeros_like(q)
    at = 0
    for L, r, b in zip(st["long"], st["rows"], range(c["B"])):
        if r == 0:
            continue
        j = torch.arange(L, device=q.device)
        K, V = _sequence(c, st, "k", b, j), _sequence(c, st, "v", b, j)
        i = torch.arange(L - r, L, device=q.device)[:, None]
        hidden = j[None] > i
        if c["left"] >= 0:
            hidden |= (i - j[None] > c["left"]) & (j[None] >= c["sinks"])
        for head in range(c["Hq"]):
            kv = head * c["Hkv"] // c["Hq"]
            P = q[at:at + r, head] @ K[:, kv].T.contiguous()
            P /= math.sqrt(c["D"])
            P[hidden] = -math.inf
            out[at:at + r, head] = torch.softmax(P, -1) @ V[:, kv].contiguous()
        at += r
    return out
