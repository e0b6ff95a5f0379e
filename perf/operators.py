"""Attention over a paged KV cache and the cache's own reads and writes, as timed cases.

A pool holds pages of `T` rows of every layer and KV head, [P, L, H, T, D], in
bf16, fp32, or as 8- or 4-bit elements (e4m3, e2m1) with one power-of-two scale
for each 32 elements of a row. Row j of stream b lies in page
table[b][j // T], slot j % T. Three operators:

  attend  a chunk of new tokens (or one) of one layer over the rows of their
          streams: softmax(scale * q k^T) v over the rows that a query at
          position p sees: j <= p, and with a window W only j > p - W or the
          first `sinks` rows
  write   rows of keys and values into the pages, keys rotated to their
          position, quantised as they are written; where the pool holds 8 or 4
          bits the pass also reads the rows back
  read    rows out of the pages, dequantised, keys rotated back

Shapes are those of the repository's workloads (7B- and 72B-class video
models of 4 and 8 KV heads of 128, frames of 196 tokens, caches of 64 to 32768
rows, the tiny fp32 cache) and odd ones.
"""
import math
import random

import torch

own = False

BLOCK = 32                    # elements that share a scale
TOP = {"fp8": 448.0, "fp4": 6.0}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, fmt, B, L, H, G, D, T, n, m, ragged=False, window=0, sinks=0, lse=False, rotary=False, src="bf16",
          token_major=False):
    c = {"op": op, "fmt": fmt, "B": B, "L": L, "H": H, "G": G, "D": D, "T": T, "n": n, "m": m, "ragged": ragged,
         "window": window, "sinks": sinks, "lse": lse, "rotary": rotary, "src": src, "token_major": token_major}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # ---- attend: n rows in the cache, of which the last m are the new tokens
        # the smallest: one token over the compacted tiny cache, latency alone
        _case("tiny-f32-token", "attend", "f32", 1, 1, 2, 2, 64, 16, 64, 1),
        # answering over a compressed 7B-class cache, one token at a time
        _case("7b-token", "attend", "bf16", 1, 2, 4, 7, 128, 64, 3203, 1),
        # 16 users answered together, each with as many rows as its video left
        _case("batch16-token-fp8", "attend", "fp8", 16, 2, 4, 7, 128, 64, 6272, 1, ragged=True, lse=True),
        # four users on the 72B-class cache, four bits an element
        _case("72b-token-fp4", "attend", "fp4", 4, 1, 8, 8, 128, 128, 32768, 1, ragged=True),
        # the next frame of a 7B-class stream over the full cache
        _case("7b-frame", "attend", "bf16", 1, 2, 4, 7, 128, 64, 6272, 196),
        # a long prompt after a 72B-class video: the largest
        _case("72b-prompt", "attend", "bf16", 1, 1, 8, 8, 128, 128, 32768, 2048, token_major=True),
        # a whole prompt with a sliding window of four frames and a first frame that stays
        _case("window-prompt-fp8", "attend", "fp8", 1, 1, 4, 7, 128, 64, 6272, 6272, window=784, sinks=196),
        # tokens of eight users over windows in long caches, few first tokens, odd pages
        _case("window-token", "attend", "bf16", 8, 1, 8, 8, 128, 100, 32768, 1, ragged=True, window=4095, sinks=5),
        # ---- write
        # one new token of 16 users, one layer
        _case("write-token-fp8", "write", "fp8", 16, 1, 4, 1, 128, 64, 6272, 1, ragged=True, rotary=True, token_major=True),
        # a compressed 7B-class cache goes into pages
        _case("write-7b-fp8", "write", "fp8", 1, 28, 4, 1, 128, 64, 3136, 3136, rotary=True),
        # ---- read
        # and comes back for the next compression
        _case("read-7b-fp8", "read", "fp8", 1, 28, 4, 1, 128, 64, 3136, 3136, rotary=True),
        # a few rows of three users from four bits, odd pages
        _case("read-odd-fp4", "read", "fp4", 3, 5, 2, 1, 64, 36, 1501, 700, ragged=True, src="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Streams 1 to 16, 1 to 32768 rows, chunks of 1 to 6272 tokens (half of
    the attention draws are single tokens or few), 1 to 12 query heads a KV
    head, every head size, type and odd page sizes; at most the largest listed
    case's products, and 1 GiB of rows read or written."""
    while True:
        op = rng.choice(("attend", "attend", "attend", "write", "read"))
        fmt = rng.choice(("bf16", "bf16", "fp8", "fp8", "fp4", "f32"))
        D = rng.choice((64, 128, 128, 256, 32))
        T = rng.choice((16, 64, 64, 128, 196, rng.randint(1, 300)))
        H = rng.choice((1, 2, 4, 8))
        B = _log(rng, 1, 16)
        n = _log(rng, 1, 32768)
        ragged = rng.random() < 0.6
        if op == "attend":
            m = min(n, _log(rng, 1, 12) if rng.random() < 0.5 else _log(rng, 12, 6272))
            G = rng.choice((1, 2, 4, 7, 8, 12))
            window = _log(rng, 1, 8192) if rng.random() < 0.4 else 0
            sinks = rng.choice((0, 1, 4, 5, 64, 196)) if window else 0
            c = _case("", op, fmt, B, rng.choice((1, 2)), H, G, D, T, n, m, ragged, window, sinks, rng.random() < 0.5,
                      token_major=rng.random() < 0.5)
            cost = B * H * G * m * n * D
            big = B * H * G * m * n
            if cost > 8 * 8 * 128 * 2048 * 32768 // (4 if fmt == "f32" else 1) or big > 64 * 2048 * 32768:
                continue
            if B * H * n * D > 1 << 28:
                continue
        else:
            L = _log(rng, 1, 28)
            m = min(n, _log(rng, 1, 6272))
            c = _case("", op, fmt, B, L, H, 1, D, T, n, m, ragged, rotary=rng.random() < 0.6,
                      src=rng.choice(("bf16", "bf16", "f32")), token_major=rng.random() < 0.5)
            if B * L * H * m * D > 1 << 26 or B * L * H * n * D > 1 << 29:
                continue
        return c


# ---------------------------------------------------------------- the 8- and 4-bit types, in plain operations
def _encode(x, fmt):
    """x [..., D] fp32 -> the elements' values before the scale, and the scales' exponents [..., D / 32]."""
    b = x.unflatten(-1, (-1, BLOCK))
    mant, exp = torch.frexp(b.abs().amax(-1))
    # the smallest e with amax <= TOP * 2^e: TOP is 0.875 * 2^9 and 0.75 * 2^3
    e = exp - (9 if fmt == "fp8" else 3) + (mant > (0.875 if fmt == "fp8" else 0.75)).int()
    e = torch.where(mant == 0, torch.full_like(e, -126), e).clamp(-126, 127)
    y = b * torch.exp2(-e.float()).unsqueeze(-1)
    if fmt == "fp8":
        y = y.to(torch.float8_e4m3fn).float()
    else:  # steps of 0.5, 1 and 2 below 2, 4 and 6, ties to even
        a = y.abs()
        r = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2))
        y = torch.copysign(r, y)
    return y.flatten(-2), e


def _decode(y, e):
    return (y.unflatten(-1, (-1, BLOCK)) * torch.exp2(e.float()).unsqueeze(-1)).flatten(-2)


def _pack(y, fmt):
    """Element values -> stored bytes: a byte each, or two elements a byte, the first in the low half."""
    if fmt == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    grid = torch.tensor(GRID4, device=y.device)
    c = torch.bucketize(y.abs(), grid).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    c = c.unflatten(-1, (-1, 2))
    return c[..., 0] | (c[..., 1] << 4)


def _unpack(b, fmt):
    if fmt == "fp8":
        return b.view(torch.float8_e4m3fn).float()
    grid = torch.tensor(GRID4 + tuple(-g for g in GRID4), device=b.device)
    return grid[torch.stack((b & 15, b >> 4), -1).flatten(-2).int()]


def _rotate(x, table, at, back=False):
    """x [B, L, H, N, D] fp32, its row i of stream b turned to position at[b][i] (or back)."""
    c, s = table[at][:, None, None].unbind(-1)  # [B, 1, 1, N, D / 2]
    s = -s if back else s
    lo, hi = x.chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


# ---------------------------------------------------------------- inputs
def _counts(case, rng):
    """Rows of each stream: n, or between half of it and n."""
    return [rng.randint(max(case["m"], (case["n"] + 1) // 2), case["n"]) if case["ragged"] and b else case["n"]
            for b in range(case["B"])]


def _fill(g, shape, spread):
    """Normal rows; keys have a few larger channels, values one log-normal scale a row."""
    x = torch.randn(shape, generator=g, device="cuda")
    if spread:
        return x.mul_(torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda")))
    return x.mul_(1 + 2 * (torch.rand(shape[-1], generator=g, device="cuda") > 0.95))


def prepare(case, seed):
    """Pools with their pages in random order and a few unused, the page table,
    the counts; queries, or the rows to write, or room for the rows to read."""
    rng = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, L, H, D, T, n, m, fmt = (case[k] for k in ("B", "L", "H", "D", "T", "n", "m", "fmt"))
    counts = _counts(case, rng)
    cols = -(-n // T)
    pages = B * cols + 2
    order = torch.randperm(pages, generator=g, device="cuda").int()
    s = {"case": case, "n": counts, "first": [c - m for c in counts], "table": order[:B * cols].view(B, cols).contiguous(), "cols": cols}
    pool = (pages, L, H, T, D)
    if case["op"] == "write":  # empty pages
        fills = [torch.zeros(pool, device="cuda") for _ in range(2)]
    else:
        fills = [_fill(g, pool, spread) for spread in (False, True)]
    for name, x in zip("KV", fills):
        if fmt in TYPE:
            s[name] = x.to(TYPE[fmt])
        else:
            y, e = _encode(x, fmt)
            s[name], s[name + "_scales"] = _pack(y, fmt), (e + 127).to(torch.uint8)
    del fills, x
    s["new"] = torch.tensor(s["first"], device="cuda")[:, None] + torch.arange(m, device="cuda")  # positions [B, m]
    if case["op"] == "attend":
        qt = torch.float32 if fmt == "f32" else torch.bfloat16
        shape = (B, m, H * case["G"], D) if case["token_major"] else (B, H * case["G"], m, D)
        q = (1.5 * torch.randn(shape, generator=g, device="cuda")).to(qt)
        s["q"] = q.transpose(1, 2) if case["token_major"] else q
        s["scale"] = 1 / math.sqrt(D)
        return s
    if case["rotary"]:
        a = torch.arange(n, device="cuda")[:, None] * torch.exp(-math.log(1e6) * torch.arange(D // 2, device="cuda") / (D // 2))
        s["rotary"] = torch.stack((a.cos(), a.sin()), -1).float().contiguous()
    shape = (B, L, m, H, D) if case["token_major"] else (B, L, H, m, D)
    for name, spread in (("K", False), ("V", True)):
        x = _fill(g, shape, spread) if case["op"] == "write" else torch.empty(shape, device="cuda")
        x = x.to(TYPE[case["src"]])
        s["rows_" + name] = x.transpose(2, 3) if case["token_major"] else x
    return s


# ---------------------------------------------------------------- plain forms
def _rows(s, name, at):
    """Rows at[b][i] of the pool, fp32 [B, L, H, N, D]."""
    T, fmt = s["case"]["T"], s["case"]["fmt"]
    page = s["table"].long().gather(1, at // T)
    x = s[name][page, :, :, at % T]  # [B, N, L, H, .]
    x = x.float() if fmt in TYPE else _decode(_unpack(x, fmt), s[name + "_scales"][page, :, :, at % T].int() - 127)
    return x.permute(0, 2, 3, 1, 4)


def _attend(s):
    c = s["case"]
    B, H, G, D, m, layer = c["B"], c["H"], c["G"], c["D"], c["m"], c["L"] - 1
    n = max(s["n"])
    counts = torch.tensor(s["n"], device="cuda")[:, None]
    at = torch.arange(n, device="cuda").expand(B, n)
    inside = at < counts
    K, V = (_rows(s, name, torch.where(inside, at, 0))[:, layer] for name in "KV")  # [B, H, n, D]
    q = s["q"].float().reshape(B, H, G * m, D)
    x = torch.matmul(q, K.transpose(2, 3).contiguous()).mul_(s["scale"]).view(B, H, G, m, n)
    p, j = s["new"][:, :, None], at[:, None, :]
    seen = (j <= p) & inside[:, None, :]
    if c["window"]:
        seen &= (j > p - c["window"]) | (j < c["sinks"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(B, H, G * m, n), V).view(B, H, G, m, D) / total
    out = out.view(B, H * G, m, D).to(s["q"].dtype)
    return [out, (top + total.log()).view(B, H * G, m)] if c["lse"] else [out]


def _write(s):
    c, at = s["case"], s["new"]
    page, slot = s["table"].long().gather(1, at // c["T"]), at % c["T"]
    K, V = s["rows_K"].float(), s["rows_V"].float()
    if c["rotary"]:
        K = _rotate(K, s["rotary"], at)
    for name, x in (("K", K), ("V", V)):
        x = x.permute(0, 3, 1, 2, 4)  # [B, N, L, H, D]
        if c["fmt"] in TYPE:
            s[name][page, :, :, slot] = x.to(TYPE[c["fmt"]])
        else:
            y, e = _encode(x, c["fmt"])
            s[name][page, :, :, slot] = _pack(y, c["fmt"])
            s[name + "_scales"][page, :, :, slot] = (e + 127).to(torch.uint8)
    if c["fmt"] in TYPE:
        return [s["K"], s["V"]]
    return [_rows(s, name, at).to(torch.bfloat16) for name in "KV"]


def _read(s):
    c, at = s["case"], s["new"]
    K, V = _rows(s, "K", at), _rows(s, "V", at)
    if c["rotary"]:
        K = _rotate(K, s["rotary"], at, back=True)
    return [x.to(TYPE[c["src"]]) for x in (K, V)]


# ---------------------------------------------------------------- the framework's
def _handles(s):
    """What a program makes once: the pool's handle, the workspace, the outputs."""
    from paper_2506_15745_amd import ipv

    c = s["case"]
    s["ipv"] = ipv
    s["pool"] = ipv.PagePool(s["K"], s["V"], s.get("K_scales"), s.get("V_scales"))
    if c["op"] == "attend":
        s["ws"] = ipv.alloc_attend_workspace(s["pool"], c["B"], c["H"] * c["G"], c["m"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device="cuda") if c["lse"] else None
    else:
        s["ws"] = ipv.alloc_page_workspace("cuda")
        if c["op"] == "write" and c["fmt"] not in TYPE:
            s["back"] = [torch.empty((c["B"], c["L"], c["H"], c["m"], c["D"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def _own(s):
    if "ipv" not in s:
        _handles(s)
    ipv, c = s["ipv"], s["case"]
    if c["op"] == "attend":
        ipv.ipv_attend(s["pool"], s["table"], s["n"], s["first"], c["L"] - 1, s["q"], s["out"], s["ws"], scale=s["scale"],
                       window=c["window"], sinks=c["sinks"], lse=s["lse"])
        return [s["out"], s["lse"]] if c["lse"] else [s["out"]]
    K, V, rotary = s["rows_K"], s["rows_V"], s.get("rotary")
    if c["op"] == "read":
        ipv.ipv_page_read(s["pool"], s["table"], s["first"], K, V, s["ws"], rotary=rotary)
        return [K, V]
    ipv.ipv_page_write(s["pool"], s["table"], s["first"], K, V, s["ws"], rotary=rotary)
    if c["fmt"] in TYPE:
        return [s["K"], s["V"]]
    ipv.ipv_page_read(s["pool"], s["table"], s["first"], *s["back"], s["ws"])
    return s["back"]


def run(state):
    if own:
        return _own(state)
    return {"attend": _attend, "write": _write, "read": _read}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without
def _seen(case, count):
    """(query, row) pairs of a stream of `count` rows, and the rows that some query sees."""
    m, w, k = case["m"], case["window"], case["sinks"]
    first = count - m
    if not w:
        return m * first + m * (m + 1) // 2, count
    pairs = 0
    for p in range(first, count):
        inside = min(w, p + 1)
        pairs += inside + min(k, p + 1 - inside)
    low = max(0, first - w + 1)
    return pairs, count - low + min(k, low)


def work(case):
    B, L, H, G, D, m = (case[k] for k in ("B", "L", "H", "G", "D", "m"))
    row = {"bf16": 2 * D, "f32": 4 * D, "fp8": D + D // BLOCK, "fp4": D // 2 + D // BLOCK}[case["fmt"]]
    if case["op"] == "attend":
        # ragged streams hold between half of n rows and n: three quarters on average, the first one n
        counts = [case["n"]] + [max(m, case["n"] * 3 // 4) if case["ragged"] else case["n"]] * (B - 1)
        seen = [_seen(case, c) for c in counts]
        qb = 4 if case["fmt"] == "f32" else 2
        return {"bytes": 2 * H * row * sum(r for _, r in seen) + B * H * G * m * (2 * D * qb + (4 if case["lse"] else 0)),
                "flops": 4 * D * H * G * sum(p for p, _ in seen)}
    rows = B * L * H * m
    src = (2 if case["src"] == "bf16" else 4) * D
    table = B * m * D * 4 if case["rotary"] else 0
    bytes_ = 2 * rows * (row + src) + table
    if case["op"] == "write" and case["fmt"] not in TYPE:
        bytes_ += 2 * rows * (row + 2 * D)  # and back, as bf16
    return {"bytes": bytes_, "flops": 3 * rows * D * (2 if case["rotary"] else 1)}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _exact_values(s, name, layer, b, h, rows):
    """The pool's rows of one (layer, stream, head) in 64 bits: stored bits taken apart."""
    fmt, T = s["case"]["fmt"], s["case"]["T"]
    page = s["table"][b].long()[rows // T]
    x = s[name][page, layer, h, rows % T]
    if fmt in TYPE:
        return x.double()
    if fmt == "fp8":
        v = x.int()
        e, f = (v >> 3) & 15, (v & 7).double()
        y = torch.where(e == 0, f * 2.0**-9, (8 + f) * torch.exp2((e - 10).double()))
        y = torch.where(v > 127, -y, y)
    else:
        v = torch.stack((x.int() % 16, x.int() // 16), -1).flatten(-2)
        e, f = (v >> 1) & 3, (v & 1).double()
        y = torch.where(e == 0, f * 0.5, (2 + f) * torch.exp2((e - 2).double()))
        y = torch.where(v > 7, -y, y)
    scale = s[name + "_scales"][page, layer, h, rows % T].double() - 127
    return y * torch.exp2(scale).repeat_interleave(BLOCK, -1)


def _exact_attend(s):
    c = s["case"]
    B, H, G, D, m = (c[k] for k in ("B", "H", "G", "D", "m"))
    out = torch.empty(B, H * G, m, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, H * G, m, dtype=torch.float64, device="cuda")
    for b in range(B):
        j = torch.arange(s["n"][b], device="cuda")
        for h in range(H):
            K, V = (_exact_values(s, name, c["L"] - 1, b, h, j) for name in "KV")
            for i in range(0, m, 1024):
                p = s["first"][b] + torch.arange(i, min(m, i + 1024), device="cuda")[:, None]
                hidden = j > p
                if c["window"]:
                    hidden |= (j <= p - c["window"]) & (j >= c["sinks"])
                for k in range(h * G, h * G + G):
                    x = s["scale"] * (s["q"][b, k, i:i + 1024].double() @ K.T)
                    x[hidden] = -math.inf
                    lse[b, k, i:i + 1024] = torch.logsumexp(x, -1)
                    out[b, k, i:i + 1024] = torch.softmax(x, -1) @ V
    return [out, lse] if c["lse"] else [out]


def _exact_turn(s, x, back):
    """Pairs (d, d + D/2) as complex numbers, times the position's unit number or its conjugate."""
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:])
    u = torch.view_as_complex(s["rotary"].double())[s["new"]][:, None, None]
    z = z * (u.conj() if back else u)
    return torch.cat((z.real, z.imag), -1)


def _exact_round(x, fmt):
    """Each element to the nearest of its block's values (ties to the even one)."""
    b = x.unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / TOP[fmt])).clamp(-126, 127)
    e = torch.where(top > TOP[fmt] * torch.exp2(e), e + 1, e)
    e = torch.where(top <= TOP[fmt] * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
    scale = torch.exp2(e)
    y = b / scale
    least, bits = (-6, 3) if fmt == "fp8" else (0, 1)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(1e-300))).clamp_min(least) - bits)
    return (torch.round(y / step) * step * scale).flatten(-2)


def exact(case, seed):
    """In 64 bits from the definitions; where a pass writes a pool whole, the pool."""
    s = prepare(case, seed)
    if case["op"] == "attend":
        if case["B"] * case["H"] * case["G"] * case["m"] * case["n"] > 5e9:
            return None
        return _exact_attend(s)
    if case["op"] == "read":
        K, V = (torch.stack([torch.stack([torch.stack([_exact_values(s, name, l, b, h, s["new"][b]) for h in range(case["H"])])
                                          for l in range(case["L"])]) for b in range(case["B"])]) for name in "KV")
        return [_exact_turn(s, K, True) if case["rotary"] else K, V]
    K, V = s["rows_K"].double(), s["rows_V"].double()
    if case["rotary"]:
        K = _exact_turn(s, K, False)
    if case["fmt"] not in TYPE:
        return [_exact_round(x, case["fmt"]) for x in (K, V)]
    got = []
    for name, x in (("K", K), ("V", V)):
        pool = s[name].double()
        for b in range(case["B"]):
            page = s["table"][b].long()[s["new"][b] // case["T"]]
            pool[page, :, :, s["new"][b] % case["T"]] = x[b].permute(2, 0, 1, 3)
        got.append(pool)
    return got
