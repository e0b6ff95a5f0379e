"""A step of new tokens over a paged cache, attention over chosen blocks of it, and its
pages' copying and compaction, as timed cases.

A pool holds pages of `T` rows of every layer and KV head, [P, L, H, T, D], in
bf16, fp32, or as 8- or 4-bit elements (e4m3, e2m1) with one power-of-two scale
for each 32 elements of a row. Row j of stream b lies in page table[b][j // T],
slot j % T. A block is `R` consecutive rows of a page; its bounds are the lowest
and the highest stored key element of each channel, [P, L, H, T / R, 2, D].
Four operators:

  qkv      new tokens of one layer: queries and keys normed for each head and
           turned to their position, queries returned, keys and values written
           into the pages, the bounds of the blocks written to brought up to date
  blocks   for each query the `top` blocks whose bounds allow the largest scores
           (the first and the last ones always among them), and attention over
           the rows of those
  compact  kept rows of every layer and head into new pages, keys turned from the
           position they had to the one they get, bounds made anew
  copy     pages onto other pages, or the first rows of them

Shapes are those of the repository's workloads (7B- and 72B-class video models
of 4 and 8 KV heads of 128, frames of 196 tokens, caches of 64 to 32768 rows)
and odd ones.
"""
import math
import random

import torch

own = False

BLOCK = 32                    # elements that share a scale
TOP = {"fp8": 448.0, "fp4": 6.0}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6
# Keys of a compacted row are stored values turned anew: a block keeps its scale where its largest value, often the type's
# largest itself, grows by less than this (it is rounded back), so that turns of next to nothing cost nothing.
SLACK = 1 + 2.0**-16


def _case(name, op, fmt, B, L, H, D, T, n, **more):
    c = {"op": op, "fmt": fmt, "B": B, "L": L, "H": H, "D": D, "T": T, "n": n, "ragged": False}
    if op in ("qkv", "blocks"):
        c.update(G=1, m=1, token_major=False)
    if op == "qkv":
        c.update(norm=True, rotary=True, R=0, src="bf16")
    elif op == "blocks":
        c.update(R=T, top=8, first=1, last=1, lse=False)
    elif op == "compact":
        c.update(C=n, rotary=True, R=0)
    else:
        c.update(pages=1, rows=T, R=0)
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # ---- qkv: the last m of n rows are new
        # one token of 16 users, blocks kept for selection
        _case("qkv-token", "qkv", "bf16", 16, 1, 4, 128, 64, 6272, G=7, m=1, ragged=True, R=64, token_major=True),
        # the next frame of four streams, rows kept in eight bits and read back
        _case("qkv-frame-fp8", "qkv", "fp8", 4, 2, 4, 128, 64, 6272, G=7, m=196, ragged=True, R=64, token_major=True),
        # a long prompt of a 72B-class model
        _case("qkv-prompt", "qkv", "bf16", 1, 1, 8, 128, 128, 6272, G=8, m=6272, R=64, token_major=True),
        # ---- blocks
        # the smallest: one token over a short fp32 cache, latency alone
        _case("blocks-tiny-f32", "blocks", "f32", 1, 1, 2, 64, 16, 500, G=2, R=16, top=4),
        # one token over a 72B-class cache of one user
        _case("blocks-token", "blocks", "bf16", 1, 1, 8, 128, 128, 32768, G=8, R=64, top=32, last=2),
        # 16 users of a 7B-class model answered together, rows in eight bits
        _case("blocks-batch16-fp8", "blocks", "fp8", 16, 1, 4, 128, 64, 32768, G=7, R=64, top=48, last=2, ragged=True, lse=True),
        # a prompt after a long video, each of its tokens with blocks of its own: the largest
        _case("blocks-prompt", "blocks", "bf16", 1, 1, 8, 128, 128, 32768, G=8, m=1024, R=64, top=16, token_major=True),
        # a few tokens of three users, odd pages, four bits an element
        _case("blocks-odd-fp4", "blocks", "fp4", 3, 2, 2, 64, 96, 5001, G=5, m=6, R=48, top=9, ragged=True, lse=True),
        # ---- compact: C of n rows are kept
        # a 7B-class cache at its cap
        _case("compact-7b", "compact", "bf16", 1, 28, 4, 128, 64, 6272, C=3136, R=64),
        # eight streams in eight bits, read back
        _case("compact-streams-fp8", "compact", "fp8", 8, 4, 4, 128, 128, 3136, C=1568, ragged=True),
        # ---- copy
        # a fork's last page, filled in part, before it is written to
        _case("copy-page", "copy", "bf16", 1, 28, 4, 128, 64, 3136, pages=1, rows=37, R=64),
        # the pages of a compressed 7B-class cache for another conversation that will change all of them
        _case("copy-cache", "copy", "bf16", 1, 28, 4, 128, 64, 3136, pages=49),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Streams 1 to 16, 1 to 32768 rows, 1 to 6272 new tokens (half of the draws
    with queries are single tokens or few), 1 to 12 query heads a KV head, every
    head size and type, pages of 16 to 256 rows in blocks of 16 to the page, 1 to
    64 blocks a query; at most the largest listed case's rows looked at, and 1 GiB
    of rows written."""
    while True:
        op = rng.choice(("qkv", "blocks", "blocks", "compact", "copy"))
        fmt = rng.choice(("bf16", "bf16", "fp8", "fp4", "f32"))
        D = rng.choice((64, 128, 128, 256, 32))
        T = rng.choice((16, 64, 64, 128, 256, 16 * rng.randint(1, 15)))
        sizes = [r for r in range(16, T + 1, 16) if T % r == 0]
        H = rng.choice((1, 2, 4, 8))
        B = _log(rng, 1, 16)
        n = _log(rng, 1, 32768)
        c = dict(ragged=rng.random() < 0.6)
        if op in ("qkv", "blocks"):
            c.update(G=rng.choice((1, 2, 4, 7, 8, 12)), token_major=rng.random() < 0.5,
                     m=min(n, _log(rng, 1, 12) if rng.random() < 0.5 else _log(rng, 12, 6272)))
        if op == "qkv":
            c.update(norm=rng.random() < 0.7, rotary=rng.random() < 0.8, R=rng.choice([0] + sizes),
                     src=rng.choice(("bf16", "bf16", "f32")))
            L, size = rng.choice((1, 2)), B * c["m"] * H * (c["G"] + 2) * D
            if size > 1 << 27:
                continue
        elif op == "blocks":
            first, last = rng.choice((0, 1, 2)), rng.choice((0, 1, 2))
            c.update(R=rng.choice(sizes), top=max(first + last, _log(rng, 1, 64)), first=first, last=last, lse=rng.random() < 0.5)
            L = rng.choice((1, 2))
            if B * H * c["m"] * c["top"] * c["R"] * D > 1 << 30 or B * H * c["m"] * (n // c["R"] + 1) > 1 << 25:
                continue
        elif op == "compact":
            L = _log(rng, 1, 28)
            # (a value of four bits turned by next to nothing can lie on a border of its rounding, where either side is as near)
            c.update(C=min(n, _log(rng, 1, n)), rotary=fmt != "fp4" and rng.random() < 0.8, R=rng.choice([0] + sizes))
            if B * L * H * c["C"] * D > 1 << 26:
                continue
        else:
            fmt = rng.choice(("bf16", "f32"))
            L, pages = _log(rng, 1, 28), _log(rng, 1, 64)
            c.update(pages=pages, rows=rng.choice((T, T, rng.randint(1, T))), R=rng.choice([0] + sizes), ragged=False)
            B, n = 1, pages * T
            if pages * L * H * T * D > 1 << 27:
                continue
        if B * L * H * n * D > 1 << 29:
            continue
        return _case("", op, fmt, B, L, H, D, T, n, **c)


# ---------------------------------------------------------------- the 8- and 4-bit types, in plain operations
def _encode(x, fmt, slack=1.0):
    """x [..., D] fp32 -> the elements' values before the scale, and the scales' exponents [..., D / 32]."""
    b = x.unflatten(-1, (-1, BLOCK))
    mant, exp = torch.frexp(b.abs().amax(-1))
    # the smallest e with amax <= slack * TOP * 2^e: TOP is 0.875 * 2^9 and 0.75 * 2^3
    e = exp - (9 if fmt == "fp8" else 3) + (mant > slack * (0.875 if fmt == "fp8" else 0.75)).int()
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
    c = torch.bucketize(y.abs().contiguous(), grid).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    c = c.unflatten(-1, (-1, 2))
    return c[..., 0] | (c[..., 1] << 4)


def _unpack(b, fmt):
    if fmt == "fp8":
        return b.view(torch.float8_e4m3fn).float()
    grid = torch.tensor(GRID4 + tuple(-g for g in GRID4), device=b.device)
    return grid[torch.stack((b & 15, b >> 4), -1).flatten(-2).int()]


def _turn(x, angles, back=False):
    """Pairs (d, d + D / 2) of x [..., D] by angles [..., D / 2, 2] (or back)."""
    c, s = angles.unbind(-1)
    s = -s if back else s
    lo, hi = x.chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


# ---------------------------------------------------------------- inputs
def _counts(case, rng):
    """Rows of each stream: n, or between half of it and n."""
    least = max(case.get("m", 1), case.get("C", 1), (case["n"] + 1) // 2)
    return [rng.randint(least, case["n"]) if case["ragged"] and b else case["n"] for b in range(case["B"])]


def _fill(g, shape, spread):
    """Normal rows; keys have a few larger channels, values one log-normal scale a row."""
    x = torch.randn(shape, generator=g, device="cuda")
    if spread:
        return x.mul_(torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda")))
    return x.mul_(1 + 2 * (torch.rand(shape[-1], generator=g, device="cuda") > 0.95))


def _store(s, name, x):
    fmt = s["case"]["fmt"]
    if fmt in TYPE:
        s[name] = x.to(TYPE[fmt])
    else:
        y, e = _encode(x, fmt)
        s[name], s[name + "_scales"] = _pack(y, fmt), (e + 127).to(torch.uint8)


def _angles(rows, D):
    a = torch.arange(rows, device="cuda")[:, None] * torch.exp(-math.log(1e6) * torch.arange(D // 2, device="cuda") / (D // 2))
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _all_bounds(s):
    """Bounds of every block from all its rows, and of the streams' last blocks from the rows that they hold."""
    c = s["case"]
    T, R = c["T"], c["R"]
    K = s["K"].float() if c["fmt"] in TYPE else _decode(_unpack(s["K"], c["fmt"]), s["K_scales"].int() - 127)
    K = K.unflatten(3, (T // R, R))
    s["bounds"] = torch.stack((K.amin(4), K.amax(4)), 4).to(torch.float32 if c["fmt"] == "f32" else torch.bfloat16)
    for b, n in enumerate(s["n"]):
        page, j, held = int(s["table"][b, (n - 1) // T]), (n - 1) % T // R, (n - 1) % R + 1
        x = K[page, :, :, j, :held]
        s["bounds"][page, :, :, j] = torch.stack((x.amin(2), x.amax(2)), 2).to(s["bounds"].dtype)


def prepare(case, seed):
    """Pools with their pages in random order and a few unused, the page tables, the counts and what the call takes."""
    rng = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, B, L, H, D, T, n, fmt = (case[k] for k in ("op", "B", "L", "H", "D", "T", "n", "fmt"))
    counts = _counts(case, rng)
    cols = -(-n // T)
    new_cols = -(-case["C"] // T) if op == "compact" else case["pages"] if op == "copy" else 0
    pages = B * (cols + new_cols) + 2
    order = torch.randperm(pages, generator=g, device="cuda").int()
    s = {"case": case, "n": counts, "table": order[:B * cols].view(B, cols).contiguous()}
    K = _fill(g, (pages, L, H, T, D), False)
    if op == "blocks":  # rows next to each other are alike, as a frame's are
        K += torch.randn((pages, L, H, T // case["R"], 1, D), generator=g, device="cuda").expand(-1, -1, -1, -1, case["R"], -1).flatten(3, 4)
    _store(s, "K", K)
    del K
    _store(s, "V", _fill(g, (pages, L, H, T, D), True))
    if case["R"]:
        _all_bounds(s)
    if op in ("qkv", "blocks"):
        G, m = case["G"], case["m"]
        s["first"] = [c - m for c in counts]
        s["new"] = torch.tensor(s["first"], device="cuda")[:, None] + torch.arange(m, device="cuda")  # positions [B, m]
        kind = TYPE[case["src"]] if op == "qkv" else TYPE["f32"] if fmt == "f32" else TYPE["bf16"]
        heads = (H * G, H, H) if op == "qkv" else (H * G,)
        for name, h in zip("qkv", heads):  # as a projection leaves them: token by token, or head by head
            shape = (B, m, h, D) if case["token_major"] else (B, h, m, D)
            x = (1.5 * _fill(g, shape, name == "v")).to(kind)
            s[name] = x.transpose(1, 2) if case["token_major"] else x
    if op == "qkv" and case["norm"]:
        s["q_norm"], s["k_norm"] = (0.5 + torch.rand(D, generator=g, device="cuda") for _ in range(2))
    if case.get("rotary"):
        s["rotary"] = _angles(n, D)
    if op == "compact":
        C = case["C"]
        s["new_table"] = order[B * cols:B * (cols + new_cols)].view(B, new_cols).contiguous()
        order = torch.rand((B, L, H, n), generator=g, device="cuda")
        order.masked_fill_(torch.arange(n, device="cuda") >= torch.tensor(counts, device="cuda")[:, None, None, None], 2.0)
        s["keep"] = order.argsort(-1)[..., :C].sort(-1).values.int().contiguous()
    if op == "copy":
        s["src"], s["dst"] = order[:new_cols].contiguous(), order[B * cols:B * cols + new_cols].contiguous()
    return s


# ---------------------------------------------------------------- plain forms
def _value(s, name, *at):
    """The pool's rows at those indices, fp32."""
    fmt = s["case"]["fmt"]
    x = s[name][at]
    return x.float() if fmt in TYPE else _decode(_unpack(x, fmt), s[name + "_scales"][at].int() - 127)


def _put(s, name, x, *at, slack=1.0):
    fmt = s["case"]["fmt"]
    if fmt in TYPE:
        s[name][at] = x.to(TYPE[fmt])
    else:
        y, e = _encode(x, fmt, slack)
        s[name][at] = _pack(y, fmt)
        s[name + "_scales"][at] = (e + 127).to(torch.uint8)


def _normed(x, weight):
    """Products rounded one by one; the mean square in 64 bits, since rows are rounded to few bits next."""
    inv = torch.rsqrt(x.double().square().mean(-1, keepdim=True) + EPS).float()
    return x * inv * weight


def _bound(s, table, blocks, end, layers):
    """Bounds of blocks [B, N] of a range of layers from their rows before end [B], as they are stored."""
    c = s["case"]
    T, R = c["T"], c["R"]
    at = blocks[:, :, None] * R + torch.arange(R, device="cuda")  # [B, N, R]
    page, sub = table.long().gather(1, blocks * R // T), blocks * R % T // R
    held = (at < end[:, None, None])[..., None, None, None]
    x = _value(s, "K", page[:, :, None], layers, slice(None), at % T)  # [B, N, R, layers, H, D]
    lo, hi = torch.where(held, x, math.inf).amin(2), torch.where(held, x, -math.inf).amax(2)
    s["bounds"][page, layers, :, sub] = torch.stack((lo, hi), -2).to(s["bounds"].dtype)


def _qkv(s):
    c, at, layer = s["case"], s["new"], s["case"]["L"] - 1
    q, k, v = (s[name].float() for name in "qkv")
    if c["norm"]:
        q, k = _normed(q, s["q_norm"]), _normed(k, s["k_norm"])
    if c["rotary"]:
        angles = s["rotary"][at][:, None]
        q, k = _turn(q, angles), _turn(k, angles)
    page, slot = s["table"].long().gather(1, at // c["T"]), at % c["T"]
    for name, x in (("K", k), ("V", v)):
        _put(s, name, x.transpose(1, 2), page, layer, slice(None), slot)
    out = [q.to(TYPE["f32" if c["fmt"] == "f32" else "bf16"])]
    if c["R"]:
        R, end = c["R"], at[:, -1] + 1
        first, last = at[:, 0] // R, at[:, -1] // R
        count = (c["m"] + R - 2) // R + 1  # blocks that so many rows can touch
        blocks = torch.minimum(first[:, None] + torch.arange(count, device="cuda"), last[:, None])
        _bound(s, s["table"], blocks, end, slice(layer, layer + 1))
        out.append(s["bounds"])
    if c["fmt"] in TYPE:
        return out + [s["K"], s["V"]]
    return out + [_value(s, name, page, layer, slice(None), slot).transpose(1, 2).to(torch.bfloat16) for name in "KV"]


def _select(s):
    c, at, layer = s["case"], s["new"], s["case"]["L"] - 1
    B, H, G, D, T, m, R, top = (c[k] for k in ("B", "H", "G", "D", "T", "m", "R", "top"))
    j = torch.arange(-(-max(s["n"]) // R), device="cuda")
    bounds = s["bounds"][s["table"].long()[:, j * R // T], layer, :, j * R % T // R].double()  # [B, N, H, 2, D]
    lo, hi = bounds.permute(3, 0, 2, 4, 1).contiguous()  # [B, H, D, N] each
    q = s["q"].double().reshape(B, H, G, m, D)
    score = torch.matmul(q.clamp_min(0).sum(2), hi) + torch.matmul(q.clamp_max(0).sum(2), lo)  # [B, H, m, N]
    held = torch.minimum(at + 1, torch.tensor(s["n"], device="cuda")[:, None])
    count = ((held + R - 1) // R)[:, None, :, None]  # blocks that a query sees
    score = torch.where((j < c["first"]) | (j >= count - c["last"]), math.inf, score)
    score = torch.where(j < count, score, -math.inf)
    picked = score.sort(dim=-1, descending=True, stable=True).indices[..., :top]
    if len(j) < top:
        picked = torch.nn.functional.pad(picked, (0, top - len(j)), value=len(j))
    picked = torch.where(picked < count, picked, len(j)).sort(-1).values
    return torch.where(picked < len(j), picked, -1).int()


def _blocks(s):
    c, layer = s["case"], s["case"]["L"] - 1
    B, H, G, D, T, m, R = (c[k] for k in ("B", "H", "G", "D", "T", "m", "R"))
    blocks = _select(s)
    at = (blocks.long()[..., None] * R + torch.arange(R, device="cuda")).flatten(-2)  # [B, H, m, top * R]
    held = torch.minimum(s["new"] + 1, torch.tensor(s["n"], device="cuda")[:, None])[:, None, :, None]
    seen = (at >= 0) & (at < held)
    at = torch.where(seen, at, 0)
    page = s["table"].long().gather(1, (at // T).flatten(1)).view(at.shape)
    h = torch.arange(H, device="cuda")[:, None, None]
    q = s["q"].float().reshape(B, H, G, m, D).permute(0, 1, 3, 4, 2).contiguous()  # [B, H, m, D, G]
    x = torch.matmul(_value(s, "K", page, layer, h, at % T), q).mul_(1 / math.sqrt(D))  # [B, H, m, rows, G]
    x.masked_fill_(~seen[..., None], -math.inf)
    most = x.amax(-2, keepdim=True)
    shift = torch.where(most == -math.inf, 0.0, most)
    x.sub_(shift).exp_()
    total = x.sum(-2, keepdim=True)
    out = torch.matmul(x.transpose(-1, -2).contiguous(), _value(s, "V", page, layer, h, at % T))  # [B, H, m, G, D]
    out = out / torch.where(total == 0, 1.0, total).transpose(-1, -2)
    out = out.transpose(2, 3).reshape(B, H * G, m, D).to(s["q"].dtype)
    lse = (shift + total.log()).squeeze(-2).transpose(2, 3).reshape(B, H * G, m)
    return [blocks, out, lse] if c["lse"] else [blocks, out]


def _compact(s):
    c = s["case"]
    B, L, H, T, C = (c[k] for k in ("B", "L", "H", "T", "C"))
    keep = s["keep"].long()
    page = s["table"].long().gather(1, (keep // T).flatten(1)).view(keep.shape)
    l, h = torch.arange(L, device="cuda")[:, None, None], torch.arange(H, device="cuda")[:, None]
    to = torch.arange(C, device="cuda")
    new = s["new_table"].long()[:, to // T][:, None, None]  # pages [B, 1, 1, C]
    K, V = (_value(s, name, page, l, h, keep % T) for name in "KV")
    if c["rotary"]:  # (a row that stays where it is stays as it is)
        K = torch.where((keep == to)[..., None], K, _turn(_turn(K, s["rotary"][keep], back=True), s["rotary"][to]))
    for name, x in (("K", K), ("V", V)):
        _put(s, name, x, new, l, h, to % T, slack=SLACK)
    out = []
    if c["R"]:
        blocks = torch.arange(-(-C // c["R"]), device="cuda").expand(B, -1)
        _bound(s, s["new_table"], blocks, torch.full((B,), C, device="cuda"), slice(None))
        out.append(s["bounds"])
    if c["fmt"] in TYPE:
        return out + [s["K"], s["V"]]
    return out + [_value(s, name, new, l, h, to % T).to(torch.bfloat16) for name in "KV"]


def _copy(s):
    c, src, dst = s["case"], s["src"].long(), s["dst"].long()
    for name in "KV":
        s[name][dst, :, :, :c["rows"]] = s[name][src, :, :, :c["rows"]]
    if not c["R"]:
        return [s["K"], s["V"]]
    blocks = -(-c["rows"] // c["R"])
    s["bounds"][dst, :, :, :blocks] = s["bounds"][src, :, :, :blocks]
    return [s["bounds"], s["K"], s["V"]]


# ---------------------------------------------------------------- the framework's
def _handles(s):
    """What a program makes once: the pool's handle, its bounds, the workspace, the outputs."""
    from paper_2506_15745_amd import ipv

    c = s["case"]
    s["ipv"] = ipv
    s["pool"] = ipv.PagePool(s["K"], s["V"], s.get("K_scales"), s.get("V_scales"))
    s["handle"] = ipv.BlockBounds(s["pool"], c["R"], s["bounds"]) if c["R"] else None
    if c["op"] == "blocks":
        s["ws"] = ipv.alloc_blocks_workspace(s["handle"], c["B"], c["H"] * c["G"], c["m"], c["top"], c["n"])
        s["out"] = torch.empty_like(s["q"])
        s["picked"] = torch.empty((c["B"], c["H"], c["m"], c["top"]), dtype=torch.int32, device="cuda")
        s["lse"] = torch.empty(s["q"].shape[:3], device="cuda") if c["lse"] else None
        return
    s["ws"] = ipv.alloc_page_workspace("cuda")
    if c["op"] == "qkv":
        s["out"] = torch.empty_like(s["q"], dtype=s["pool"].dtype)
    if c["fmt"] not in TYPE and c["op"] != "copy":
        rows = (c["B"], 1, c["H"], c["m"], c["D"]) if c["op"] == "qkv" else (c["B"], c["L"], c["H"], c["C"], c["D"])
        s["back"] = [torch.empty(rows, dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def _own(s):
    if "ipv" not in s:
        _handles(s)
    ipv, c, layer = s["ipv"], s["case"], s["case"]["L"] - 1
    if c["op"] == "blocks":
        ipv.ipv_attend_blocks(s["pool"], s["table"], s["n"], s["first"], layer, s["q"], s["picked"], s["out"], s["ws"],
                              bounds=s["handle"], first_blocks=c["first"], last_blocks=c["last"], lse=s["lse"])
        return [s["picked"], s["out"], s["lse"]] if c["lse"] else [s["picked"], s["out"]]
    if c["op"] == "copy":
        ipv.ipv_page_copy(s["pool"], s["src"], s["dst"], s["ws"], rows=c["rows"], bounds=s["handle"])
        return [s["bounds"], s["K"], s["V"]] if c["R"] else [s["K"], s["V"]]
    if c["op"] == "qkv":
        ipv.ipv_qkv_write(s["pool"], s["table"], s["first"], layer, s["q"], s["k"], s["v"], s["out"], s["ws"], q_norm=s.get("q_norm"),
                          k_norm=s.get("k_norm"), eps=EPS, rotary=s.get("rotary"), bounds=s["handle"])
        out = [s["out"], s["bounds"]] if c["R"] else [s["out"]]
        if c["fmt"] in TYPE:
            return out + [s["K"], s["V"]]
        ipv.ipv_page_read(s["pool"], s["table"], s["first"], *s["back"], s["ws"], first_layer=layer)
        return out + [x[:, 0] for x in s["back"]]
    ipv.ipv_page_compact(s["pool"], s["table"], s["new_table"], s["n"], s["keep"], s["ws"], rotary=s.get("rotary"), bounds=s["handle"])
    out = [s["bounds"]] if c["R"] else []
    if c["fmt"] in TYPE:
        return out + [s["K"], s["V"]]
    ipv.ipv_page_read(s["pool"], s["new_table"], 0, *s["back"], s["ws"])
    return out + s["back"]


def run(state):
    if own:
        return _own(state)
    return {"qkv": _qkv, "blocks": _blocks, "compact": _compact, "copy": _copy}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, B, L, H, D, n, R = (case[k] for k in ("op", "B", "L", "H", "D", "n", "R"))
    row = {"bf16": 2 * D, "f32": 4 * D, "fp8": D + D // BLOCK, "fp4": D // 2 + D // BLOCK}[case["fmt"]]
    wide = 4 if case["fmt"] == "f32" else 2  # bytes of a query's, an output's or a bound's element
    back = 0 if case["fmt"] in TYPE else 2 * (row + 2 * D)  # a row of K and of V read back as bf16
    # ragged streams hold between half of n rows and n: three quarters on average, the first one n
    least = max(case.get("m", 1), n * 3 // 4) if case["ragged"] else n
    counts = [n] + [least] * (B - 1)
    if op == "qkv":
        G, m, src = case["G"], case["m"], TYPE[case["src"]].itemsize
        bytes_ = B * m * H * (G * D * (src + wide) + 2 * (D * src + row) + back) + (B * m * D * 4 if case["rotary"] else 0)
        if R:  # each block written to: its bounds, and the rows that it held (half of one a stream)
            bytes_ += B * H * (2 * D * wide * (m // R + 1) + R // 2 * row)
        return {"bytes": bytes_, "flops": B * m * H * (G + 1) * D * ((4 if case["norm"] else 0) + (3 if case["rotary"] else 0)) + 1}
    if op == "blocks":
        G, m, top = case["G"], case["m"], case["top"]
        bytes_ = flops = 0
        for c in counts:
            seen = min(top * R, c)  # rows a query looks at; all queries together see at most the cache
            blocks = -(-c // R)
            bytes_ += H * (2 * row * min(c, m * seen) + 2 * D * wide * blocks) + H * G * m * (2 * D * wide + (4 if case["lse"] else 0)) + 4 * H * m * top
            flops += H * m * (4 * D * G * seen + 4 * D * blocks)
        return {"bytes": bytes_, "flops": flops}
    if op == "compact":
        rows = B * L * H * case["C"]
        bounds = B * L * H * 2 * D * wide * -(-case["C"] // R) if R else 0
        return {"bytes": rows * (4 * row + 4 + back) + bounds + (n * D * 4 if case["rotary"] else 0),
                "flops": rows * D * (6 if case["rotary"] else 1)}
    rows = case["pages"] * L * H * case["rows"]
    bounds = case["pages"] * L * H * 4 * D * wide * -(-case["rows"] // R) if R else 0
    return {"bytes": 4 * rows * row + bounds, "flops": rows}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _exact_values(s, name, *at):
    """The pool's rows at those indices in 64 bits: stored bits taken apart."""
    fmt = s["case"]["fmt"]
    x = s[name][at]
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
    return y * torch.exp2(s[name + "_scales"][at].double() - 127).repeat_interleave(BLOCK, -1)


def _exact_round(x, fmt, slack=1.0):
    """Each element to the nearest of its block's values (ties to the even one)."""
    if fmt in TYPE:
        return x
    b = x.unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True) / slack
    e = torch.ceil(torch.log2(top / TOP[fmt])).clamp(-126, 127)
    e = torch.where(top > TOP[fmt] * torch.exp2(e), e + 1, e)
    e = torch.where(top <= TOP[fmt] * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
    scale = torch.exp2(e)
    y = b / scale
    least, bits = (-6, 3) if fmt == "fp8" else (0, 1)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(1e-300))).clamp_min(least) - bits)
    return ((torch.round(y / step) * step).clamp(-TOP[fmt], TOP[fmt]) * scale).flatten(-2)


def _exact_turn(x, angles):
    """Pairs (d, d + D/2) as complex numbers, times the unit numbers `angles`."""
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:]) * angles
    return torch.cat((z.real, z.imag), -1)


def _exact_bounds(s, table, first, end, layer, rows):
    """The bounds with those of the blocks of positions first[b] .. end[b] - 1 made anew; rows(b): all of stream b's keys [H, end[b], D]."""
    c, got = s["case"], s["bounds"].double()
    T, R = c["T"], c["R"]
    for b in range(c["B"]):
        K = rows(b)
        for j in range(first[b] // R, -(-end[b] // R)):
            x = K[:, j * R:min(end[b], j * R + R)]
            got[int(table[b, j * R // T]), layer, :, j * R % T // R] = torch.stack((x.amin(1), x.amax(1)), 1)
    return got


def _exact_qkv(s):
    c, layer, fmt = s["case"], s["case"]["L"] - 1, s["case"]["fmt"]
    x = {name: s[name].double() for name in "qkv"}
    for name in "qk":
        if c["norm"]:
            rms = torch.sqrt((x[name] ** 2).sum(-1, keepdim=True) / c["D"] + EPS)
            x[name] = x[name] / rms * s[name + "_norm"].double()
        if c["rotary"]:
            x[name] = _exact_turn(x[name], torch.view_as_complex(s["rotary"].double())[s["new"]][:, None])
    k, v = _exact_round(x["k"], fmt), _exact_round(x["v"], fmt)
    out = [x["q"]]
    if c["R"]:
        def rows(b):
            j = torch.arange(s["first"][b], device="cuda")
            old = _exact_values(s, "K", s["table"][b].long()[j // c["T"]], layer, slice(None), j % c["T"])  # [rows, H, D]
            return torch.cat((old.transpose(0, 1), k[b]), 1)
        out.append(_exact_bounds(s, s["table"], s["first"], s["n"], layer, rows))
    if fmt not in TYPE:
        return out + [k, v]
    for name, y in (("K", k), ("V", v)):
        pool = s[name].double()
        for b in range(c["B"]):
            pool[s["table"][b].long()[s["new"][b] // c["T"]], layer, :, s["new"][b] % c["T"]] = y[b].transpose(0, 1)
        out.append(pool)
    return out


def _exact_blocks(s):
    c, layer = s["case"], s["case"]["L"] - 1
    B, H, G, D, T, m, R, top = (c[k] for k in ("B", "H", "G", "D", "T", "m", "R", "top"))
    out = torch.zeros(B, H * G, m, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, H * G, m, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = s["n"][b]
        j = torch.arange(n, device="cuda")
        starts = torch.arange(0, n, R, device="cuda")
        bounds = s["bounds"][s["table"][b].long()[starts // T], layer, :, starts % T // R].double()  # [N, H, 2, D]
        p = s["new"][b][:, None]
        visible = starts <= p  # [m, N]
        count = visible.sum(-1, keepdim=True)
        index = torch.arange(len(starts), device="cuda")
        always = (index < c["first"]) | (index >= count - c["last"])
        for h in range(H):
            q = s["q"][b, h * G:h * G + G].double()  # [G, m, D]
            best = sum(torch.where(x > 0, x, 0) @ bounds[:, h, 1].T + torch.where(x < 0, x, 0) @ bounds[:, h, 0].T for x in q)
            best = best.masked_fill(always, math.inf).masked_fill(~visible, -math.inf)
            rank = best.argsort(dim=-1, descending=True, stable=True).argsort(-1)  # a block's place among them
            chosen = (rank < top) & visible
            seen = chosen.repeat_interleave(R, -1)[:, :n] & (j <= p)
            K, V = (_exact_values(s, name, s["table"][b].long()[j // T], layer, h, j % T) for name in "KV")
            for a in range(G):
                x = (q[a] @ K.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                some = seen.any(-1)
                lse[b, h * G + a] = torch.logsumexp(x, -1)
                out[b, h * G + a] = torch.where(some[:, None], torch.softmax(x, -1), 0) @ V
    return [None, out, lse] if c["lse"] else [None, out]


def _exact_compact(s):
    c, fmt = s["case"], s["case"]["fmt"]
    B, L, H, T, C = (c[k] for k in ("B", "L", "H", "T", "C"))
    got = {}
    for name in "KV":
        rows = []
        for b in range(B):
            at = s["keep"][b].long()  # [L, H, C]
            x = torch.stack([torch.stack([_exact_values(s, name, s["table"][b].long()[at[l, h] // T], l, h, at[l, h] % T)
                                          for h in range(H)]) for l in range(L)])
            if name == "K" and c["rotary"]:
                unit = torch.view_as_complex(s["rotary"].double())
                x = torch.where((at == torch.arange(C, device="cuda"))[..., None], x, _exact_turn(x, unit[:C] * unit[at].conj()))
            rows.append(_exact_round(x, fmt, SLACK))
        got[name] = torch.stack(rows)
    out = []
    if c["R"]:
        bounds = s["bounds"]
        for l in range(L):
            bounds = _exact_bounds(dict(s, bounds=bounds), s["new_table"], [0] * B, [C] * B, l, lambda b: got["K"][b, l])
        out.append(bounds)
    if fmt not in TYPE:
        return out + [got["K"], got["V"]]
    to = torch.arange(C, device="cuda")
    for name in "KV":
        pool = s[name].double()
        for b in range(B):
            pool[s["new_table"][b].long()[to // T], :, :, to % T] = got[name][b].permute(2, 0, 1, 3)
        out.append(pool)
    return out


def _exact_copy(s):
    c = s["case"]
    got = {name: s[name].double() for name in ("bounds", "K", "V") if name in s}
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        for name, x in got.items():
            held = c["rows"] if name != "bounds" else -(-c["rows"] // c["R"])
            x[b, :, :, :held] = s[name][a, :, :, :held].double()
    return list(got.values())


def exact(case, seed):
    """In 64 bits from the definitions; where a pass writes a pool whole, the pool."""
    s = prepare(case, seed)
    if case["op"] == "blocks" and case["B"] * case["H"] * case["G"] * case["m"] * case["n"] > 5e9:
        return None
    return {"qkv": _exact_qkv, "blocks": _exact_blocks, "compact": _exact_compact, "copy": _exact_copy}[case["op"]](s)
