"""The operators around the attention of a served or trained rank, as timed cases: rotary positions (forward and backward),
block tables and slot maps of a paged cache, K and V written to that cache in 8 bits, and attention over it.

A case is one call of one operator.  A serving step makes one of each: `usp_cache_extend` (pages for the tokens that come),
`usp_rope_rows` (their Q and K), `usp_cache_append` (K and V into the pages), `usp_cache_attn` (Q against what is cached).  A
training step has `usp_rope_shards` before `usp_attn_fwd` and, as its gradient, after `usp_attn_bwd`.

The cache: pages of `page` tokens, codes of 8 bits (e4m3), one exponent byte x for each page, KV head and tensor; a value is
code * 2^(x - 127).  K codes lie as [pages][hk][page][hs], V codes as [pages][hk][page / 16][hs][16].
"""
import math
import random

import torch

own = False

_F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    heads = {"hq": 32, "hk": 8, "hs": 128}     # what the benchmark's configurations share
    return [
        # the new tokens of eight requests that answer, as slices of one QKV product: latency is all there is
        dict(name="rope_decode_8", kind="rope_rows", rows=8, far=32768, **heads, dtype="bf16", pairs=False, rotary=128,
             scaling="none", backward=False, strided=True),
        # one rank's shard of the training configuration, L = 65536 on Ulysses 2 x ring 4
        dict(name="rope_train_L65536_u2r4", kind="rope_shards", bs=1, L=65536, U=2, R=4, rank=1, zigzag=True, **heads,
             dtype="bf16", pairs=False, rotary=128, scaling="parts", backward=False),
        # gradients in single precision, interleaved pairs in half of a smaller head, both halves of a batch
        dict(name="rope_grad_fp32_pairs_hs64", kind="rope_shards", bs=2, L=32768, U=4, R=2, rank=5, zigzag=False, hq=32, hk=8,
             hs=64, dtype="fp32", pairs=True, rotary=32, scaling="base", backward=True),
        # one token for each of 256 requests
        dict(name="extend_decode_256", kind="extend", n=256, page=64, len_lo=1, len_hi=32768, new_lo=1, new_hi=1, ragged=1),
        # prompts and pieces of prompts of 48 requests
        dict(name="extend_prompts_48", kind="extend", n=48, page=16, len_lo=1, len_hi=8192, new_lo=64, new_hi=8192, ragged=2),
        # K and V of one token for each of 64 requests, most of them inside a page that holds tokens already
        dict(name="append_decode_64", kind="append", n=64, page=64, len_lo=1, len_hi=4096, new_lo=1, new_hi=1, ragged=3, **heads,
             dtype="bf16", strided=True),
        # K and V of ragged prompts, some of which begin inside a page
        dict(name="append_prompts_12", kind="append", n=12, page=64, len_lo=1, len_hi=1024, new_lo=512, new_hi=8192, ragged=4,
             **heads, dtype="bf16", strided=True),
        # one request's next token after a short prompt
        dict(name="attend_one_1003", kind="attend", n=1, page=64, len_lo=1003, len_hi=1003, new_lo=1, new_hi=1, ragged=5, **heads,
             causal=True, held=1),
        # the next tokens of a ragged batch
        dict(name="attend_batch_64", kind="attend", n=64, page=64, len_lo=256, len_hi=32768, new_lo=1, new_hi=1, ragged=6, **heads,
             causal=True, held=1),
        # the next token after the benchmark's longest prompt
        dict(name="attend_long_212992", kind="attend", n=1, page=64, len_lo=212993, len_hi=212993, new_lo=1, new_hi=1, ragged=7,
             **heads, causal=True, held=1),
        # a piece of a long prompt against what came before it and itself
        dict(name="attend_chunk_4096", kind="attend", n=1, page=64, len_lo=49152, len_hi=49152, new_lo=4096, new_hi=4096, ragged=8,
             **heads, causal=True, held=1),
        # cross attention: a few tokens of each of 20 requests against an encoder's states of other, odd lengths
        dict(name="attend_cross_hs64", kind="attend", n=20, page=16, len_lo=301, len_hi=6007, new_lo=1, new_hi=9, ragged=9, hq=16,
             hk=16, hs=64, causal=False, held=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["rope_rows", "rope_shards", "extend", "append", "attend"], [12, 12, 14, 20, 42])[0]
    hs = rng.choice([128, 128, 64])
    hq, hk = rng.choice([(32, 8), (32, 8), (32, 32), (16, 8), (32, 1), (12, 4), (4, 4)])
    page = rng.choice([16, 32, 64, 64, 128])
    rope = dict(hq=hq, hk=hk, hs=hs, dtype=rng.choice(["bf16", "bf16", "fp32"]), pairs=rng.random() < 0.5,
                rotary=rng.choice([hs, hs, hs // 2, hs // 4, hs - 16]), scaling=rng.choice(["none", "linear", "base", "parts"]),
                backward=rng.random() < 0.4)
    if kind == "rope_rows":
        return dict(kind=kind, rows=_log(rng, 1, 32768), far=_log(rng, 64, 1 << 21), strided=rng.random() < 0.5, **rope)
    if kind == "rope_shards":
        if hk < 8:
            hq, hk = 32, 8
        U, R = rng.choice([(8, 1), (4, 2), (2, 4), (1, 8), (8, 2), (2, 2), (1, 1)])
        rope.update(hq=hq, hk=hk)
        unit = 2 * U * R
        L = max(unit, _log(rng, 256, 65536) // unit * unit)
        return dict(kind=kind, bs=rng.choice([1, 1, 2]), L=L, U=U, R=R, rank=rng.randrange(U * R), zigzag=rng.random() < 0.7, **rope)
    while True:
        n = _log(rng, 1, 256)
        case = dict(kind=kind, n=n, page=page, len_lo=1, len_hi=_log(rng, 16, 65536), new_lo=1, new_hi=1,
                    ragged=rng.randrange(1 << 20))
        if kind != "attend":
            if rng.random() < 0.6:
                case["new_hi"] = _log(rng, 2, 8192)
            if kind == "append":
                case.update(hq=hq, hk=hk, hs=hs, dtype=rng.choice(["bf16", "bf16", "fp32"]), strided=rng.random() < 0.6)
            _, new = _lengths(case)
            if sum(new) <= 40000 and (kind == "extend" or _pages(case) * page * hk * hs <= 5e8):
                return case
            continue
        case["len_hi"] = _log(rng, 64, 212993)
        if rng.random() < 0.5:
            case["new_hi"] = _log(rng, 2, 4096)
        case.update(hq=hq, hk=hk, hs=hs, causal=rng.random() < 0.75, held=rng.choice([1, 1, 1, 2]))
        before, new = _lengths(case)
        longest, most = max(b + m for b, m in zip(before, new)), max(new)
        if work(case)["flops"] <= 3e12 and n * longest * hk * hs <= 2.2e9 and n * most * hq * longest <= 6.5e9:
            return case


def _lengths(case):
    """(tokens that each request holds before, tokens that come), from the case alone.  `attend`: len_* are lengths in all."""
    rng = random.Random(case["ragged"])
    held = [_log(rng, case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    new = [_log(rng, case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    held[rng.randrange(case["n"])] = case["len_hi"]
    if case["kind"] == "attend":
        held = [max(0, h - m) for h, m in zip(held, new)]
    return held, new


def _pages(case):
    """Pages that the requests hold in the end."""
    return sum(-(-(h + m) // case["page"]) for h, m in zip(*_lengths(case)))


def _pairs(case):
    held, new = _lengths(case)
    if case["causal"]:
        return sum(m * h + m * (m + 1) // 2 for h, m in zip(held, new))
    return sum(m * (h + m) for h, m in zip(held, new))


def work(case):
    kind, es = case["kind"], 4 if case.get("dtype") == "fp32" else 2
    if kind in ("rope_rows", "rope_shards"):
        rows = case["rows"] if kind == "rope_rows" else case["bs"] * case["L"] // (case["U"] * case["R"])
        heads = case["hq"] + case["hk"]
        return {"bytes": 2 * rows * heads * case["hs"] * es + 4 * rows, "flops": 3 * rows * heads * case["rotary"]}
    held, new = _lengths(case)
    if kind == "extend":
        taken = sum(-(-(h + m) // case["page"]) - -(-h // case["page"]) for h, m in zip(held, new))
        return {"bytes": 4 * (3 * case["n"] + 2 * sum(new) + 2 * taken), "flops": 0}
    if kind == "append":
        values = 2 * sum(new) * case["hk"] * case["hs"]
        return {"bytes": values * (es + 1) + 4 * sum(new), "flops": 2 * values}
    tokens = sum(h + m for h, m in zip(held, new))
    cached = 2 * (tokens // case["held"]) * case["hk"] * (case["hs"] + 1 / case["page"])
    rows = sum(new) * case["hq"]
    return {"bytes": cached + 4 * rows * case["hs"] + 4 * rows + 4 * _pages(case), "flops": 4 * case["hs"] * case["hq"] * _pairs(case) / case["held"]}


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------------
_SCALED = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
           "parts": {"factor": 8.0, "alpha": 1.0, "beta": 32.0, "original_len": 8192, "magnitude": 0.1 * math.log(8.0) + 1.0}}
_BASE = 500000.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float32 if case.get("dtype") == "fp32" else torch.bfloat16
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if kind == "rope_rows":
        rows, hq, hk, hs = case["rows"], case["hq"], case["hk"], case["hs"]
        s["positions"] = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        if case["strided"]:                 # Q and K where a QKV product leaves them
            qkv = normal(rows, hq + 2 * hk, hs)
            s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        else:
            s["q"], s["k"] = normal(rows, hq, hs), normal(rows, hk, hs)
        s["q_out"], s["k_out"] = (torch.empty(rows, h, hs, device="cuda", dtype=dtype) for h in (hq, hk))
        return s
    if kind == "rope_shards":
        N = case["U"] * case["R"]
        shape = N, case["bs"], case["L"] // N
        for name, h in (("q", case["hq"]), ("k", case["hk"])):
            s[name] = torch.zeros(*shape, h, case["hs"], device="cuda", dtype=dtype)     # all shards, the rank's own filled
            s[name][case["rank"]] = normal(case["bs"], case["L"] // N, h, case["hs"])
            s[name + "_out"] = torch.empty_like(s[name])
        return s

    held, new = _lengths(case)
    page, n = case["page"], case["n"]
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    most = max(-(-(h + m) // page) for h, m in zip(held, new)) + 1          # pages in a row of the table
    before = [-(-h // page) for h in held]
    after = [-(-(h + m) // page) for h, m in zip(held, new)]
    spare = 5
    pages = sum(after) + spare
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    index = torch.arange(most, device="cuda").expand(n, most)

    def table_of(counts):
        """A table whose rows hold the next counts[i] pages of `order`, and -1 behind them."""
        first = torch.tensor([0] + counts[:-1], device="cuda").cumsum(0)[:, None]
        c = torch.tensor(counts, device="cuda")[:, None]
        return torch.where(index < c, order[(first + index).clamp_max(pages - 1)], -1).to(torch.int32).contiguous()

    s.update(cu=ints(cu), total=cu[-1], pages=pages, max_pages=most)
    if kind == "extend":
        s["len_before"], s["table"] = ints(held), table_of(before)
        s["free"] = order[sum(before):].contiguous()
        s["len_after"], s["taken"] = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        s["slots"], s["positions"] = (torch.empty(cu[-1], dtype=torch.int32, device="cuda") for _ in range(2))
        return s

    hk, hs = case["hk"], case["hs"]
    # a cache in use: values about N(0, 1), of which 448 * 2^-6 = 7 is beyond the largest
    s["k_codes"] = torch.empty(pages, hk, page, hs, dtype=_F8, device="cuda")
    s["v_codes"] = torch.empty(pages, hk, page // 16, hs, 16, dtype=_F8, device="cuda")
    for name in ("k_codes", "v_codes"):
        flat = s[name].view(pages, -1)
        for at in range(0, pages, 8192):
            part = flat[at:at + 8192]
            part.copy_((torch.randn(part.shape, generator=gen, device="cuda") * 64).clamp_(-448, 448))
    s["k_scale"], s["v_scale"] = (torch.randint(120, 122, (pages, hk), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2))
    if kind == "append":
        table = table_of(after)
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(new, device="cuda"), output_size=cu[-1])
        pos = ints(held)[seq] + torch.arange(cu[-1], device="cuda") - ints(cu)[seq]
        s["slots"] = (table[seq, pos // page] * page + pos % page).to(torch.int32)
        s["runs"] = sum((h + m - 1) // page - h // page + 1 for h, m in zip(held, new))     # pages that are written
        rows, hq = cu[-1], case["hq"]
        if case["strided"]:
            qkv = normal(rows, hq + 2 * hk, hs)
            s["k"], s["v"] = qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        else:
            s["k"], s["v"] = normal(rows, hk, hs), normal(rows, hk, hs)
        return s
    s["len"] = ints([h + m for h, m in zip(held, new)])
    s["table"] = table_of(after)
    if case["held"] > 1:                    # the pages of one of `held` ranks that share the sequence
        s["table"] = torch.where(index % case["held"] == seed % case["held"], s["table"], -1).contiguous()
    s["most_new"], s["longest"] = max(new), max(h + m for h, m in zip(held, new))
    s["q"] = normal(cu[-1], case["hq"], hs)
    s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(case["hq"], cu[-1], device="cuda")
    s["workspace"] = torch.empty(96 << 20, dtype=torch.uint8, device="cuda")     # one for all calls of a program
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    return {"rope_rows": _plain_rope, "rope_shards": _plain_rope, "extend": _plain_extend, "append": _plain_append,
            "attend": _plain_attend}[s["case"]["kind"]](s)


def _own(s):
    import paper_2405_07719_amd as usp
    case = s["case"]
    kind, dtype = case["kind"], usp.USP_FP32 if case.get("dtype") == "fp32" else usp.USP_BF16
    if kind in ("rope_rows", "rope_shards"):
        if "rope" not in s:
            s["rope"] = usp.rope(case["hs"], case["rotary"], usp.USP_ROPE_PAIRS if case["pairs"] else usp.USP_ROPE_HALVES, _BASE,
                                 {"none": usp.USP_ROPE_UNSCALED, "linear": usp.USP_ROPE_LINEAR, "base": usp.USP_ROPE_BASE,
                                  "parts": usp.USP_ROPE_BY_PARTS}[case["scaling"]], **_SCALED[case["scaling"]])
    if kind == "rope_rows":
        usp.usp_rope_rows(s["rope"], s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], case["rows"], case["hq"], case["hk"],
                          case["hs"], s["q"].stride(0), s["k"].stride(0), s["q_out"].stride(0), s["k_out"].stride(0), dtype,
                          case["backward"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "rope_shards":
        if "p" not in s:
            s["p"] = usp.problem(case["bs"], case["L"], case["hq"], case["hk"], case["hs"], case["U"], case["R"], True,
                                 usp.USP_SPLIT_ZIGZAG if case["zigzag"] else usp.USP_SPLIT_CONTIG, dtype)
        rank = case["rank"]
        usp.usp_rope_shards(s["p"], s["rope"], s["q"], s["k"], s["q_out"], s["k_out"], case["backward"], rank, rank + 1)
        return {"q": s["q_out"][rank], "k": s["k_out"][rank]}
    if kind == "extend":
        usp.usp_cache_extend(s["cu"], s["len_before"], case["n"], s["total"], s["table"], s["max_pages"], case["page"], s["pages"],
                             s["free"], s["free"].numel(), s["len_after"], s["slots"], s["positions"], s["taken"])
        return {"table": s["table"], "len": s["len_after"], "slots": s["slots"], "positions": s["positions"], "taken": s["taken"]}
    if "cache" not in s:
        s["cache"] = usp.cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["pages"], case["page"], case["hk"], case["hs"])
    if kind == "append":
        usp.usp_cache_append(s["cache"], s["k"], s["v"], s["slots"], s["total"], s["k"].stride(0), s["v"].stride(0), dtype)
        return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    usp.usp_cache_attn(s["cache"], s["q"], s["q"].stride(0), s["cu"], s["len"], s["table"], s["max_pages"], case["n"], s["total"],
                       s["most_new"], case["hq"], 0.0, case["causal"], s["o"], s["lse"], usp.USP_BF16, s["workspace"])
    return {"o": s["o"], "lse": s["lse"]}


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _plain_rope(s):
    case = s["case"]
    d, hs, by = case["rotary"], case["hs"], _SCALED[case["scaling"]]
    j = torch.arange(d // 2, device="cuda", dtype=torch.float64)
    base = _BASE * (by["factor"] ** (d / (d - 2)) if case["scaling"] == "base" else 1.0)
    f = base ** (-2 * j / d)
    if case["scaling"] == "linear":
        f = f / by["factor"]
    if case["scaling"] == "parts":
        kept = ((by["original_len"] * f / (2 * math.pi) - by["alpha"]) / (by["beta"] - by["alpha"])).clamp(0, 1)
        f = kept * f + (1 - kept) * f / by["factor"]
    if case["kind"] == "rope_rows":
        pos, q, k = s["positions"].double(), s["q"], s["k"]
    else:
        U, R, n = case["U"], case["R"], case["L"] // (case["U"] * case["R"])
        r, u = divmod(case["rank"], U)
        i = u * n + torch.arange(n, device="cuda")
        if case["zigzag"]:
            c = case["L"] // (2 * R)
            pos = torch.where(i < c, r * c + i, (2 * R - 1 - r) * c + i - c).double()
        else:
            pos = (r * (case["L"] // R) + i).double()
        q, k = s["q"][case["rank"]], s["k"][case["rank"]]
    angle = pos[:, None] * f * (-1 if case["backward"] else 1)
    m = by.get("magnitude", 1.0)
    cos, sin = (angle.cos() * m).float()[:, None], (angle.sin() * m).float()[:, None]      # [rows, 1, d / 2]

    def turned(x):
        y = x.float()
        a, b = (y[..., 0:d:2], y[..., 1:d:2]) if case["pairs"] else (y[..., :d // 2], y[..., d // 2:d])
        a, b = a * cos - b * sin, a * sin + b * cos
        first = torch.stack([a, b], -1).flatten(-2) if case["pairs"] else torch.cat([a, b], -1)
        return torch.cat([first, y[..., d:]], -1).to(x.dtype)

    return {"q": turned(q), "k": turned(k)}


def _plain_extend(s):
    case = s["case"]
    page, cu, before, table, free = case["page"], s["cu"], s["len_before"], s["table"], s["free"]
    after = before + (cu[1:] - cu[:-1])
    had = (before + page - 1) // page
    need = (after + page - 1) // page - had
    end = need.cumsum(0, dtype=torch.int32)
    t = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(cu[1:], t, right=True)
    pos = before[seq] + t - cu[seq]
    at = pos // page
    fresh = at >= had[seq]
    number = torch.where(fresh, free[torch.where(fresh, (end - need)[seq] + at - had[seq], 0)], table[seq, at])
    table[seq, at] = number
    return {"table": table, "len": after, "slots": number * page + pos % page, "positions": pos, "taken": end[-1:].expand(2)}


def _plain_append(s):
    case = s["case"]
    page, hk, hs, slots, runs = case["page"], case["hk"], case["hs"], s["slots"].long(), s["runs"]
    number, place = slots // page, slots % page
    lead = torch.ones_like(number, dtype=torch.bool)
    lead[1:] = number[1:] != number[:-1]
    run = lead.cumsum(0) - 1                                          # which written page a row belongs to
    first = torch.argsort((~lead).to(torch.uint8), stable=True)[:runs]      # its first row
    written, old = number[first], place[first]                       # page number, tokens that it held
    kept = torch.arange(page, device="cuda") < old[:, None]          # [runs, page]

    def put(x, codes, scale):
        """`codes` as [pages, hk, page, hs] in bytes, a view or not; returns them and the scales."""
        x = x.float()
        most = torch.zeros(runs, hk, device="cuda").scatter_reduce_(0, run[:, None].expand(-1, hk), x.abs().amax(-1), "amax")
        part, power = torch.frexp(most)                              # most = part * 2^power, part in [0.5, 1)
        least = torch.where(most > 0, power - 9 + (part > 0.875), -117).clamp(-117, 119) + 127      # 448 = 0.875 * 2^9
        was = scale[written].int()
        now = torch.where(old[:, None] > 0, torch.maximum(was, least), least)
        held = codes[written].view(_F8).float() * torch.exp2((was - now).float())[:, :, None, None]
        codes[written] = torch.where(kept[:, None, :, None], held.to(_F8).view(torch.uint8), codes[written])
        codes[number, :, place] = (x * torch.exp2((127 - now).float())[run][:, :, None]).to(_F8).view(torch.uint8)
        scale[written] = now.to(torch.uint8)

    put(s["k"], s["k_codes"].view(torch.uint8), s["k_scale"])
    # V tiles [page / 16][hs][16] as rows: the pages that are written are laid out anew
    v = s["v_codes"].view(torch.uint8)
    rows = torch.empty(v.shape[0], hk, page, hs, dtype=torch.uint8, device="cuda")
    rows[written] = v[written].transpose(3, 4).reshape(runs, hk, page, hs)
    put(s["v"], rows, s["v_scale"])
    v[written] = rows[written].view(runs, hk, page // 16, 16, hs).transpose(3, 4)
    return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attend(s):
    case = s["case"]
    page, n, hq, hk, hs, m = case["page"], case["n"], case["hq"], case["hk"], case["hs"], s["most_new"]
    cu, length = s["cu"].long(), s["len"].long()
    table = s["table"][:, :-(-s["longest"] // page)].long()
    keys = table.shape[1] * page
    at = table.clamp_min(0)
    k = s["k_codes"].view(torch.uint8)[at].view(_F8).float() * torch.exp2(s["k_scale"][at].float() - 127)[..., None, None]
    v = s["v_codes"].view(torch.uint8)[at].view(_F8).float() * torch.exp2(s["v_scale"][at].float() - 127)[..., None, None, None]
    k = k.permute(0, 2, 1, 3, 4).reshape(n, hk, keys, hs)
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(n, hk, keys, hs)
    # queries padded to [n, hk, m * group, hs]
    i = torch.arange(m, device="cuda")
    new = cu[1:] - cu[:-1]
    q = s["q"].float()[(cu[:-1, None] + i).clamp_max(s["total"] - 1)]
    q = q.view(n, m, hk, hq // hk, hs).transpose(1, 2).reshape(n, hk, m * (hq // hk), hs)
    scores = torch.matmul(q, k.transpose(2, 3)) * hs ** -0.5
    j = torch.arange(keys, device="cuda")
    last = (length - new)[:, None] + i + 1 if case["causal"] else length[:, None].expand(-1, m)      # keys that a token sees
    seen = (j < last[:, :, None]) & (table >= 0).repeat_interleave(page, 1)[:, None]                 # [n, m, keys]
    scores.view(n, hk, m, -1, keys).masked_fill_(~seen[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = (total.log() + top).squeeze(-1)
    t = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(cu[1:], t, right=True)
    o = o.view(n, hk, m, -1, hs)[seq, :, t - cu[seq]].reshape(-1, hq, hs)
    lse = lse.view(n, hk, m, -1)[seq, :, t - cu[seq]].reshape(-1, hq).t().contiguous()
    return {"o": o.to(s["q"].dtype), "lse": lse}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope_rows": _exact_rope, "rope_shards": _exact_rope, "extend": _exact_extend, "append": _exact_append,
            "attend": _exact_attend}[case["kind"]](s)


def _exact_rope(s):
    """Each pair as a complex number times magnitude * e^(i position frequency), or its conjugate."""
    case = s["case"]
    d, by = case["rotary"], _SCALED[case["scaling"]]
    freq = []
    for j in range(d // 2):
        base = _BASE
        if case["scaling"] == "base":
            base *= by["factor"] ** (d / (d - 2))
        f = base ** (-2.0 * j / d)
        if case["scaling"] == "linear":
            f /= by["factor"]
        if case["scaling"] == "parts":
            turns = by["original_len"] * f / (2 * math.pi)
            g = min(1.0, max(0.0, (turns - by["alpha"]) / (by["beta"] - by["alpha"])))
            f = (1 - g) * f / by["factor"] + g * f
        freq.append(f)
    if case["kind"] == "rope_rows":
        pos, q, k = s["positions"].double(), s["q"], s["k"]
    else:
        N, rank = case["U"] * case["R"], case["rank"]
        if case["zigzag"]:          # the ring rank's chunks of the sequence, then the Ulysses rank's piece of them
            chunks = torch.arange(case["L"], device="cuda").view(2 * case["R"], -1)
            r = rank // case["U"]
            block = torch.cat([chunks[r], chunks[2 * case["R"] - 1 - r]])
        else:
            block = torch.arange(case["L"], device="cuda").view(case["R"], -1)[rank // case["U"]]
        pos = block.view(case["U"], -1)[rank % case["U"]].double()
        q, k = s["q"][rank], s["k"][rank]
    angle = pos[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    w = torch.polar(torch.full_like(angle, by.get("magnitude", 1.0)), -angle if case["backward"] else angle)[:, None]
    got = {}
    for name, x in (("q", q), ("k", k)):
        y = x.double().clone()
        if case["pairs"]:
            z = torch.complex(y[..., 0:d:2], y[..., 1:d:2]) * w
            y[..., 0:d:2], y[..., 1:d:2] = z.real, z.imag
        else:
            z = torch.complex(y[..., :d // 2], y[..., d // 2:d]) * w
            y[..., :d // 2], y[..., d // 2:d] = z.real, z.imag
        got[name] = y
    return got


def _exact_extend(s):
    """Whole numbers, one request after the other, on the host."""
    page, cu, held = s["case"]["page"], s["cu"].tolist(), s["len_before"].tolist()
    table, free = s["table"].tolist(), s["free"].tolist()
    used, slots, positions, after = 0, [], [], []
    for i, h in enumerate(held):
        for p in range(h, h + cu[i + 1] - cu[i]):
            if p % page == 0:
                table[i][p // page] = free[used]
                used += 1
            slots.append(table[i][p // page] * page + p % page)
            positions.append(p)
        after.append(h + cu[i + 1] - cu[i])
    whole = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return {"table": whole(table), "len": whole(after), "slots": whole(slots), "positions": whole(positions), "taken": whole([used, used])}


def _exact_append(s):
    """The codes' values and the exponent bytes that stand for: the smallest power of two that holds every value of the page
    and head within 448, not below what older tokens of the page have; rounding to the nearest of e4m3, ties to even."""
    page, slots = s["case"]["page"], s["slots"].tolist()
    starts = [t for t in range(len(slots)) if t == 0 or slots[t] // page != slots[t - 1] // page] + [len(slots)]

    def rounded(x):
        step = torch.exp2(torch.frexp(x.abs().clamp_min(2.0 ** -6)).exponent.double() - 4)
        return torch.round(x / step) * step

    got = {}
    for name in ("k", "v"):
        value = s[name + "_codes"].double()
        if name == "v":
            value = value.transpose(3, 4).reshape(value.shape[0], value.shape[1], page, -1).contiguous()
        scale = s[name + "_scale"].clone()
        x = s[name].double()
        for a, b in zip(starts, starts[1:]):
            number, old = slots[a] // page, slots[a] % page
            y = x[a:b].transpose(0, 1)                                          # [hk, rows, hs]
            most = y.abs().amax((1, 2))
            least = torch.ceil(torch.log2((most / 448).clamp_min(2.0 ** -117)))
            least = torch.where(most > 448 * torch.exp2(least), least + 1, least)
            least = torch.where(most <= 448 * torch.exp2(least - 1), least - 1, least).clamp(-117, 119)
            was = scale[number].double() - 127
            now = torch.maximum(least, was) if old else least
            value[number, :, :old] = rounded(value[number, :, :old] * torch.exp2(was - now)[:, None, None])
            value[number, :, old:old + b - a] = rounded(y / torch.exp2(now)[:, None, None])
            scale[number] = (now + 127).to(torch.uint8)
        if name == "v":
            value = value.view(value.shape[0], value.shape[1], page // 16, 16, -1).transpose(3, 4).contiguous()
        got[name], got[name + "_scale"] = value, scale
    return got


def _exact_attend(s):
    """Request by request and KV head by KV head."""
    case = s["case"]
    page, hq, hk, hs, group = case["page"], case["hq"], case["hk"], case["hs"], case["hq"] // case["hk"]
    cu, lengths = s["cu"].tolist(), s["len"].tolist()
    o = torch.zeros(s["total"], hq, hs, dtype=torch.float64, device="cuda")
    lse = torch.full((hq, s["total"]), -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(lengths):
        row = s["table"][i, :-(-length // page)].tolist()
        there = [b for b, number in enumerate(row) if number >= 0]
        if not there:
            continue
        where = torch.tensor([row[b] for b in there], device="cuda")
        pos = (torch.tensor(there, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)
        real = pos < length
        k = s["k_codes"].view(torch.uint8)[where].view(_F8).double() * torch.ldexp(torch.ones((), device="cuda", dtype=torch.float64), s["k_scale"][where].int() - 127)[..., None, None]
        v = s["v_codes"].view(torch.uint8)[where].view(_F8).double() * torch.ldexp(torch.ones((), device="cuda", dtype=torch.float64), s["v_scale"][where].int() - 127)[..., None, None, None]
        v = v.transpose(3, 4).flatten(2, 3)                                     # [pages, hk, page, hs]
        new = cu[i + 1] - cu[i]
        last = length - new + torch.arange(new, device="cuda") if case["causal"] else torch.full((new,), length - 1, device="cuda")
        hidden = (pos[real][None] > last[:, None])[:, None]                     # [new, 1, keys]
        for h in range(hk):
            kh, vh = k[:, h].reshape(-1, hs)[real], v[:, h].reshape(-1, hs)[real]
            qh = s["q"][cu[i]:cu[i + 1], h * group:(h + 1) * group].double()
            x = (qh.reshape(-1, hs) @ kh.t() / math.sqrt(hs)).view(new, group, -1).masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, -1)
            w = torch.exp_(x.sub_(torch.where(z == -math.inf, 0.0, z)[..., None]))
            o[cu[i]:cu[i + 1], h * group:(h + 1) * group] = (w.view(new * group, -1) @ vh).view(new, group, hs)
            lse[h * group:(h + 1) * group, cu[i]:cu[i + 1]] = z.t()
    return {"o": o, "lse": lse}
