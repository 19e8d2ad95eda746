"""Performance cases of the attention side of a layer, second part: norms of the query and key heads, the cache of 8-bit
elements, and the attention of sequences that share a prefix.

Operators (kind `op`):
  append   a norm of each query and key head and the rotary position on the new tokens, keys and values written into
           their pages; into a cache of 8-bit elements they are quantised, and read back from it afterwards
  decode   attention of one new token per sequence over a cache of 8-bit elements
  prompt   causal attention of many new tokens per sequence, packed, over a cache of 8-bit elements
  shared   attention of one new token per sequence, where groups of sequences share the pages of a long prefix

`run` computes each either with elementary torch operations in 32 bits (own = False) or with the framework's calls
(own = True), on the same inputs; `exact` evaluates the definitions in 64 bits.

The cache: pages of P tokens, page_table [sequences][pages] (-1: none).  A plain one is a pool [n_pages][2][kv_heads][P]
[dim] of the type of the queries (2: keys, values).  One of 8-bit elements is bytes [n_pages][2][kv_heads][P dim + P]: P
rows of dim elements (4 exponent and 3 mantissa bits, no infinities), then P bytes b, one a row, whose elements x stand
for x 2^(b - 127).  A row with largest magnitude m takes the least b >= 1 for which m <= 448 2^(b - 127), and each value
the nearest element (ties to the even one) that stands for no more than the largest number of the type: x <= 240 where 256
would be past it.

Row b of a batch brings tokens cu[b] .. cu[b+1] at positions pos0[b], pos0[b] + 1, ...; a token at position p sees the
keys max(0, p - window + 1) .. p (window 0: all of 0 .. p).  pos0[b] < 0 marks a row that is not served: nothing is
written for it, and its attention output, and what is read back for it, is zero.

Head layouts and sizes are those of the decode configurations (d_model 256, 4096, 5120 and 8192 as 4, 32, 40 and 64
heads, with as many or fewer key-value heads) and head sizes from 64 to 256.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
TOP = {"f32": 120, "f16": 8, "bf16": 120}  # the exponent at which 256 2^e is past the type's largest number
EPS = 1e-6
DEV = "cuda"


def _case(name, op, heads, kv_heads, dim, dtype, cache, page, n_seq, new, ctx, mix, window=0, rotary=0,
          interleaved=False, groups=0):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache,
            "page": page, "n_seq": n_seq, "new": new, "ctx": ctx, "mix": mix, "window": window, "rotary": rotary,
            "interleaved": interleaved, "groups": groups}


def listed():
    return [
        # one decode step of a small batch with normed heads: what each layer of each token pays, latency counts
        _case("append_norm_step", "append", 32, 8, 128, "f16", "same", 64, 8, 1, 3000, 1, rotary=128),
        # four ragged prompts of a large model with normed heads, one of them behind a cached prefix
        _case("append_norm_prompts", "append", 64, 8, 128, "bf16", "same", 64, 4, 5001, 700, 2, rotary=128),
        # one decode step of a serving batch into 8-bit pages, half of each head turned; read back as a check would
        _case("append8_step", "append", 40, 8, 128, "bf16", "e4m3", 32, 17, 1, 4000, 3, rotary=64),
        # prompts of a model with a key-value head per head into 8-bit pages, read back as for handing them on
        _case("append8_prompts", "append", 32, 32, 128, "f16", "e4m3", 64, 3, 4097, 900, 4, rotary=128, interleaved=True),
        # one user's chat, one head group per head: the smallest attention call of a 7B decode
        _case("decode8_one", "decode", 32, 32, 128, "f16", "e4m3", 64, 1, 1, 777, 5),
        # one user over a very long document, grouped heads: a single row against 131071 keys
        _case("decode8_long", "decode", 64, 8, 128, "bf16", "e4m3", 64, 1, 1, 131071, 6),
        # a serving batch of conversations from a few tokens to 8192, one of them not served in this step
        _case("decode8_batch", "decode", 32, 8, 128, "f16", "e4m3", 16, 64, 1, 8192, 7),
        # ragged prompts packed into one call, half of them behind cached prefixes, with a sliding window
        _case("prompt8_packed", "prompt", 40, 8, 128, "bf16", "e4m3", 32, 12, 2111, 3000, 8, window=4096),
        # a long document of a large model
        _case("prompt8_long", "prompt", 64, 8, 128, "bf16", "e4m3", 64, 1, 8192, 0, 9),
        # two samples of a short chat of a small model: the smallest call
        _case("shared_two", "shared", 4, 4, 64, "f32", "same", 16, 2, 1, 300, 10, groups=1),
        # parallel sampling: prompts of up to 3000 tokens, eight samples or fewer each, some hundred tokens along
        _case("shared_samples", "shared", 32, 8, 128, "f16", "same", 64, 32, 300, 3000, 11, groups=4),
        # one long document, many questions about it, in 8-bit pages
        _case("shared_document8", "shared", 64, 8, 128, "bf16", "e4m3", 64, 48, 1000, 32768, 12, groups=1),
    ]


HEADS = [(4, 4), (4, 2), (8, 1), (32, 32), (32, 8), (40, 40), (40, 8), (64, 8)]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "decode", "decode", "prompt", "shared", "shared"])
    heads, kv = rng.choice(HEADS)
    dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    page = rng.choice([16, 32, 64, 128, 256])
    mix = rng.randrange(1 << 30)
    if op == "append":
        n = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 8192 // n))
        return _case("", op, heads, kv, dim, dtype, "same" if dtype == "f32" else rng.choice(["same", "e4m3"]), page, n,
                     new, _log(rng, 1, 4000), mix, rotary=rng.choice([0, 16, 32, dim, dim]),
                     interleaved=rng.random() < 0.5)
    if op == "decode":
        n = _log(rng, 1, 96)
        ctx = _log(rng, 1, max(1, min(131071, (1 << 27) // (kv * dim * n))))
        return _case("", op, heads, kv, dim, dtype, "e4m3", page, n, 1, ctx, mix,
                     window=rng.choice([0, 0, _log(rng, 1, 4096)]))
    if op == "prompt":
        n = _log(rng, 1, 16)
        new = _log(rng, 2, max(2, int(((4.0e8 if dtype == "f32" else 2.0e9) * 64 / (heads * n * dim)) ** 0.5)))
        return _case("", op, heads, kv, dim, dtype, "e4m3", page, n, new, rng.choice([0, _log(rng, 1, 1000)]), mix,
                     window=rng.choice([0, 0, _log(rng, 1, 4096)]))
    groups = _log(rng, 1, 12)
    n = groups * _log(rng, 1, max(2, 96 // groups))
    own_tokens = _log(rng, 1, 1000)
    ctx = _log(rng, 1, max(1, min(32768, (1 << 27) // (kv * dim * n))))
    return _case("", op, heads, kv, dim, dtype, rng.choice(["same", "e4m3"]), page, n, own_tokens, ctx, mix,
                 window=rng.choice([0, 0, 0, _log(rng, 1, 8192)]), groups=groups)


def _members(case):
    """op shared: of each row its group's first row and the positions that the group shares (from the case alone)."""
    rng = random.Random(case["mix"] + 2)
    n, g = case["n_seq"], case["groups"]
    # the first group is a full one; the others end where chance has it, some of them with one row alone
    cuts = sorted(rng.sample(range(1, n), g - 1)) if g > 1 else []
    lead, prefix = [], []
    for k, (a, b) in enumerate(zip([0] + cuts, cuts + [n])):
        lead += [a] * (b - a)
        prefix += [case["ctx"] if k == 0 else _log(rng, 1, case["ctx"])] * (b - a)
    return lead, prefix


def _rows(case):
    """(first position, new tokens) of each row of the batch, from the case alone."""
    rng = random.Random(case["mix"])
    op, n, ctx, new = case["op"], case["n_seq"], case["ctx"], case["new"]
    out = []
    if op == "shared":
        for b, p in enumerate(_members(case)[1]):
            out.append((p - 1 + (new if b == 0 else _log(rng, 1, new)), 1))
    else:
        for b in range(n):
            if op == "decode":
                out.append((ctx - 1 if b == 0 else _log(rng, 1, ctx) - 1, 1))
            elif op == "append":
                k = new if b == 0 or new == 1 else _log(rng, 1, new)
                out.append((_log(rng, 1, ctx) - 1 if new == 1 or b == n - 1 else 0, k))
            else:
                k = new if b == 0 else _log(rng, 1, new)
                out.append((_log(rng, 1, ctx) if ctx and b % 2 else 0, k))
    if n >= 8 and op != "prompt":  # one row is not served in this step
        out[n - 2] = (-1, out[n - 2][1])
    return out


def _pairs(case):
    """Pairs of a token and a key that it sees."""
    tot, w = 0, case["window"]
    for p0, n in _rows(case):
        if p0 < 0:
            continue
        if w == 0:
            tot += n * (p0 + 1) + n * (n - 1) // 2
        else:
            full = max(0, min(n, w - p0))  # tokens whose whole past fits the window
            tot += full * (p0 + 1) + full * (full - 1) // 2 + (n - full) * w
    return tot


def _ceil(a, b):
    return -(-a // b)


def _first(case, p):
    return 0 if case["window"] == 0 else max(0, p + 1 - case["window"])


def work(case):
    op, w, D = case["op"], SIZE[case["dtype"]], case["dim"]
    hq, hk = case["heads"], case["kv_heads"]
    rows = _rows(case)
    row_bytes = D + 1 if case["cache"] == "e4m3" else D * w  # of a key or a value in the cache
    if op == "append":
        t = sum(n for p0, n in rows if p0 >= 0)
        moved = (2 * hq + 2 * hk) * D * w + 2 * hk * row_bytes + case["rotary"] * 4
        if case["cache"] == "e4m3":  # and back
            moved += 2 * hk * (row_bytes + D * w)
        return {"bytes": t * moved + 2 * D * w, "flops": t * (hq + hk) * (case["rotary"] * 3 + D * 4)}
    t = sum(n for p0, n in rows)
    if op == "shared":
        lead, prefix = _members(case)
        keys = 0
        for a in sorted(set(lead)):
            live = [p0 for (p0, _), x in zip(rows, lead) if x == a and p0 >= 0]
            if live:  # the shared keys that some row of the group sees, then those of each row alone
                keys += max(0, prefix[a] - min(_first(case, p) for p in live))
                keys += sum(p + 1 - max(prefix[a], _first(case, p)) for p in live)
    else:
        keys = sum(p0 + n - _first(case, p0) for p0, n in rows if p0 >= 0)
    return {"bytes": 2 * t * hq * D * w + 2 * keys * hk * row_bytes, "flops": 4 * hq * D * _pairs(case)}


def _layout(case):
    """The page table of a case as lists (from the case alone): random pages of the pool, as they come to lie after a
    while of serving, and the sizes of the pool and the table.  Rows of a group have the shared prefix's whole pages in
    common, and a page each for what its last, partly filled page held."""
    rng = random.Random(case["mix"] + 1)
    P = case["page"]
    rows = _rows(case)
    need = [_ceil(max(p0, 0) + n, P) for p0, n in rows]
    held = [0] * len(rows)  # pages that a row has from its group's first one
    lead = list(range(len(rows)))
    if case["op"] == "shared":
        lead, prefix = _members(case)
        need = [max(k, _ceil(p, P)) for k, p in zip(need, prefix)]
        held = [0 if a == b else prefix[b] // P for b, a in enumerate(lead)]
    n_pages = sum(need) - sum(held) + 3
    pages = list(range(n_pages))
    rng.shuffle(pages)
    table, at = [], 0
    for b, k in enumerate(need):
        table.append((table[lead[b]][:held[b]] if held[b] else []) + pages[at:at + k - held[b]])
        at += k - held[b]
    return {"table": table, "n_pages": n_pages, "width": max(need) + 1}


def _pow2(e):
    """2^e of whole numbers e, -126 .. 127, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _quantise(x, top):
    """The elements and exponents of rows x [..., dim] of 32-bit values."""
    m, ex = torch.frexp(x.abs().amax(-1))
    e = torch.where(m <= 0.875, ex - 9, ex - 8).clamp(min=-126)  # 448 is 0.875 times 2^9
    e = torch.where(m == 0, torch.full_like(e, -126), e)
    most = torch.where(e >= top, 240.0, 448.0)[..., None]
    y = (x * _pow2(-e)[..., None]).clamp(-most, most)
    return y.to(torch.float8_e4m3fn), e


def _bytes_of(elements, e):
    """Rows [pages][heads][P][dim] as the bytes of pages [pages][heads][P dim + P]."""
    body = elements.view(torch.uint8).flatten(-2)
    return torch.cat((body, (e + 127).to(torch.uint8)), dim=-1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, dt = case["op"], DT[case["dtype"]]
    hq, hk, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    rows, lay = _rows(case), _layout(case)
    n, N, M = len(rows), lay["n_pages"], lay["width"]

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)

    table = np.full((n, M), -1, dtype=np.int32)
    for b, r in enumerate(lay["table"]):
        table[b, :len(r)] = r
    T = sum(k for _, k in rows)
    cu = [0]
    for _, k in rows:
        cu.append(cu[-1] + k)
    longest = max(max(p0 + k for p0, k in rows), 1)
    st = {"case": case, "rows": rows, "table": i32(table), "N": N, "M": M, "T": T, "cu": i32(cu), "cu_host": cu,
          "pos0": i32([p0 for p0, _ in rows]), "longest": longest, "scale": 1.0 / math.sqrt(D)}
    if op == "append":
        # views of one fused projection, as a layer produces them
        qkv = (normal(T, hq + 2 * hk, D) * (0.5 + normal(1, hq + 2 * hk, 1).abs())).to(dt)
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        st["wq"], st["wk"] = (1 + 0.2 * normal(D)).to(dt), (1 + 0.2 * normal(D)).to(dt)
        st["q_out"] = torch.zeros((T, hq, D), dtype=dt, device=DEV)
        if case["cache"] == "e4m3":
            st["pool"] = torch.zeros((1, N, 2, hk, P * D + P), dtype=torch.uint8, device=DEV)
            st["k_out"], st["v_out"] = (torch.zeros((T, hk, D), dtype=dt, device=DEV) for _ in range(2))
        else:
            st["pool"] = torch.zeros((1, N, 2, hk, P, D), dtype=dt, device=DEV)
        R = case["rotary"]
        if R:
            f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEV) / R)
            ang = torch.arange(longest, dtype=torch.float64, device=DEV)[:, None] * f[None]
            st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
    else:
        st["q"] = normal(T, hq, D).to(dt)
        st["out"] = torch.empty((T, hq, D), dtype=dt, device=DEV)
        lens = [max(0, p0 + k) if p0 >= 0 else 0 for p0, k in rows]
        if op == "shared":
            lead, prefix = _members(case)
            lens = [max(x, p) for x, p in zip(lens, prefix)]
            st["lead"], st["prefix"], st["lead_host"] = i32(lead), i32(prefix), lead
        # what no token may see holds NaN: unused pages and the ends of last pages
        fill = {}
        for b, r in enumerate(lay["table"]):
            for j, page in enumerate(r):
                fill[page] = max(0, min(P, lens[b] - j * P))
        used = torch.tensor(sorted(fill), dtype=torch.long, device=DEV)
        full = torch.tensor([fill[p] for p in sorted(fill)], device=DEV)
        data = normal(len(fill), 2, hk, P, D).to(dt)
        if op == "shared":  # a member's copy of the prefix's last, partly filled page
            order = {p: i for i, p in enumerate(sorted(fill))}
            for b, a in enumerate(lead):
                j, r = divmod(prefix[b], P)
                if a != b and r:
                    data[order[lay["table"][b][j]], :, :, :r] = data[order[lay["table"][a][j]], :, :, :r]
        none = (torch.arange(P, device=DEV)[None] >= full[:, None])[:, None, None]
        if case["cache"] == "e4m3":
            st["pool"] = torch.full((1, N, 2, hk, P * D + P), 127, dtype=torch.uint8, device=DEV)  # 127: NaN
            for i in range(0, len(fill), 512):
                x, e = _quantise(data[i:i + 512].float(), TOP[case["dtype"]])
                x = x.view(torch.uint8).masked_fill(none[i:i + 512, ..., None], 127)
                st["pool"][0, used[i:i + 512]] = _bytes_of(x, e.masked_fill(none[i:i + 512], 0))
        else:
            st["pool"] = torch.full((1, N, 2, hk, P, D), float("nan"), dtype=dt, device=DEV)
            st["pool"][0, used] = data.masked_fill(none[..., None], float("nan"))
    if own:
        from paper_2608_22643_amd import binding as B

        st["B"] = B
        st["shape"] = B.make_kv_shape(1, hq, hk, D, P, N, n, M, case["dtype"], case["cache"])
        st["ws"] = torch.zeros(B.np_kv_workspace_size(st["shape"]), dtype=torch.uint8, device=DEV)
        st["batch"] = B.make_kv_batch(n, T, max(k for _, k in rows), longest, st["pos0"],
                                      cu_tokens=None if op in ("decode", "shared") else st["cu"])
        if op == "append":
            st["qkv"] = B.make_qkv(st["q"], st["k"], st["v"], st["q_out"])
            st["norm"] = B.make_qk_norm(st["wq"], st["wk"], EPS)
            st["rotary"] = B.make_rotary(st["cos"], st["sin"], case["interleaved"]) if case["rotary"] else None
        elif op == "shared":
            st["shared"] = B.make_kv_shared(st["lead"], st["prefix"], max(prefix))
    return st


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    B, case = st["B"], st["case"]
    op, shape, ws = case["op"], st["shape"], st["ws"]
    if op == "append":
        B.np_kv_append_norm(shape, 0, st["batch"], st["table"], st["qkv"], st["norm"], st["rotary"], st["pool"], ws)
        if case["cache"] != "e4m3":
            return [st["q_out"], st["pool"]]
        B.np_kv_read(shape, 0, st["batch"], st["table"], st["pool"], st["k_out"], st["v_out"], ws)
        return [st["q_out"], st["k_out"], st["v_out"]]
    args = (st["table"], st["q"], st["pool"], st["scale"], case["window"], st["out"], ws)
    if op == "shared":
        B.np_attn_decode_shared(shape, 0, st["batch"], st["shared"], *args)
    elif op == "decode":
        B.np_attn_decode(shape, 0, st["batch"], *args)
    else:
        B.np_attn_prompt(shape, 0, st["batch"], *args)
    return [st["out"]]


def _run_plain(st):
    op = st["case"]["op"]
    return _plain_append(st) if op == "append" else _plain_prompt(st) if op == "prompt" else _plain_single(st)


def _plain_append(st):
    case = st["case"]
    P, R, D = case["page"], case["rotary"], case["dim"]
    row = torch.repeat_interleave(torch.arange(case["n_seq"], device=DEV), (st["cu"][1:] - st["cu"][:-1]).long(),
                                  output_size=st["T"])
    first = st["pos0"].long()[row]
    pos = (first + torch.arange(st["T"], device=DEV) - st["cu"].long()[row]).clamp(min=0)
    live = first >= 0
    dt = st["q"].dtype

    def turned(x, weight):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        if not R:
            return x
        c, s = st["cos"][pos][:, None], st["sin"][pos][:, None]
        if case["interleaved"]:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            r = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
        else:
            a, b = x[..., :R // 2], x[..., R // 2:R]
            r = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
        return torch.cat((r, x[..., R:]), dim=-1)

    here = live[:, None, None]
    st["q_out"].copy_(torch.where(here, turned(st["q"], st["wq"]).to(dt), st["q_out"]))
    keys, values = turned(st["k"], st["wk"]).to(dt), st["v"]
    at = live.nonzero().flatten()
    page, slot = st["table"].long()[row, pos // P][at], (pos % P)[at]
    if case["cache"] != "e4m3":
        st["pool"][0, :, 0][page, :, slot] = keys[at]
        st["pool"][0, :, 1][page, :, slot] = values[at]
        return [st["q_out"], st["pool"]]
    body = st["pool"][0][..., :P * D].unflatten(-1, (P, D))
    exps = st["pool"][0][..., P * D:]
    for i, x in enumerate((keys, values)):
        y, e = _quantise(x.float(), TOP[case["dtype"]])
        body[:, i][page, :, slot] = y.view(torch.uint8)[at]
        exps[:, i][page, :, slot] = (e + 127).to(torch.uint8)[at]
    for i, to in enumerate((st["k_out"], st["v_out"])):
        x = body[:, i][page, :, slot].view(torch.float8_e4m3fn).float()
        x = x * _pow2(exps[:, i][page, :, slot].int() - 127)[..., None]
        to.zero_()
        to[at] = x.to(dt)
    return [st["q_out"], st["k_out"], st["v_out"]]


def _heads(st, pages, kind, h):
    """Keys (kind 0) or values (1) of heads h (a slice) in `pages` [...][count], 32 bits: [...][heads][positions][dim]."""
    case = st["case"]
    P, D = case["page"], case["dim"]
    x = st["pool"][0, :, kind, h][pages]
    if case["cache"] == "e4m3":
        x = (x[..., :P * D].unflatten(-1, (P, D)).view(torch.float8_e4m3fn).float()
             * _pow2(x[..., P * D:].int() - 127)[..., None])
    return x.float().movedim(-4, -3).flatten(-3, -2)


def _softmax(s, hide):
    """Of scores whose hidden places get no weight; zero where all are hidden."""
    s = s.masked_fill(hide, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e30))
    return p / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_single(st):
    """One token a row: all rows at once, as long as the longest, so many heads at a time that keys and scores stay
    below 1 GiB each."""
    case = st["case"]
    hk, G, w = case["kv_heads"], case["heads"] // case["kv_heads"], case["window"]
    n, D = case["n_seq"], case["dim"]
    pages = st["table"][:, :_ceil(st["longest"], case["page"])].long().clamp(min=0)
    pos = st["pos0"].long()
    key = torch.arange(pages.shape[1] * case["page"], device=DEV)
    see = key[None] <= pos[:, None]
    if w:
        see &= key[None] > pos[:, None] - w
    hide = ~see[:, None, None]
    q, out = st["q"].view(n, hk, G, D), st["out"].view(n, hk, G, D)
    step = max(1, (1 << 28) // (n * key.numel() * max(G, D)))
    for h0 in range(0, hk, step):
        h = slice(h0, min(hk, h0 + step))
        k = _heads(st, pages, 0, h)
        v = _heads(st, pages, 1, h).masked_fill(hide[..., 0, :, None], 0.0)
        s = (q[:, h].float() @ k.transpose(-1, -2).contiguous()) * st["scale"]
        out[:, h] = (_softmax(s, hide) @ v).to(out.dtype)
    return [st["out"]]


def _plain_prompt(st):
    """A row at a time, so many heads and, where one head is too much, so many queries at a time that the scores stay
    below 1 GiB."""
    case = st["case"]
    hk, G, w, P, D = case["kv_heads"], case["heads"] // case["kv_heads"], case["window"], case["page"], case["dim"]
    for b, (p0, n) in enumerate(st["rows"]):
        lo = _first(case, p0) // P * P  # the first page that a token of the row can see
        ln = p0 + n
        pages = st["table"][b, lo // P:_ceil(ln, P)].long()
        key = torch.arange(lo, ln, device=DEV)
        t0 = st["cu_host"][b]
        q = st["q"][t0:t0 + n].view(n, hk, G, D).movedim(0, 1)
        out = st["out"][t0:t0 + n].view(n, hk, G, D).movedim(0, 1)
        rows = max(1, min(n, (1 << 28) // (G * (ln - lo))))
        step = max(1, (1 << 28) // (G * (ln - lo) * rows))
        for h0 in range(0, hk, step):
            h = slice(h0, min(hk, h0 + step))
            k = _heads(st, pages, 0, h)[:, :ln - lo].transpose(1, 2).contiguous()
            v = _heads(st, pages, 1, h)[:, :ln - lo]
            for i in range(0, n, rows):
                m = min(rows, n - i)
                pos = torch.arange(p0 + i, p0 + i + m, device=DEV)
                hide = key[None] > pos[:, None]
                if w:
                    hide |= key[None] <= pos[:, None] - w
                s = (q[h, i:i + m].float().flatten(1, 2) @ k).unflatten(1, (m, G)) * st["scale"]
                o = _softmax(s, hide[None, :, None]).flatten(1, 2) @ v
                out[h, i:i + m] = o.unflatten(1, (m, G)).to(out.dtype)
    return [st["out"]]


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = keep
    return _exact_append(case, st) if case["op"] == "append" else _exact_attention(case, st)


def _tokens(rows):
    """(row, position) of each token of the rows that are served, and its place among the tokens."""
    got, t = [], 0
    for b, (p0, n) in enumerate(rows):
        got += [(t + i, b, p0 + i) for i in range(n) if p0 >= 0]
        t += n
    return got


def _exact_append(case, st):
    P, R, D = case["page"], case["rotary"], case["dim"]
    toks = _tokens(st["rows"])
    at = torch.tensor([t for t, _, _ in toks], dtype=torch.long, device=DEV)
    p = torch.tensor([q for _, _, q in toks], dtype=torch.long, device=DEV)

    def turned(x, weight):
        x = x[at].double()
        x = weight.double() * x / ((x ** 2).sum(-1, keepdim=True) / D + EPS).sqrt()
        y = x.clone()
        for i in range(R // 2):
            j, k = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
            c, s = st["cos"][p, i].double()[:, None], st["sin"][p, i].double()[:, None]
            y[..., j] = c * x[..., j] - s * x[..., k]
            y[..., k] = s * x[..., j] + c * x[..., k]
        return y

    q_out = torch.zeros(st["q_out"].shape, dtype=torch.float64, device=DEV)
    q_out[at] = turned(st["q"], st["wq"])
    keys, values = turned(st["k"], st["wk"]), st["v"][at].double()
    if case["cache"] == "e4m3":
        # the elements' rounding is part of the definition: of what the type of the heads holds
        k_out = torch.zeros(st["k_out"].shape, dtype=torch.float64, device=DEV)
        v_out = torch.zeros_like(k_out)
        k_out[at] = _exact_elements(keys.to(DT[case["dtype"]]).double(), TOP[case["dtype"]])
        v_out[at] = _exact_elements(values, TOP[case["dtype"]])
        return [q_out, k_out, v_out]
    lists = _layout(case)["table"]
    page = torch.tensor([lists[b][q // P] for _, b, q in toks], dtype=torch.long, device=DEV)
    pool = torch.zeros(st["pool"].shape, dtype=torch.float64, device=DEV)
    for h in range(case["kv_heads"]):
        pool[0, page, 0, h, p % P] = keys[:, h]
        pool[0, page, 1, h, p % P] = values[:, h]
    return [q_out, pool]


def _exact_elements(x, top):
    """What rows x stand for once quantised, from the element's definition: multiples of 2^(k - 3) between 2^k and
    2^(k + 1), from 2^-6 on, of 2^-9 below that, 448 the largest."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -126.0)
    some = most > 0
    e[some] = torch.log2(most[some] / 448).ceil().clamp(min=-126)
    e = torch.where((e > -126) & (most <= 448 * torch.exp2(e - 1)), e - 1, e)
    e = torch.where(most > 448 * torch.exp2(e), e + 1, e)
    y = x / torch.exp2(e)
    k = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    k = torch.where(torch.exp2(k + 1) <= y.abs(), k + 1, k)
    unit = torch.exp2(k - 3)
    y = torch.round(y / unit) * unit  # round: ties to even
    limit = torch.where(e >= top, 240.0, 448.0)
    return torch.minimum(torch.maximum(y, -limit), limit) * torch.exp2(e)


def _exact_attention(case, st):
    hq, hk, D, P, w = case["heads"], case["kv_heads"], case["dim"], case["page"], case["window"]
    if 4.0 * hq * D * _pairs(case) > 3e12:
        return None
    lists = _layout(case)["table"]
    out = torch.zeros((st["T"], hq, D), dtype=torch.float64, device=DEV)

    def cached(pages, kind, h):
        x = st["pool"][0, pages, kind, h]
        if case["cache"] == "e4m3":
            e = x[:, P * D:].double() - 127
            x = x[:, :P * D].reshape(-1, P, D).view(torch.float8_e4m3fn).double() * torch.exp2(e)[..., None]
        return x.reshape(-1, D).double()

    for b, (p0, n) in enumerate(st["rows"]):
        if p0 < 0:
            continue
        ln, t0 = p0 + n, st["cu_host"][b]
        pages = torch.tensor(lists[b][:_ceil(ln, P)], dtype=torch.long, device=DEV)
        for h in range(hk):
            k, v = cached(pages, 0, h)[:ln], cached(pages, 1, h)[:ln]
            for i in range(0, n, max(1, (1 << 27) // (ln * (hq // hk)))):
                m = min(n - i, max(1, (1 << 27) // (ln * (hq // hk))))
                q = st["q"][t0 + i:t0 + i + m, h * hq // hk:(h + 1) * hq // hk].double()
                p = torch.arange(p0 + i, p0 + i + m, device=DEV)[:, None, None]
                j = torch.arange(ln, device=DEV)[None, None]
                see = (j <= p) & (j > p - w) if w else j <= p
                z = (q.reshape(-1, D) @ k.T * st["scale"]).view(m, -1, ln)
                z = torch.where(see, z, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
                y = torch.softmax(z, dim=-1).view(-1, ln) @ v
                out[t0 + i:t0 + i + m, h * hq // hk:(h + 1) * hq // hk] = y.view(m, -1, D)
    return [out]
