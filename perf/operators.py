"""The 8-bit serving operators whose speed counts: what a policy server that keeps its weights and its K/V cache in
8 bits asks of this library, call by call.

Four kinds of call, each through the package's public entry points:

* "linear": quantize_tokens (an int8 code per value, an absolute maximum per token) and int8_gemm with int8 weights
  that carry a scale per output channel;
* "append": kv_pages_write, the keys and values of new tokens into the pages of their requests;
* "restore": kv_pages_read, a request's cached rows back as dense [request][head][row][dim] values; with write true
  the rows are written first, the whole way of a prefix through a quantised cache;
* "attend": paged_attention, the new tokens of every request over its pages (the new tokens' own rows among them).

Widths and head counts are those of this repository's workloads (workloads/__init__.py).  Keys and values are N(0, 1)
with a few channels several times larger, as projections of real hidden states have them; requests have lengths of
their own, and their pages lie anywhere in the pool.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"i8": 127.0, "e4m3": 448.0}
ELEM = {"f32": 0, "bf16": 1}
SMALLEST = 1e-5      # the least absolute maximum of a quantised row
BYTES = {"f32": 4, "bf16": 2, "i8": 1, "e4m3": 1}


def _linear(name, M, N, K, elem, bias):
    c = dict(kind="linear", M=M, N=N, K=K, elem=elem, bias=bias)
    return dict(c, name=name) if name else c


def _append(name, requests, longest, tokens, heads, dim, page, pages):
    c = dict(kind="append", requests=requests, longest=longest, tokens=tokens, heads=heads, dim=dim, page=page, pages=pages)
    return dict(c, name=name) if name else c


def _restore(name, requests, longest, heads, dim, page, pages, elem, write):
    c = dict(kind="restore", requests=requests, longest=longest, heads=heads, dim=dim, page=page, pages=pages, elem=elem,
             write=write)
    return dict(c, name=name) if name else c


def _attend(name, requests, longest, tokens, heads, group, dim, page, pages, causal, window):
    c = dict(kind="attend", requests=requests, longest=longest, tokens=tokens, heads=heads, group=group, dim=dim,
             page=page, pages=pages, causal=causal, window=window)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token through a square projection of the 2560-wide backbone: latency, then the weights' bytes.
        _linear("linear_one_token", 1, 2560, 2560, "bf16", False),
        # A short prefix of the 720-wide expert with an odd output width, fp32 out, with a bias.
        _linear("linear_ragged", 241, 1601, 720, "f32", True),
        # One observation's prefix through the 2048-wide backbone's down projection: few tiles, a long reduction.
        _linear("linear_prefix_down", 816, 2048, 16384, "bf16", False),
        # Ten observations at once through its up projection: the matrix cores' rate.
        _linear("linear_prefix_up_batch", 8160, 16384, 2048, "bf16", False),
        # A decoding batch: one new token for each of 64 requests, int8 pages.
        _append("append_decode", 64, 1024, 1, 5, 128, 64, "i8"),
        # Sixteen 2048-row prefixes of the 256-wide head through int8 pages and back: what keeping them costs.
        _restore("store_and_restore_prefix", 16, 2048, 1, 256, 64, "i8", "bf16", True),
        # Four long histories out of e4m3 pages.
        _restore("restore_long", 4, 32768, 5, 128, 32, "e4m3", "bf16", False),
        # One token of one request over its 867 cached rows: latency.
        _attend("attend_one_request", 1, 867, 1, 8, 8, 256, 64, "bf16", True, 0),
        # The fp32 expert's chunk.
        _attend("attend_f32_chunk", 2, 72, 8, 4, 4, 64, 16, "f32", False, 0),
        # Eight action chunks of 50 tokens over 816-row prefixes, all rows visible.
        _attend("attend_action_chunks", 8, 866, 50, 8, 8, 256, 64, "bf16", False, 0),
        # A decoding batch of 64 requests of up to 8192 rows: the cache's bytes.
        _attend("attend_decode_batch", 64, 8192, 1, 20, 4, 128, 32, "i8", True, 0),
        # Three long prompts in chunks of up to 2048 tokens, causal: the matrix cores' rate.
        _attend("attend_prefill_chunks", 3, 10007, 2048, 20, 4, 128, 128, "e4m3", True, 0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        largest[c["kind"]] = max(largest.get(c["kind"], 0.0), w["bytes"] / 4e12 + w["flops"] / 1e15)
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] / 4e12 + w["flops"] / 1e15 <= largest[c["kind"]]:
            return c


def _draw(rng):
    kind = rng.choice(["linear", "linear", "append", "restore", "attend", "attend", "attend"])
    dim = rng.choice([64, 128, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "linear":
        return _linear(None, _log(rng, 1, 8192), _log(rng, 16, 16384), 16 * _log(rng, 4, 1024), rng.choice(["bf16", "f32"]),
                       rng.random() < 0.5)
    if kind == "append":
        tokens = rng.choice([1, _log(rng, 1, 512)])
        return _append(None, _log(rng, 1, 64), tokens + _log(rng, 1, 1024), tokens, rng.choice([1, 2, 5, 8]), dim, page,
                       rng.choice(["bf16", "i8", "e4m3", "f32"]))
    if kind == "restore":
        return _restore(None, _log(rng, 1, 32), _log(rng, 16, 32768), rng.choice([1, 2, 5, 8]), dim, page,
                        rng.choice(["bf16", "i8", "e4m3"]), rng.choice(["bf16", "f32"]), rng.random() < 0.5)
    tokens = rng.choice([1, 1, 50, _log(rng, 2, 2048)])
    pages = rng.choice(["bf16", "bf16", "i8", "i8", "e4m3", "e4m3", "f32"])
    group = rng.choice([1, 2, 3, 4, 8])
    return _attend(None, _log(rng, 1, 64), tokens + _log(rng, 1, 32768), tokens, group * rng.choice([1, 2, 5]), group,
                   min(dim, 128) if pages == "f32" else dim, page, pages, rng.random() < 0.6,
                   rng.choice([0, 0, 0, _log(rng, 16, 4096)]))


def _lengths(c):
    """(cached rows, new tokens) of each request: between a sixteenth of the longest and the longest, spread evenly, the
    first one the longest."""
    part = [1.0 - 15 / 16 * ((b * 0.6180339887) % 1.0) for b in range(c["requests"])]
    tokens = [max(1, int(c.get("tokens", 0) * p)) if c.get("tokens", 0) else 0 for p in part]
    rows = [max(n, int(c["longest"] * p)) for p, n in zip(part, tokens)]
    if c["kind"] == "restore" and c["write"]:
        tokens = rows
    return rows, tokens


def _visible(c):
    """(rows that some new token sees, pairs of new token and row that it sees), over all requests."""
    rows, pairs = 0, 0
    for length, n in zip(*_lengths(c)):
        w = c["window"] or length
        last = range(length - n, length) if c["causal"] else [length - 1] * n
        # with a window a token sees the rows after its own position less the window
        seen = [min(top + 1, top + 1 - max(0, at - w + 1)) for top, at in zip(last, range(length - n, length))]
        pairs += sum(seen)
        rows += length - max(0, length - n - w + 1)
    return rows, pairs


def work(c):
    if c["kind"] == "linear":
        M, N, K, e = c["M"], c["N"], c["K"], BYTES[c["elem"]]
        # x is bf16; the codes are an output, and the product's input as well
        return {"bytes": 2.0 * M * K + M * K + 4.0 * M + N * K + 4.0 * N + e * M * N, "flops": 2.0 * M * N * K}
    scale = 4 if c["pages"] in TOP else 0
    row = 2.0 * c["heads"] * (c["dim"] * BYTES[c["pages"]] + scale)      # a cached row, K and V (attend: below)
    lens, tokens = _lengths(c)
    if c["kind"] == "append":
        wide = 4 if c["pages"] == "f32" else 2
        return {"bytes": sum(tokens) * (2.0 * c["heads"] * c["dim"] * wide + row), "flops": 4.0 * sum(tokens) * c["heads"] * c["dim"]}
    if c["kind"] == "restore":
        dense = 2.0 * c["heads"] * c["dim"] * sum(lens)
        return {"bytes": sum(lens) * row * (2 if c["write"] else 1) + dense * (BYTES[c["elem"]] + (2 if c["write"] else 0)),
                "flops": 2.0 * dense}
    rows, pairs = _visible(c)
    row = row / c["group"]      # c["heads"] counts query heads here
    wide = 4 if c["pages"] == "f32" else 2
    return {"bytes": rows * row + sum(tokens) * c["heads"] * (2.0 * c["dim"] * wide + 4), "flops": 4.0 * pairs * c["heads"] * c["dim"]}


def _values(gen, shape, dtype):
    """N(0, 1), every sixteenth channel or so four times larger."""
    x = torch.randn(shape, generator=gen, device="cuda")
    big = 1.0 + 3.0 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.06)
    return (x * big).to(dtype)


def _pool(gen, c, heads, count):
    """Page pools with something in every row, as a server's pool has: K, V and, for 8-bit pages, their scales."""
    shape = (count, heads, c["page"], c["dim"])
    out = []
    for _ in range(2):
        if c["pages"] in TOP:
            x = torch.randn(shape, generator=gen, device="cuda") * (TOP[c["pages"]] / 3)
            x = x.clamp_(-TOP[c["pages"]], TOP[c["pages"]])
            out += [x.round_().to(torch.int8) if c["pages"] == "i8" else x.to(torch.float8_e4m3fn),
                    (0.5 + torch.rand(shape[:3], generator=gen, device="cuda")) * (3 / TOP[c["pages"]])]
        else:
            out += [torch.randn(shape, generator=gen, device="cuda").to(TYPES[c["pages"]]), None]
    return dict(k=out[0], k_scale=out[1], v=out[2], v_scale=out[3])


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=c)
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _values(gen, (M, K), torch.bfloat16)
        s["w"] = torch.randint(-127, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
        s["w_scale"] = (0.5 + torch.rand(N, generator=gen, device="cuda")) / (127 * K ** 0.5)
        s["bias"] = torch.randn(N, generator=gen, device="cuda") if c["bias"] else None
        s["q"] = torch.zeros(M, K, dtype=torch.int8, device="cuda")
        s["r"] = torch.zeros(M, device="cuda")
        s["y"] = torch.zeros(M, N, dtype=TYPES[c["elem"]], device="cuda")
        return s
    lens, tokens = _lengths(c)
    B, dim, page = c["requests"], c["dim"], c["page"]
    heads = c["heads"] // c["group"] if c["kind"] == "attend" else c["heads"]
    need = [-(-n // page) for n in lens]
    count = sum(need) + 3                                    # some pages are nobody's
    s.update(_pool(gen, c, heads, count))
    order = torch.randperm(count, generator=gen, device="cuda", dtype=torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32)   # places that no page holds are -1
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.arange(at, at + n, dtype=torch.int32)
        at += n
    table = table.cuda()
    s["table"] = torch.where(table < 0, table, order[table.clamp_min(0).long()])
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    starts = [0]
    for n in tokens:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32).cuda()
    s["longest"], s["most"], s["kv_heads"] = max(lens), max(tokens), heads
    total = starts[-1] + (3 if c["kind"] == "attend" else 0)  # a padded batch: rows behind the last request
    s["total"] = total
    wide = torch.float32 if c["pages"] == "f32" else torch.bfloat16
    if c["kind"] == "append" or c.get("write"):
        # [query | key | value] rows of a fused projection: the keys and values are views with its pitch
        fused = _values(gen, (total, 4 * heads, dim), wide)
        s["k_new"], s["v_new"] = fused[:, 2 * heads:3 * heads], fused[:, 3 * heads:]
    if c["kind"] == "restore":
        s["k_out"] = torch.zeros(B, heads, s["longest"], dim, dtype=TYPES[c["elem"]], device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
    if c["kind"] == "attend":
        s["queries"] = _values(gen, (total, c["heads"], dim), wide)
        s["o"] = torch.zeros(total, c["heads"], dim, dtype=wide, device="cuda")
        s["lse"] = torch.zeros(total, c["heads"], device="cuda")
    return s


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["kind"] == "linear":
        return _plain_linear(s)
    if c["kind"] == "append":
        return _plain_append(s)
    if c["kind"] == "restore":
        return _plain_restore(s)
    return _plain_attend(s)


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _own(s):
    from paper_2606_08094_amd import vla
    c = s["case"]
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        vla.quantize_tokens(1, s["x"], M, K, K, s["q"], K, s["r"])
        vla.int8_gemm(s["q"], K, s["r"], s["w"], K, s["w_scale"], s["bias"], M, N, K, ELEM[c["elem"]], s["y"], N)
        return {"y": s["y"], "q": s["q"], "r": s["r"]}
    if "pages" not in s:      # what a server makes once for its pool, its batch and the shape of its calls
        s["pages"] = vla.KVPages(c["pages"], s["k"].shape[0], c["page"], s["kv_heads"], c["dim"], s["k"], s["v"],
                                 s["k_scale"], s["v_scale"])
        s["batch"] = vla.KVBatch(c["requests"], s["table"].shape[1], s["total"], s["longest"], s["table"], s["lens"],
                                 s["starts"])
        if c["kind"] == "attend":
            s["bytes"] = vla.paged_attention_workspace(s["pages"], s["batch"], c["heads"])
            s["space"] = torch.empty(max(16, s["bytes"]), dtype=torch.uint8, device="cuda")
    elem = 0 if c["pages"] == "f32" else 1
    if c["kind"] == "append" or c.get("write"):
        vla.kv_pages_write(s["pages"], s["batch"], elem, s["k_new"], s["v_new"], 4 * s["kv_heads"] * c["dim"], c["dim"])
    if c["kind"] == "append":
        return _pages(s)
    if c["kind"] == "restore":
        vla.kv_pages_read(s["pages"], s["batch"], s["longest"], ELEM[c["elem"]], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    vla.paged_attention(s["pages"], s["batch"], c["heads"], elem, s["queries"], c["heads"] * c["dim"], s["o"],
                        c["heads"] * c["dim"], c["dim"] ** -0.5, causal=c["causal"], window=c["window"], lse=s["lse"],
                        workspace=s["space"], workspace_bytes=s["bytes"])
    return {"o": s["o"], "lse": s["lse"]}


def _pages(s):
    """The pool as it stands: its codes and scales, or its values."""
    return {n: s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None}


# ---- the plain form: elementary operations in fp32 -------------------------------------------------------------------

def _quantise(x, top):
    """(x scaled to the codes' range, absolute maximum), in fp32: the codes are defined by these roundings."""
    r = x.abs().amax(-1, keepdim=True).clamp_min(SMALLEST)
    return x * torch.div(torch.full_like(r, top), r), r


def _codes(x, kind):
    y, r = _quantise(x.float(), TOP[kind])
    code = y.round().clamp(-128, 127).to(torch.int8) if kind == "i8" else y.to(torch.float8_e4m3fn)
    return code, torch.div(r, torch.full_like(r, TOP[kind]))[..., 0]


def _plain_linear(s):
    c = s["case"]
    y, r = _quantise(s["x"].float(), 127.0)
    q = y.round().clamp(-128, 127)
    out = (q @ s["w"].float().t().contiguous()) * (r * s["w_scale"] / 127.0)
    if s["bias"] is not None:
        out = out + s["bias"]
    return {"y": out.to(TYPES[c["elem"]]), "q": q.to(torch.int8), "r": r[:, 0]}


def _places(s):
    """(page, row within it) of every new token."""
    c = s["case"]
    t = torch.arange(s["total"], device="cuda")
    b = torch.searchsorted(s["starts"][1:].long().contiguous(), t, right=True)
    end = s["starts"][1:].long()[b]
    at = s["lens"].long()[b] - end + t
    return s["table"].long()[b, at // c["page"]], at % c["page"]


def _plain_append(s):
    c = s["case"]
    page, row = _places(s)
    k, v = s["k_new"], s["v_new"]
    if c["pages"] in TOP:
        (kq, ks), (vq, vs) = _codes(k, c["pages"]), _codes(v, c["pages"])
        s["k"].view(torch.uint8)[page, :, row], s["v"].view(torch.uint8)[page, :, row] = kq.view(torch.uint8), vq.view(torch.uint8)
        s["k_scale"][page, :, row], s["v_scale"][page, :, row] = ks, vs
    else:
        s["k"][page, :, row], s["v"][page, :, row] = k, v
    return _pages(s)


def _gathered(s):
    """K and V of every request as [request][row][head][dim] fp32, and which rows exist."""
    c = s["case"]
    at = torch.arange(s["longest"], device="cuda")
    page = s["table"].long()[:, at // c["page"]].clamp_min(0)
    row = (at % c["page"]).expand_as(page)
    there = at < s["lens"].long()[:, None]
    k, v = s["k"][page, :, row].float(), s["v"][page, :, row].float()
    if c["pages"] in TOP:
        k, v = k * s["k_scale"][page, :, row][..., None], v * s["v_scale"][page, :, row][..., None]
    return k, v, there


def _plain_restore(s):
    c = s["case"]
    if c["write"]:
        _plain_append(s)
    k, v, there = _gathered(s)
    there = there[:, None, :, None]
    return {n: torch.where(there, x.transpose(1, 2), torch.zeros((), device="cuda")).to(TYPES[c["elem"]]).contiguous()
            for n, x in (("k", k), ("v", v))}


def _plain_attend(s):
    c = s["case"]
    B, n, L, G, R, d = c["requests"], s["most"], s["longest"], s["kv_heads"], c["group"], c["dim"]
    k, v, there = _gathered(s)
    starts, lens = s["starts"].long(), s["lens"].long()
    count = starts[1:] - starts[:-1]
    i = torch.arange(n, device="cuda")
    real = i < count[:, None]                                            # [B][n]
    token = torch.where(real, starts[:-1, None] + i, s["total"])         # the last row of the padded tensors is nobody's
    q = torch.cat([s["queries"].float(), torch.zeros(1, G * R, d, device="cuda")])[token]
    q = q.view(B, n, G, R, d).permute(0, 2, 1, 3, 4).reshape(B * G, n * R, d)
    score = torch.bmm(q, k.permute(0, 2, 3, 1).reshape(B * G, d, L).contiguous()).view(B, G, n, R, L) * d ** -0.5
    at = (lens - count)[:, None] + i                                     # position of each new token
    row = torch.arange(L, device="cuda")
    see = there[:, None, :].expand(B, n, L)
    if c["causal"]:
        see = see & (row <= at[:, :, None])
    if c["window"]:
        see = see & (row > at[:, :, None] - c["window"])
    score = score.masked_fill_(~see[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp_(score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * G, n * R, L), v.permute(0, 2, 1, 3).reshape(B * G, L, d).contiguous()).view(B, G, n, R, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + torch.log(total))[..., 0]
    out = torch.zeros(s["total"] + 1, G * R, d, device="cuda")
    out[token] = o.permute(0, 2, 1, 3, 4).reshape(B, n, G * R, d)
    out_lse = torch.zeros(s["total"] + 1, G * R, device="cuda")
    out_lse[token] = lse.permute(0, 2, 1, 3).reshape(B, n, G * R)
    out[-1:] = 0
    return {"o": out[:-1].to(s["o"].dtype), "lse": out_lse[:-1].clone()}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _exact_codes(x, top):
    """Codes (before their own rounding) and scale of every row: fp32 by definition, on the host."""
    import numpy as np
    x = x.detach().float().cpu().numpy()
    r = np.maximum(np.abs(x).max(-1, keepdims=True), np.float32(SMALLEST))
    return torch.from_numpy(x * (np.float32(top) / r)), torch.from_numpy(r), torch.from_numpy(r / np.float32(top))


def _exact_rows(x, kind):
    """The values that a row stands for once it is quantised."""
    y, _, scale = _exact_codes(x, TOP[kind])
    code = torch.round(y) if kind == "i8" else y.to(torch.float8_e4m3fn).float()
    return (code.double() * scale.double()).cuda()


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "linear":
        y, r, _ = _exact_codes(s["x"], 127.0)
        q = torch.round(y).double().cuda()
        out = (q @ s["w"].double().t().contiguous()) * (r.double().cuda() / 127.0) * s["w_scale"].double()
        return {"y": out + s["bias"].double() if s["bias"] is not None else out, "q": None, "r": r[:, 0].double().cuda()}
    lens, tokens = _lengths(c)
    h, d, page = s["kv_heads"], c["dim"], c["page"]
    if c["kind"] == "append":
        # int8 codes are whole numbers; the rest are the values that the rows and their scales have
        out = {n: None if x.dtype == torch.int8 else x.double() for n, x in _pages(s).items()}
        for b, first in enumerate(s["starts"][:-1].tolist()):
            at = torch.arange(lens[b] - tokens[b], lens[b], device="cuda")
            to = s["table"][b].long()[at // page]
            for n in ("k", "v"):
                x = s[n + "_new"][first:first + tokens[b]]
                if c["pages"] not in TOP:
                    out[n][to, :, at % page] = x.double()
                    continue
                y, _, scale = _exact_codes(x, TOP[c["pages"]])
                out[n + "_scale"][to, :, at % page] = scale[..., 0].double().cuda()
                if c["pages"] == "e4m3":
                    out[n][to, :, at % page] = y.to(torch.float8_e4m3fn).double().cuda()
        return out

    def cached(b, n, scales):
        pages = s["table"][b, :-(-lens[b] // page)].long()
        x = s[n][pages].double()
        if scales is not None:
            x = x * scales[pages].double()[..., None]
        return x.permute(0, 2, 1, 3).reshape(-1, h, d)[:lens[b]].transpose(0, 1)      # [head][row][dim]

    if c["kind"] == "restore":
        out = {n: torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda") for n in ("k", "v")}
        for b, first in enumerate(s["starts"][:-1].tolist()):
            for n in ("k", "v"):
                if not c["write"]:
                    out[n][b, :, :lens[b]] = cached(b, n, s[n + "_scale"])
                    continue
                x = s[n + "_new"][first:first + lens[b]]
                out[n][b, :, :lens[b]] = (_exact_rows(x, c["pages"]) if c["pages"] in TOP else x.double()).transpose(0, 1)
        return out
    if work(c)["flops"] > 4e12:
        return None
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, first in enumerate(s["starts"][:-1].tolist()):
        k, v = (cached(b, n, s[n + "_scale"]) for n in ("k", "v"))
        n = tokens[b]
        where = torch.arange(lens[b] - n, lens[b], device="cuda")[:, None]
        row = torch.arange(lens[b], device="cuda")[None]
        hidden = torch.zeros(n, lens[b], dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden |= row > where
        if c["window"]:
            hidden |= row <= where - c["window"]
        for j in range(c["heads"]):
            g = j // c["group"]
            z = (s["queries"][first:first + n, j].double() @ k[g].t().contiguous()) / math.sqrt(d)
            z = z.masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(z, -1, keepdim=True)
            o[first:first + n, j] = torch.exp(z - norm) @ v[g]
            lse[first:first + n, j] = norm[:, 0]
    return {"o": o, "lse": lse}
