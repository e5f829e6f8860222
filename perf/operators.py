"""Serving from a compressed cache, as measurable cases: positions rotated into queries and keys, new tokens written to a cache in pages,
rows and pages of caches moved, attention of new tokens over the pages.

A case is one call.  Head shapes are those of `paper_2604_10235_amd/workloads.py` and the tests; lengths, budgets and chunk sizes those of the
compression workloads, and what a server has between its prefill and its steps of one token.

Four operators:
  rotate  rotary positions on the query and key heads of a fused projection, or their gradient (the inverse rotation).
  append  a step's or a chunk's new tokens: queries rotated, keys rotated and stored, values stored, in the cache's type.
  rows    rows and pages of caches: the kept rows of a paged cache into new pages (compact), the compact rows of many chunks into the pages
          of the requests they belong to (store), a paged cache into the dense layout that scores read (load), pages copied for
          requests that fork (copy).
  attend  softmax attention of the new tokens over the pages, with the log-sum-exp of every row.
"""
import math
import random

import numpy as np
import torch

own = False

DEFAULTS = dict(op="attend", q_heads=28, kv_heads=4, head_dim=128, kv="bf16", page=64, layers=1, seqs=1,
                # rotate, append: rotated elements of a head, pairs, frequencies
                tokens=1, rot_dim=128, interleaved=False, scaling="plain", inverse=False, far=0,
                # append, attend: new tokens of a request, tokens in its cache with them
                new_min=1, new=1, kv_min=1, kv_len=2048, causal=True,
                # rows
                how="compact", capacity=0.0625)


def case(name=None, **over):
    c = dict(DEFAULTS, **over)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step's queries and keys, 16 requests: launches and latency are all there is
        case("rotate_step", op="rotate", tokens=16, far=40000),
        # a long prompt of an 8B-shaped model, positions scaled for a long context
        case("rotate_prompt", op="rotate", tokens=32768, q_heads=32, kv_heads=8, scaling="wavelength", far=90000),
        # one new token of each of 64 requests into a bf16 cache
        case("append_step", op="append", seqs=64, kv_min=300, kv_len=9000),
        # chunks of four prompts, odd lengths, into an 8-bit cache; half of each head rotated, in neighbouring pairs
        case("append_chunks_fp8", op="append", q_heads=32, kv_heads=8, seqs=4, new_min=1501, new=4001, kv_min=4100, kv_len=9001, kv="fp8_e4m3", page=32,
             rot_dim=64, interleaved=True, scaling="linear"),
        # all layers of a compressed 32K request, from its pages into new ones
        case("compact_32k", op="rows", how="compact", layers=28, kv_len=32768, page=64),
        # 64 compressed chunks, one after the other, into the pages of the eight requests that they make up
        case("store_chunks", op="rows", how="store", layers=28, seqs=64, kv_min=128, kv_len=2300, capacity=0.5, page=16),
        # the last pages of 24 requests that fork, all layers
        case("fork_pages", op="rows", how="copy", layers=28, seqs=24, kv_min=1, kv_len=1, page=128),
        # one request, one token, a compressed 32K context: the smallest step
        case("attend_one_token", kv_len=2113, page=64),
        # a server's step: 64 requests of half a thousand to 16K tokens, 8-bit cache
        case("attend_steps_fp8", q_heads=32, kv_heads=8, seqs=64, kv_min=500, kv_len=16384, kv="fp8_e4m3", page=32),
        # one request, one token, the longest context
        case("attend_step_128k", kv_len=131072, page=128),
        # a prefill chunk behind 30K cached tokens
        case("attend_chunk_32k", new_min=2048, new=2048, kv_len=32768, page=128),
        # prompts and chunks of odd lengths together, small heads
        case("attend_mixed_d64", q_heads=8, kv_heads=4, head_dim=64, seqs=12, new_min=1, new=1501, kv_min=1600, kv_len=6001, page=16),
    ]


MOST_PAIRS = 28 * 128 * 2048 * 31700          # (query, key) products of attend_chunk_32k
MOST_CACHE = 131072 * 4 * 128                 # elements of K or V of attend_step_128k
MOST_ROWS = 28 * 4 * 2048 * 128               # elements of K or V that compact_32k moves


def log_int(rng, low, high):
    return int(round(2 ** rng.uniform(math.log2(low), math.log2(high))))


def draw(rng):
    op = rng.choice(["attend"] * 5 + ["rotate"] * 2 + ["append"] * 2 + ["rows"] * 3)
    q_heads, kv_heads, head_dim = rng.choice([(28, 4, 128), (28, 4, 128), (32, 8, 128), (8, 2, 128), (14, 2, 128), (4, 4, 64), (8, 4, 64)])
    c = case(op=op, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 16, 32, 64, 128, 256]))
    c["kv"] = "fp8_e4m3" if op != "rotate" and rng.random() < 0.35 else "bf16"
    c["rot_dim"] = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
    c["interleaved"] = rng.random() < 0.35
    c["scaling"] = rng.choice(["plain", "plain", "linear", "base", "wavelength", "ramp"])
    c["far"] = rng.choice([0, 0, 5000, 100000])
    if op == "rotate":
        c["tokens"] = log_int(rng, 1, 32768)
        c["inverse"] = rng.random() < 0.3
        return c
    c["seqs"] = log_int(rng, 1, 64)
    if op == "append":
        steps = rng.random() < 0.5
        c["new"] = 1 if steps else log_int(rng, 2, 4096)
        c["new_min"] = max(1, c["new"] // rng.randint(1, 6))
        c["kv_len"] = c["new"] + log_int(rng, 16, 8192)
        c["kv_min"] = c["new"]
        while c["seqs"] > 1 and (c["seqs"] * c["new"] > 16384 or c["seqs"] * c["kv_len"] > 1 << 18):
            c["seqs"] = (c["seqs"] + 1) // 2
        return c
    if op == "rows":
        c["how"] = rng.choice(["compact", "store", "load", "copy"])
        c["layers"] = log_int(rng, 1, 28)
        c["kv_len"] = 1 if c["how"] == "copy" else log_int(rng, 64, 32768)
        c["kv_min"] = max(1, c["kv_len"] // rng.randint(1, 6))
        c["capacity"] = round(rng.uniform(0.03, 0.5), 3)
        share = c["capacity"] if c["how"] in ("compact", "store") else 1.0
        length = c["page"] if c["how"] == "copy" else c["kv_len"]
        while True:
            per = c["seqs"] * kv_heads * head_dim * length
            if c["layers"] * per * share <= MOST_ROWS and c["layers"] * per <= 16 * MOST_ROWS:
                break
            if c["layers"] > 1:
                c["layers"] //= 2
            else:
                c["seqs"] = max(1, c["seqs"] // 2)
                if c["seqs"] == 1:
                    c["kv_len"] = min(c["kv_len"], 8191)
                    length = min(length, 8191)
        return c
    kind = rng.choice(["step", "step", "few", "chunk", "chunk", "prompt"])
    c["causal"] = rng.random() < 0.8
    c["new"] = 1 if kind == "step" else log_int(rng, 2, 64) if kind == "few" else log_int(rng, 64, 2048)
    c["new_min"] = max(1, c["new"] // rng.randint(1, 5))
    c["kv_len"] = c["new"] if kind == "prompt" else c["new"] + log_int(rng, 16, 65536)
    c["kv_min"] = max(c["new"], c["kv_len"] // rng.randint(1, 8))
    while c["seqs"] > 1 and (c["seqs"] * c["kv_len"] * kv_heads * head_dim > MOST_CACHE or c["seqs"] * c["new"] * c["kv_len"] * q_heads * head_dim > MOST_PAIRS // 2):
        c["seqs"] = (c["seqs"] + 1) // 2 if c["seqs"] > 2 else 1
    c["kv_len"] = max(c["new"], min(c["kv_len"], MOST_PAIRS // 2 // (c["new"] * q_heads * head_dim), MOST_CACHE // (kv_heads * head_dim)))
    c["kv_min"] = min(c["kv_min"], c["kv_len"])
    return c


def spread(c, low, high, salt):
    """One length per request between two bounds: part of the case, the same for every seed."""
    r = random.Random(1000003 * c["seqs"] + 101 * high + low + salt)
    return [high] + [r.randint(low, high) for _ in range(c["seqs"] - 1)]


def new_of(c):
    return spread(c, c["new_min"], c["new"], 1)


def kept_of(c):
    """Tokens in the cache of every request, its new ones among them."""
    return [max(n, k) for n, k in zip(new_of(c), spread(c, c["kv_min"], c["kv_len"], 2))]


def budgets_of(c):
    return [max(1, int(c["capacity"] * n)) for n in spread(c, c["kv_min"], c["kv_len"], 2)]


STORE_GROUP = 8                               # chunks that one request's prompt is made of


def cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def on_gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---------------------------------------------------------------- rotary frequencies

SCALING = dict(factor=4.0, context=8192.0, low=1.0, high=4.0, fast=32.0, slow=1.0)


def frequencies(c):
    """Radians a position, of every pair, in 64 bits."""
    dim, base, s = c["rot_dim"], 10000.0, SCALING
    if c["scaling"] == "base":
        base *= s["factor"] ** (dim / (dim - 2))
    i = np.arange(dim // 2, dtype=np.float64)
    f = base ** (-2.0 * i / dim)
    if c["scaling"] == "linear":
        return f / s["factor"]
    if c["scaling"] == "wavelength":          # turns in the trained context decide: few, slowed down; many, left; between, a blend
        t = np.clip((s["context"] * f / (2 * np.pi) - s["low"]) / (s["high"] - s["low"]), 0.0, 1.0)
        return (1 - t) * f / s["factor"] + t * f
    if c["scaling"] == "ramp":                # the same by the pair's number, on a line between two of them
        at = lambda turns: dim * np.log(s["context"] / (turns * 2 * np.pi)) / (2 * np.log(base))  # noqa: E731
        a, b = max(np.floor(at(s["fast"])), 0.0), min(np.ceil(at(s["slow"])), dim - 1.0)
        t = np.clip((i - a) / max(b - a, 0.001), 0.0, 1.0)
        return t * f / s["factor"] + (1 - t) * f
    return f


def magnitude(c):
    return 0.1 * math.log(SCALING["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def rotated(x, positions, freq, c):
    """Plain form: x float32 [T, H, d]."""
    a = positions.double()[:, None] * freq[None, :]
    if c["inverse"]:
        a = -a
    m = magnitude(c)
    cos, sin = (m * a.cos()).float()[:, None, :], (m * a.sin()).float()[:, None, :]
    dim, out = c["rot_dim"], x.clone()
    x0, x1 = (x[..., 0:dim:2], x[..., 1:dim:2]) if c["interleaved"] else (x[..., : dim // 2], x[..., dim // 2 : dim])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    if c["interleaved"]:
        out[..., 0:dim:2], out[..., 1:dim:2] = y0, y1
    else:
        out[..., : dim // 2], out[..., dim // 2 : dim] = y0, y1
    return out


def turned(x, positions, freq, c):
    """The same in 64 bits: complex numbers times exp(i a)."""
    dim = c["rot_dim"]
    a = (-1.0 if c["inverse"] else 1.0) * positions.to(torch.float64)[:, None] * freq[None, :]
    turn = magnitude(c) * torch.polar(torch.ones_like(a), a)[:, None, :]
    head = x[..., :dim].double()
    pairs = head.unflatten(-1, (dim // 2, 2)) if c["interleaved"] else head.unflatten(-1, (2, dim // 2)).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = y.flatten(-2) if c["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., dim:].double()], -1)


# ---------------------------------------------------------------- inputs

K_SCALE, V_SCALE = 0.02, 0.0125               # of the 8-bit cache: a value is its code times this


def pool(c, pages, gen, layers):
    """K or V pages [layers, pages, heads, page, d] of N(0, 1) rows, in the cache's type."""
    shape = (pages, c["kv_heads"], c["page"], c["head_dim"])
    out = torch.empty((layers, *shape), dtype=torch.float8_e4m3fn if c["kv"] == "fp8_e4m3" else torch.bfloat16, device="cuda")
    for x in out:
        x.copy_(torch.randn(shape, generator=gen, device="cuda") * (40.0 if c["kv"] == "fp8_e4m3" else 1.0))
    return out


def table_of(c, lengths, gen, more=1.13):
    """Page table [requests, width] over pages in no order, and how many pages the pool has (some are nobody's)."""
    need = [-(-n // c["page"]) for n in lengths]
    pages = int(sum(need) * more) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device="cuda")
    held = torch.arange(max(need), device="cuda")[None, :] < torch.tensor(need, device="cuda")[:, None]
    table[held] = order[: sum(need)]
    return table, pages


def prepare(c, seed):
    c = dict(DEFAULTS, **c)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    {"rotate": prepare_rotate, "append": prepare_append, "rows": prepare_rows, "attend": prepare_attend}[c["op"]](c, s, gen)
    return s


def rotary_handle(c):
    from paper_2604_10235_amd import binding as cc
    p = SCALING
    return cc.make_rotary(c["rot_dim"], base=10000.0, interleaved=c["interleaved"], inverse=c["inverse"], scaling=cc.ROTARY_SCALINGS[c["scaling"]],
                          factor=p["factor"], context=p["context"], low=p["low"] if c["scaling"] == "wavelength" else p["slow"],
                          high=p["high"] if c["scaling"] == "wavelength" else p["fast"], magnitude=magnitude(c))


def pages_handle(c, s):
    from paper_2604_10235_amd import binding as cc
    fp8 = c["kv"] == "fp8_e4m3"
    return cc.make_pages(s["k_pages"], s["v_pages"], k_scale=K_SCALE if fp8 else 1.0, v_scale=V_SCALE if fp8 else 1.0)


def prepare_rotate(c, s, gen):
    T, heads = c["tokens"], c["q_heads"] + c["kv_heads"]
    fused = torch.randn((T, heads + c["kv_heads"], c["head_dim"]), generator=gen, device="cuda").bfloat16()
    s["x"] = fused[:, :heads]                 # the projection's value heads lie behind them
    s["positions"] = (torch.randint(0, 7 * T + 1, (1,), generator=gen, device="cuda") + c["far"] + torch.arange(T, device="cuda")).int()
    if T <= 64:                               # a step: every token is of another request
        s["positions"] = torch.randint(0, c["far"] + 4096, (T,), generator=gen, device="cuda").int()
    s["out"] = torch.empty((T, heads, c["head_dim"]), dtype=torch.bfloat16, device="cuda")
    s["freq"] = on_gpu(frequencies(c))
    if own:
        s["rotary"] = rotary_handle(c)


def batch_of(c, s, gen, q_stride=0, new_stride=0):
    """Cache and new tokens of every request: pages, table, lengths, packed token offsets."""
    news, kept = new_of(c), kept_of(c)
    s["table"], pages = table_of(c, kept, gen)
    s["k_pages"], s["v_pages"] = pool(c, pages, gen, c["layers"]), pool(c, pages, gen, c["layers"])
    s["kv_lens"], s["cu"] = on_gpu(np.array(kept, np.int32)), on_gpu(cu(news))
    s["news"], s["kept"] = news, kept
    if own:
        from paper_2604_10235_amd import binding as cc
        s["pages"] = pages_handle(c, s)
        s["batch"] = cc.make_batch(n_q_heads=c["q_heads"], cu_q_host=cu(news), cu_q=s["cu"], kv_lens=s["kv_lens"], table=s["table"], max_kv_len=max(kept),
                                   causal=c["causal"], q_stride_tok=q_stride, new_stride_tok=new_stride)


def prepare_append(c, s, gen):
    d, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    batch_of(c, s, gen, (Hq + 2 * Hkv) * d, (Hq + 2 * Hkv) * d)
    T = sum(s["news"])
    fused = torch.randn((T, Hq + 2 * Hkv, d), generator=gen, device="cuda").bfloat16()
    s["q"], s["k"], s["v"] = fused[:, :Hq], fused[:, Hq : Hq + Hkv], fused[:, Hq + Hkv :]
    # the new tokens lie behind what was compressed: positions further than the cache is long
    s["of"] = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), on_gpu(np.array(s["news"])), output_size=T)
    s["slot"] = torch.arange(T, device="cuda") - s["cu"][s["of"] + 1] + s["kv_lens"][s["of"]]
    s["positions"] = (s["slot"] + c["far"] + torch.randint(0, 50000, (c["seqs"],), generator=gen, device="cuda")[s["of"]]).int()
    s["q_out"] = torch.empty((T, Hq, d), dtype=torch.bfloat16, device="cuda")
    s["freq"] = on_gpu(frequencies(c))
    if own:
        s["rotary"] = rotary_handle(c)


def prepare_attend(c, s, gen):
    batch_of(c, s, gen)
    T = sum(s["news"])
    # logits of a few units, some queries that look at single keys
    sharp = 1.0 + 2.0 * (torch.rand((T, c["q_heads"], 1), generator=gen, device="cuda") < 0.1)
    s["q"] = (sharp * torch.randn((T, c["q_heads"], c["head_dim"]), generator=gen, device="cuda")).bfloat16()
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((T, c["q_heads"]), dtype=torch.float32, device="cuda")
    if own:
        from paper_2604_10235_amd import binding as cc
        s["workspace"] = torch.empty(max(256, cc.codecomp_attend_workspace_bytes(s["batch"], s["pages"])), dtype=torch.uint8, device="cuda")


def prepare_rows(c, s, gen):
    H, L, d, how = c["kv_heads"], c["layers"], c["head_dim"], c["how"]
    if how == "copy":                         # the last page of every request that forks, into one of its own
        n = c["seqs"]
        order = torch.randperm(3 * n + 5, generator=gen, device="cuda").int()
        s["k_pages"], s["v_pages"] = pool(c, 3 * n + 5, gen, L), pool(c, 3 * n + 5, gen, L)
        s["pairs"] = order[: 2 * n].view(n, 2).contiguous()
        if own:
            s["pages"] = pages_handle(c, s)
        return
    lengths, budgets = spread(c, c["kv_min"], c["kv_len"], 2), budgets_of(c)
    rows = budgets if how == "compact" else budgets if how == "store" else lengths
    s["rows"], s["cu_rows"] = rows, on_gpu(cu(rows))
    T, TB = sum(lengths), sum(rows)
    if how == "compact":
        s["from_table"], pages = table_of(c, lengths, gen)
        s["from_k"], s["from_v"] = pool(c, pages, gen, L), pool(c, pages, gen, L)
        near = torch.rand((L, H, T), generator=gen, device="cuda")
        s["idx"] = torch.cat([near[:, :, a : a + n].topk(b, dim=2).indices.sort(dim=2).values for a, n, b in zip(cu(lengths), lengths, budgets)], 2).int().contiguous()
    else:
        dense = lambda: pool(dict(c, page=TB), 1, gen, L)[:, 0]  # noqa: E731  [layers, heads, TB, d]
        s["k"], s["v"] = dense(), dense()
    if how == "store":                        # chunk r goes behind the chunks before it of the same request
        of = [r // STORE_GROUP for r in range(c["seqs"])]
        first = [sum(rows[STORE_GROUP * o : r]) for r, o in enumerate(of)]
        table, pages = table_of(c, [sum(rows[STORE_GROUP * o : STORE_GROUP * (o + 1)]) for o in range(of[-1] + 1)], gen)
        s["table"], s["first"] = table[on_gpu(np.array(of))].contiguous(), on_gpu(np.array(first, np.int32))
    else:
        s["table"], pages = table_of(c, rows, gen)
        s["first"] = torch.zeros(c["seqs"], dtype=torch.int32, device="cuda")
    s["k_pages"], s["v_pages"] = pool(c, pages, gen, L), pool(c, pages, gen, L)
    if own:
        from paper_2604_10235_amd import binding as cc
        s["pages"] = pages_handle(c, s)
        if how == "compact":
            s["from"] = pages_handle(c, {"k_pages": s["from_k"], "v_pages": s["from_v"]})
        s["cu_tokens"] = on_gpu(cu(lengths))
        s["params"] = cc.make_params(n_layers=L, n_q_heads=c["q_heads"], n_kv_heads=H, head_dim=d, window=1, pool_kernel=1, prior_weight=0.0,
                                     cu_seqlens_host=cu(lengths), cu_budgets_host=cu(rows), cu_seqlens_dev=s["cu_tokens"].data_ptr(),
                                     cu_budgets_dev=s["cu_rows"].data_ptr(), kv_dtype=cc.KV_FP8_E4M3 if c["kv"] == "fp8_e4m3" else cc.KV_BF16)


# ---------------------------------------------------------------- one pass

def run(s):
    return {"rotate": run_rotate, "append": run_append, "rows": run_rows, "attend": run_attend}[s["case"]["op"]](s)


def run_rotate(s):
    if own:
        from paper_2604_10235_amd import binding as cc
        cc.codecomp_rotate(s["x"], s["positions"], s["rotary"], s["out"])
    else:
        s["out"].copy_(rotated(s["x"].float(), s["positions"], s["freq"], s["case"]))
    return {"out": s["out"]}


def to_cache(x, scale, like):
    return (x / scale).clamp(-448.0, 448.0).to(like.dtype).view(torch.uint8) if like.dtype == torch.float8_e4m3fn else x.to(like.dtype)


def bits(x):
    """8-bit floats as bytes, which can be indexed."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def run_append(s):
    c = s["case"]
    if own:
        from paper_2604_10235_amd import binding as cc
        cc.codecomp_append(s["q"], s["k"], s["v"], s["positions"], s["rotary"], s["batch"], s["pages"], 0, s["q_out"])
    else:
        s["q_out"].copy_(rotated(s["q"].float(), s["positions"], s["freq"], c))
        page, at = s["table"][s["of"], s["slot"] // c["page"]].long(), s["slot"] % c["page"]
        bits(s["k_pages"])[0][page, :, at] = to_cache(rotated(s["k"].float(), s["positions"], s["freq"], c), K_SCALE, s["k_pages"])
        bits(s["v_pages"])[0][page, :, at] = to_cache(s["v"].float(), V_SCALE, s["v_pages"])
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def places(s, table, rows, cu_rows, first):
    """(page, row in it) of every packed row of the requests."""
    page = s["case"]["page"]
    of = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), cu_rows.diff(), output_size=sum(rows))
    slot = torch.arange(sum(rows), device="cuda") - cu_rows[of] + first[of]
    return of, table[of, slot // page].long(), slot % page


def run_rows(s):
    c = s["case"]
    if c["how"] == "copy":
        if own:
            from paper_2604_10235_amd import binding as cc
            cc.codecomp_pages_copy(s["pages"], s["pairs"])
        else:
            a, b = s["pairs"].long().unbind(1)
            bits(s["k_pages"])[:, b] = bits(s["k_pages"])[:, a]
            bits(s["v_pages"])[:, b] = bits(s["v_pages"])[:, a]
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if own:
        from paper_2604_10235_amd import binding as cc
        if c["how"] == "compact":
            cc.codecomp_pages_compact(s["from"], s["from_table"], None, s["idx"], s["params"], s["pages"], s["table"], None)
        elif c["how"] == "store":
            cc.codecomp_pages_store(s["k"], s["v"], None, s["params"], s["pages"], s["table"], s["first"])
        else:
            cc.codecomp_pages_load(s["pages"], s["table"], None, None, s["params"], s["k"], s["v"])
        return {"k": s["k"], "v": s["v"]} if c["how"] == "load" else {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    of, page, at = places(s, s["table"], s["rows"], s["cu_rows"], s["first"])
    if c["how"] == "load":
        bits(s["k"]).copy_(bits(s["k_pages"])[:, page, :, at].permute(1, 2, 0, 3))
        bits(s["v"]).copy_(bits(s["v_pages"])[:, page, :, at].permute(1, 2, 0, 3))
        return {"k": s["k"], "v": s["v"]}
    if c["how"] == "compact":                 # kept rows differ from layer to layer and from head to head
        layer = torch.arange(c["layers"], device="cuda")[:, None, None]
        head = torch.arange(c["kv_heads"], device="cuda")[None, :, None]
        there = s["from_table"][of[None, None, :], s["idx"].long() // c["page"]].long()
        k, v = (bits(x)[layer, there, head, s["idx"].long() % c["page"]] for x in (s["from_k"], s["from_v"]))
    else:
        k, v = bits(s["k"]), bits(s["v"])
    bits(s["k_pages"])[:, page, :, at] = k.permute(2, 0, 1, 3)
    bits(s["v_pages"])[:, page, :, at] = v.permute(2, 0, 1, 3)
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def run_attend(s):
    if own:
        from paper_2604_10235_amd import binding as cc
        cc.codecomp_attend(s["q"], s["batch"], s["pages"], 0, s["out"], s["workspace"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    c = s["case"]
    n, H, G, d = c["seqs"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    most, longest, fp8 = max(s["news"]), max(s["kept"]), c["kv"] == "fp8_e4m3"
    key, new = torch.arange(longest, device="cuda"), torch.arange(most, device="cuda")
    page, at = s["table"][:, key // c["page"]].clamp_min(0).long(), (key % c["page"])[None, :]
    held = key[None, :] < s["kv_lens"][:, None]
    rows = lambda p, scale: (bits(p)[0][page, :, at].view(p.dtype).float().mul_(scale).masked_fill_(~held[:, :, None, None], 0.0)).transpose(1, 2).contiguous()  # noqa: E731
    k, v = rows(s["k_pages"], K_SCALE if fp8 else 1.0), rows(s["v_pages"], V_SCALE if fp8 else 1.0)                 # [n, H, longest, d]
    counts = s["cu"].diff()
    there = new[None, :] < counts[:, None]                                                                          # [n, most]
    q = torch.zeros((n, most, H, G, d), device="cuda")
    q[there] = s["q"].float().unflatten(1, (H, G))
    q = q.permute(0, 2, 1, 3, 4).reshape(n, H, most * G, d)
    logits = (q @ k.transpose(2, 3)).mul_(d ** -0.5).view(n, H, most, G, longest)
    last = s["kv_lens"][:, None] - counts[:, None] + new[None, :] + 1 if c["causal"] else s["kv_lens"][:, None].expand(n, most)
    hidden = key[None, None, :] >= torch.minimum(last, s["kv_lens"][:, None])[:, :, None]                           # [n, most, longest]
    logits.masked_fill_(hidden[:, None, :, None, :], -torch.inf)
    top = logits.amax(-1, keepdim=True).clamp_min(-1e30)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(n, H, most * G, longest) @ v).view(n, H, most, G, d) / total.clamp_min(1e-30)
    lse = (total.log() + top)[..., 0]
    s["out"].copy_(out.permute(0, 2, 1, 3, 4)[there].flatten(1, 2))
    s["lse"].copy_(lse.permute(0, 2, 1, 3)[there].flatten(1, 2))
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- work and exact values

def work(c):
    c = dict(DEFAULTS, **c)
    d, Hq, Hkv, esz = c["head_dim"], c["q_heads"], c["kv_heads"], 1 if c["kv"] == "fp8_e4m3" else 2
    if c["op"] == "rotate":
        vectors = c["tokens"] * (Hq + Hkv)
        return {"bytes": 4 * vectors * d + 4 * c["tokens"], "flops": 3 * vectors * c["rot_dim"]}
    if c["op"] == "append":
        T = sum(new_of(c))
        return {"bytes": T * (2 * d * (2 * Hq + 2 * Hkv) + 2 * d * Hkv * esz + 4), "flops": 3 * T * (Hq + Hkv) * c["rot_dim"]}
    if c["op"] == "rows":
        if c["how"] == "copy":
            rows = c["seqs"] * c["page"]
        else:
            rows = sum(spread(c, c["kv_min"], c["kv_len"], 2) if c["how"] == "load" else budgets_of(c))
        return {"bytes": c["layers"] * Hkv * rows * (4 * d * esz + (4 if c["how"] == "compact" else 0)), "flops": 0}
    news, kept = new_of(c), kept_of(c)
    pairs = sum(n * k - (n * (n - 1) // 2 if c["causal"] else 0) for n, k in zip(news, kept))
    return {"bytes": 2 * sum(kept) * Hkv * d * esz + sum(news) * Hq * (4 * d + 4), "flops": 4 * pairs * Hq * d}


def exact(c, seed):
    """Copies of rows have nothing computed: no value in 64 bits is asked for."""
    c = dict(DEFAULTS, **c)
    if c["op"] == "rows":
        return None
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "rotate":
        return {"out": turned(s["x"], s["positions"], s["freq"], c)}
    fp8 = c["kv"] == "fp8_e4m3"
    if c["op"] == "append":
        q, k, v = turned(s["q"], s["positions"], s["freq"], c), turned(s["k"], s["positions"], s["freq"], c), s["v"].double()
        pools = []
        for pages, x, scale in ((s["k_pages"], k, K_SCALE), (s["v_pages"], v, V_SCALE)):
            whole = pages.to(torch.float64) if not fp8 else pages.float().double()
            for r in range(c["seqs"]):
                a, n, at = int(s["cu"][r]), s["news"][r], s["kept"][r] - s["news"][r]
                slot = torch.arange(at, at + n, device="cuda")
                whole[0, s["table"][r].long()[slot // c["page"]], :, slot % c["page"]] = (x[a : a + n] / scale).clamp(-448.0, 448.0) if fp8 else x[a : a + n]
            pools.append(whole)
        return {"q": q, "k_pages": pools[0], "v_pages": pools[1]}
    T, Hq, d, G = sum(s["news"]), c["q_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"]
    out, lse = torch.zeros((T, Hq, d), dtype=torch.float64, device="cuda"), torch.full((T, Hq), -torch.inf, dtype=torch.float64, device="cuda")
    for r in range(c["seqs"]):
        a, n, kept = int(s["cu"][r]), s["news"][r], s["kept"][r]
        slots = torch.arange(kept, device="cuda")
        of_request = lambda p, scale: bits(p)[0][s["table"][r].long()[slots // c["page"]], :, slots % c["page"]].view(p.dtype).float().double() * scale  # noqa: E731
        k, v = of_request(s["k_pages"], K_SCALE if fp8 else 1.0), of_request(s["v_pages"], V_SCALE if fp8 else 1.0)
        limit = torch.arange(kept - n + 1, kept + 1, device="cuda") if c["causal"] else torch.full((n,), kept, device="cuda")
        for h in range(Hq):
            z = (s["q"][a : a + n, h].double() @ k[:, h // G].T) / math.sqrt(d)
            z = torch.where(slots[None, :] < limit[:, None], z, -torch.inf)
            lse[a : a + n, h] = torch.logsumexp(z, 1)
            out[a : a + n, h] = torch.softmax(z, 1) @ v[:, h // G]
    return {"out": out, "lse": lse}
