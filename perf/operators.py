"""The operators of a serving step on a paged KV cache, as they are measured: writing new tokens' K and V into the pages
(bf16, or e4m3 in blocks of 32 channels), reading cached rows back, and the layer's attention of new tokens over the pages.

  write    l2a_cache_write:  k, v [N, Hkv, D] of the packed new tokens -> rows of the sequences' pages
  read     l2a_cache_read:   rows of the sequences' pages -> k, v [N, Hkv, D]
  extend   l2a_attn_extend:  q [N, Hq, D] of the packed new tokens against their sequences' pages, Local attention over the last
           W + 1 keys of every token, Global attention over all keys up to a routed token, o = s + d a

Head layouts, windows and routed fractions are those of the workloads in paper_2603_17484_amd/inputs.py and of the decode
cases in perf/cases.py.  Tensors are N(0,1), as everywhere in this repository; pages are handed out in random order.  The
sequences' lengths follow from the case alone, everything else from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
BLOCK = 32  # channels that share a scale in an fp8 cache


# --------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------
def case_of(kind, name=None, **kw):
    """B sequences, `new` tokens each (`chunk`: the first one's number where it differs) behind up to `cached` tokens; page: tokens
    of a page; dtype: the cache's elements; f: routed fraction; mask_heads: 1, or a decision per query head; ragged: lengths
    differ from sequence to sequence."""
    case = {"kind": kind, "B": 1, "new": 1, "chunk": 0, "cached": 0, "heads": 28, "kv": 4, "page": 64, "dtype": "bf16",
            "W": 4096, "f": 0.2, "mask_heads": 1, "ragged": False}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a generation step's new rows, one per sequence of a wide batch: latency
        case_of("write", "write_64x1_bf16", B=64, cached=8192, ragged=True),
        # a long prefill chunk quantised as it is written
        case_of("write", "write_8k_fp8", new=8192, cached=5, heads=32, kv=8, page=256, dtype="fp8"),
        # a few short cached prefixes handed back, small pages, odd lengths
        case_of("read", "read_7x1501_bf16", B=7, new=1501, page=16, ragged=True),
        # a long cached prefix handed back whole
        case_of("read", "read_64k_fp8", new=65536, heads=32, kv=8, dtype="fp8"),
        # one conversation being generated, its token routed: latency of a step
        case_of("extend", "decode_1x32k_bf16", cached=32767, f=1.0),
        # a wide serving batch on a cache of 8 bits
        case_of("extend", "decode_64x8k_fp8", B=64, cached=8191, heads=32, kv=8, dtype="fp8", ragged=True),
        # drafts of five tokens checked at once, small pages
        case_of("extend", "draft_16x5_32k_bf16", B=16, new=5, cached=32000, page=16, ragged=True),
        # first chunks of three prompts of odd lengths, a decision per head, a short window
        case_of("extend", "first_3x777_bf16", B=3, new=777, W=100, mask_heads=28, page=16, ragged=True),
        # a prefill chunk in the middle of a long prompt
        case_of("extend", "chunk_2k_at_32k_bf16", new=2048, cached=32768),
        # the same of the layer with 32 / 8 heads on a cache of 8 bits
        case_of("extend", "chunk_2k_at_32k_fp8", new=2048, cached=32768, heads=32, kv=8, dtype="fp8"),
        # a chunk of one prompt beside the steps of 31 sequences
        case_of("extend", "mixed_32_at_16k_fp8", B=32, chunk=1001, cached=16000, dtype="fp8", ragged=True),
        # a large chunk near the end of a very long prompt
        case_of("extend", "chunk_4k_at_124k_bf16", new=4096, cached=126976),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, kv = rng.choice([(28, 4), (32, 8), (16, 16), (12, 1)])
    more = {"heads": heads, "kv": kv, "page": rng.choice([16, 32, 64, 128, 256]), "dtype": rng.choice(["bf16", "fp8"]),
            "ragged": rng.random() < 0.7}
    kind = rng.choice(["write", "read", "decode", "draft", "chunk", "mixed"])
    if kind in ("write", "read"):
        B = log(1, 64)
        return case_of(kind, B=B, new=log(1, 65536 // B), cached=log(1, 4096), **more)
    more.update(W=log(1, 8192), f=rng.choice([0.0, 0.1, 0.2, 0.5, 1.0]), mask_heads=rng.choice([1, heads]))
    if kind == "decode":
        B = log(1, 128)
        return case_of("extend", B=B, cached=log(16, min(131072, (1 << 19) // B)), **more)
    if kind == "draft":
        B = log(1, 32)
        return case_of("extend", B=B, new=rng.randint(2, 9), cached=log(16, min(65536, (1 << 18) // B)), **more)
    if kind == "chunk":
        B = rng.randint(1, 4)
        return case_of("extend", B=B, new=log(10, 4096 // B), cached=log(1, 32768 // B), **more)
    return case_of("extend", B=rng.randint(2, 48), chunk=log(16, 2048), cached=log(16, 16384), **more)


def lengths(case):
    """(new tokens, tokens cached before them) of every sequence."""
    spread = [1.0 - 0.5 * (i * 0.6180339887 % 1.0) if case["ragged"] else 1.0 for i in range(case["B"])]
    new = [max(1, int(case["new"] * s)) for s in spread]
    if case["chunk"]:
        new[0] = case["chunk"]
    return new, [int(case["cached"] * s) for s in spread[::-1]]


# --------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new, cached = lengths(case)
    B, N, kv, page = case["B"], sum(new), case["kv"], case["page"]
    held = [-(-(n + c) // page) for n, c in zip(new, cached)]
    pages = sum(held)
    order = torch.randperm(pages, generator=g, device=DEV, dtype=torch.int32)
    table = torch.zeros(B, max(held), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    state = {"case": case, "table": table, "new": new, "cached": cached, "max_new": max(new),
             "start": torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEV),
             "pos": torch.tensor(cached, dtype=torch.int32, device=DEV)}

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)

    if case["kind"] == "write":
        state.update(k=normal(N, kv, D), v=normal(N, kv, D))
        pools = [torch.zeros(pages, kv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    else:
        pools = [normal(pages, kv, page, D) for _ in range(2)]
    if case["dtype"] == "fp8":
        (state["pk"], state["sk"]), (state["pv"], state["sv"]) = (quantise(x) for x in pools)
    else:
        state.update(pk=pools[0], sk=None, pv=pools[1], sv=None)
    if case["kind"] == "read":
        state.update(k=torch.empty(N, kv, D, dtype=torch.bfloat16, device=DEV), v=torch.empty(N, kv, D, dtype=torch.bfloat16, device=DEV))
    if case["kind"] == "extend":
        state["q"] = normal(N, case["heads"], D)
        # round(f N) of the N decisions of every mask head
        mask = torch.zeros(case["mask_heads"], N, dtype=torch.uint8, device=DEV)
        for h in range(case["mask_heads"]):
            mask[h, torch.randperm(N, generator=g, device=DEV)[:round(case["f"] * N)]] = 1
        state["mask"] = mask
    return state


# --------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------
def quantise(x):
    """[..., D] -> e4m3 elements and [..., D / 32] exponents (biased by 127): per block of 32 channels the least power of two with
    which no element passes 448."""
    blocks = x.float().unflatten(-1, (-1, BLOCK))
    amax = blocks.abs().amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -118).clamp(-118, 119).int()
    return torch.ldexp(blocks, -e.unsqueeze(-1)).flatten(-2).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def values(elements, exponents):
    if exponents is None:
        return elements.float()
    return torch.ldexp(elements.float().unflatten(-1, (-1, BLOCK)), exponents.unsqueeze(-1).int() - 127).flatten(-2)


def places(s):
    """Page and row within it of every new token."""
    token = torch.arange(sum(s["new"]), device=DEV, dtype=torch.int32)
    b = torch.searchsorted(s["start"][1:].contiguous(), token, right=True)
    at = s["pos"][b] + token - s["start"][b]
    page = s["case"]["page"]
    return s["table"][b, torch.div(at, page, rounding_mode="floor")].long(), (at % page).long()


def write_plain(s):
    page, row = places(s)
    for x, pool, scale in ((s["k"], s["pk"], s["sk"]), (s["v"], s["pv"], s["sv"])):
        if scale is None:
            pool[page, :, row] = x
        else:
            q, e = quantise(x)
            pool.view(torch.uint8)[page, :, row] = q.view(torch.uint8)
            scale[page, :, row] = e


def read_plain(s):
    page, row = places(s)
    for x, pool, scale in ((s["k"], s["pk"], s["sk"]), (s["v"], s["pv"], s["sv"])):
        elements = pool.view(torch.uint8)[page, :, row].view(pool.dtype) if scale is not None else pool[page, :, row]
        x.copy_(values(elements, None if scale is None else scale[page, :, row]))


def rows_of(s, pool, scale, b, first, last):
    """Rows first .. last - 1 of sequence b's cache, [Hkv, rows, D] in 32 bits."""
    page = s["case"]["page"]
    t = s["table"][b, first // page:-(-last // page)].long()
    x = values(pool.view(torch.uint8)[t].view(pool.dtype) if scale is not None else pool[t], None if scale is None else scale[t])
    return x.transpose(0, 1).flatten(1, 2)[:, first - first // page * page:][:, :last - first]


def attend(q, k, v, lo, hi):
    """q [Hkv, rows, D], k, v [Hkv, keys, D]; row i sees keys lo[i] .. hi[i]."""
    key = torch.arange(k.shape[1], device=DEV)
    p = torch.matmul(q, k.transpose(1, 2)) * (1.0 / math.sqrt(D))
    p = p.masked_fill_((key < lo[:, None]) | (key > hi[:, None]), -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total


def extend_plain(s):
    c = s["case"]
    kv, G, W = c["kv"], c["heads"] // c["kv"], c["W"]
    out = torch.empty_like(s["q"])
    at = 0
    for b, (n, before) in enumerate(zip(s["new"], s["cached"])):
        first = max(before - W, 0)
        some = s["mask"].shape[1] and bool(c["f"] > 0)
        k, v = (rows_of(s, s[x], s[y], b, 0 if some else first, before + n) for x, y in (("pk", "sk"), ("pv", "sv")))
        base = 0 if some else first
        step = max(1, (1 << 30) // (c["heads"] * (before + n)))  # rows at a time: at most 4 GB of scores
        for t in range(0, n, step):
            cnt = min(step, n - t)
            q = s["q"][at + t:at + t + cnt].float().view(cnt, kv, G, D)
            pos = before + t + torch.arange(cnt, device=DEV)
            lo, hi = (pos - W).clamp(min=0), pos
            keys = slice(max(before + t - W, 0) - base, before + t + cnt - base)
            rows = q.permute(1, 0, 2, 3).reshape(kv, cnt * G, D)
            o = attend(rows, k[:, keys], v[:, keys], (lo - base - keys.start).repeat_interleave(G), (hi - base - keys.start).repeat_interleave(G))
            o = o.view(kv, cnt, G, D).permute(1, 0, 2, 3)
            if some:
                d = s["mask"][:, at + t:at + t + cnt] != 0
                who = d.any(0).nonzero().flatten()
                m = who.numel()
                if m:
                    rows = q[who].permute(1, 0, 2, 3).reshape(kv, m * G, D)
                    a = attend(rows, k[:, :before + t + cnt], v[:, :before + t + cnt], torch.zeros(m * G, device=DEV), hi[who].repeat_interleave(G))
                    a = a.view(kv, m, G, D).permute(1, 0, 2, 3)
                    a = a * d[:, who].t().expand(m, c["heads"]).reshape(m, kv, G, 1)
                    o = o.index_add(0, who, a)
            out[at + t:at + t + cnt] = o.reshape(cnt, c["heads"], D)
        at += n
    return out


# --------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------
def handle(s):
    """The description of the cache, the sizes and the workspace that a serving program keeps."""
    from paper_2603_17484_amd import binding as B
    if "handle" not in s:
        c = s["case"]
        cache = B.make_cache(s["pk"], s["pv"], s["table"], s["sk"], s["sv"])
        p = B.make_params(c["B"], sum(s["new"]), c["heads"], c["kv"], D, c["W"], c["mask_heads"])
        kept = None
        if c["kind"] == "extend":
            kept = (torch.empty_like(s["q"]), B.alloc_extend_workspace(p, cache, s["max_new"]))
        s["handle"] = B, cache, p, kept
    return s["handle"]


def run(state):
    kind = state["case"]["kind"]
    if own:
        B, cache, p, kept = handle(state)
        if kind == "write":
            B.l2a_cache_write(p, cache, state["k"], state["v"], state["start"], state["pos"])
        elif kind == "read":
            B.l2a_cache_read(p, cache, state["start"], state["pos"], state["k"], state["v"])
        else:
            out, workspace = kept
            B.l2a_attn_extend(p, cache, state["q"], state["start"], state["pos"], state["mask"], state["max_new"], out, workspace=workspace)
            return out
    elif kind == "write":
        write_plain(state)
    elif kind == "read":
        read_plain(state)
    else:
        return extend_plain(state)
    if kind == "write":
        return [state[x] for x in ("pk", "pv", "sk", "sv") if state[x] is not None]
    return state["k"], state["v"]


# --------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------
def work(case):
    new, cached = lengths(case)
    row = (2 * D if case["dtype"] == "bf16" else D + D // BLOCK) * 2 * case["kv"]  # K and V of a token in the cache
    if case["kind"] != "extend":
        return {"bytes": sum(new) * (row + 2 * 2 * D * case["kv"]), "flops": 0}
    W, f, heads = case["W"], case["f"], case["heads"]
    # that some decision of a token is 1, and of some token of a sequence
    some = f if case["mask_heads"] == 1 else 1.0 - (1.0 - f) ** (heads // case["kv"])
    pairs = rows = 0.0
    for n, before in zip(new, cached):
        ts = (before, before + n - 1)
        total = n * (ts[0] + ts[1] + 2) / 2  # sum of t + 1
        lost = [max(t - W, 0) for t in ts]   # keys before the window: a run of numbers behind some zeros
        m = min(n, lost[1])
        before_window = m * (lost[1] - m + 1 + lost[1]) / 2
        pairs += (total - before_window) + f * before_window
        first = max(before - W, 0)
        rows += before + n - first + first * (1.0 - (1.0 - some) ** n)
    return {"bytes": rows * row + sum(new) * heads * D * 2 * 2, "flops": 4 * D * heads * pairs}


# --------------------------------------------------------------------------------------
# the definition, in 64 bits
# --------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    new, cached, page = s["new"], s["cached"], case["page"]
    start = [sum(new[:b]) for b in range(case["B"] + 1)]
    table = s["table"].cpu().tolist()

    def cell(b, t):
        return table[b][t // page] * page + t % page

    def cells(b, t0, t1):
        return torch.tensor([cell(b, t) for t in range(t0, t1)], device=DEV)

    def flat(pool):  # [rows of all pages, Hkv, ...]
        return pool.transpose(1, 2).flatten(0, 1)

    def real(pool, scale):
        x = flat(pool).double()
        if scale is None:
            return x
        return x * torch.exp2(flat(scale).double() - 127.0).repeat_interleave(BLOCK, -1)

    if case["kind"] == "write":
        where = torch.cat([cells(b, cached[b], cached[b] + new[b]) for b in range(case["B"])])
        elements, exponents = [], []
        for x, pool, scale in ((s["k"], s["pk"], s["sk"]), (s["v"], s["pv"], s["sv"])):
            full = flat(pool).double()
            y = x.double()
            if scale is not None:
                y = y.reshape(*y.shape[:-1], -1, BLOCK)
                amax = y.abs().amax(-1)
                e = torch.full_like(amax, -118.0)
                for up in range(-117, 120):  # the least e with amax <= 448 2^e
                    e = torch.where(amax > 448.0 * 2.0 ** (up - 1), torch.full_like(e, float(up)), e)
                # e4m3 holds 4 bits from 2^-6 on and steps of 2^-9 below
                y = y * torch.exp2(-e)[..., None]
                unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))) / 8
                y = (torch.round(y / unit) * unit).flatten(-2)
                full_scale = flat(scale).double()
                full_scale[where] = e + 127.0
                exponents.append(full_scale.unflatten(0, (-1, page)).transpose(1, 2).contiguous())
            full[where] = y
            elements.append(full.unflatten(0, (-1, page)).transpose(1, 2).contiguous())
        return elements + exponents
    k, v = real(s["pk"], s["sk"]), real(s["pv"], s["sv"])
    if case["kind"] == "read":
        where = torch.cat([cells(b, cached[b], cached[b] + new[b]) for b in range(case["B"])])
        return k[where], v[where]
    G, W = case["heads"] // case["kv"], case["W"]
    out = torch.zeros(sum(new), case["heads"], D, dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        where = cells(b, 0, cached[b] + new[b])
        pos = cached[b] + torch.arange(new[b], device=DEV)
        for hk in range(case["kv"]):
            kb, vb = k[where, hk], v[where, hk]
            for h in range(hk * G, hk * G + G):
                d = s["mask"][h if case["mask_heads"] > 1 else 0] != 0
                for t0 in range(0, new[b], 1024):
                    t = pos[t0:t0 + 1024]
                    at = start[b] + t0
                    low = max(int(t[0]) - W, 0)
                    q = s["q"][at:at + len(t), h].double() / math.sqrt(D)
                    for routed in (False, True):
                        pick = d[at:at + len(t)].nonzero().flatten() if routed else torch.arange(len(t), device=DEV)
                        first = 0 if routed else low
                        if not len(pick):
                            continue
                        key = torch.arange(first, int(t[-1]) + 1, device=DEV)
                        seen = key[None] <= t[pick, None]
                        if not routed:
                            seen &= key[None] >= t[pick, None] - W
                        score = torch.where(seen, q[pick] @ kb[first:int(t[-1]) + 1].t(), -math.inf)
                        out[at + pick, h] += torch.softmax(score, -1) @ vb[first:int(t[-1]) + 1]
    return out
