"""Performance cases of the paged-cache operators: what a serving system does with the blocks that the index finds.

A case is a plain dict; its "op" says which operator it takes:

  rotate   norms of queries and keys for each head, with the position rotation                    (lsm_rotate_heads)
  append   keys and values of new tokens into the paged cache, normed and rotated on the way      (lsm_kv_append)
  attend   attention of a batch whose requests share long prefixes, each with pages of its own    (lsm_prefix_attention)

A page holds one 16-token block of the index unless a case says otherwise; a layer's pages are a strided view of blocks
that hold keys and values side by side. Queries, keys and values are strided views of one fused projection. Prefixes are
512..1536 tokens and sequences 16..2048, as in the repository's workloads, and up to 16k tokens for long prompts; 40 KB per
token over 40 layers is 2 KV heads of 128, 128 KB over 32 layers is 8 of them.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
THETA = 10000.0
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # queries and keys of one decode step of a few requests: latency counts
        {"name": "rotate 8", "op": "rotate", "tokens": 8, "hq": 32, "hkv": 2, "d": 128, "rot": 128, "interleaved": False,
         "norm": True, "dtype": "bf16", "far": 16384},
        # the tokens of a batch of prompts
        {"name": "rotate 8192", "op": "rotate", "tokens": 8192, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "norm": True, "dtype": "bf16", "far": 16384},
        # an odd number of tokens, every head with keys of its own, half of a head of 80 rotated, 32 bits
        {"name": "rotate 1003, heads of 80", "op": "rotate", "tokens": 1003, "hq": 32, "hkv": 32, "d": 80, "rot": 40,
         "interleaved": True, "norm": False, "dtype": "fp32", "far": 4096},
        # one decode step of 64 requests, half of each head rotated in neighbouring pairs
        {"name": "append 64", "op": "append", "tokens": 64, "hq": 32, "hkv": 2, "d": 128, "rot": 64, "interleaved": True,
         "norm": False, "dtype": "bf16", "far": 16384, "page": 16, "skipped": 0.0, "queries": True},
        # prompts of many requests, ragged, some of their tokens cached already
        {"name": "append 5001, some skipped", "op": "append", "tokens": 5001, "hq": 12, "hkv": 12, "d": 64, "rot": 64,
         "interleaved": False, "norm": True, "dtype": "fp16", "far": 4096, "page": 32, "skipped": 0.1, "queries": False},
        # a full step of prompts
        {"name": "append 16384", "op": "append", "tokens": 16384, "hq": 32, "hkv": 8, "d": 128, "rot": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "far": 16384, "page": 16, "skipped": 0.0, "queries": True},
        # decode of a few requests behind one short prefix: latency counts
        {"name": "attend 4, prefix 512", "op": "attend", "requests": 4, "groups": 1, "prefix_min": 512, "prefix_max": 512, "q_min": 1, "q_max": 1,
         "before_min": 15, "before_max": 127, "hq": 32, "hkv": 2, "d": 128, "page": 16, "dtype": "bf16", "lse": False, "lens": 1},
        # decode of an ordinary batch behind eight prefixes
        {"name": "attend 64, 8 prefixes", "op": "attend", "requests": 64, "groups": 8, "prefix_min": 512, "prefix_max": 1536, "q_min": 1, "q_max": 1,
         "before_min": 15, "before_max": 511, "hq": 32, "hkv": 8, "d": 128, "page": 16, "dtype": "bf16", "lse": False, "lens": 2},
        # decode of a large batch behind two long prompts
        {"name": "attend 256, 2 long prefixes", "op": "attend", "requests": 256, "groups": 2, "prefix_min": 8192, "prefix_max": 16384, "q_min": 1, "q_max": 1,
         "before_min": 15, "before_max": 2047, "hq": 32, "hkv": 2, "d": 128, "page": 16, "dtype": "bf16", "lse": False, "lens": 3},
        # decode of unrelated requests, from one token to 8,000: nothing is shared
        {"name": "attend 96, no prefix", "op": "attend", "requests": 96, "groups": 96, "prefix_min": 0, "prefix_max": 0, "q_min": 1, "q_max": 1,
         "before_min": 0, "before_max": 7999, "hq": 28, "hkv": 4, "d": 128, "page": 64, "dtype": "fp16", "lse": True, "lens": 4},
        # requests whose prompts end differently behind shared prefixes: 1 to 256 new tokens each
        {"name": "attend 24, q 1..256", "op": "attend", "requests": 24, "groups": 4, "prefix_min": 500, "prefix_max": 1536, "q_min": 1, "q_max": 256,
         "before_min": 0, "before_max": 300, "hq": 32, "hkv": 8, "d": 128, "page": 16, "dtype": "bf16", "lse": False, "lens": 5},
        # long prompts behind long shared prefixes: bound by the matrix cores
        {"name": "attend 8, q 1024..2048", "op": "attend", "requests": 8, "groups": 2, "prefix_min": 1536, "prefix_max": 4096, "q_min": 1024, "q_max": 2048,
         "before_min": 0, "before_max": 0, "hq": 32, "hkv": 8, "d": 128, "page": 16, "dtype": "bf16", "lse": False, "lens": 6},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to about hi, spread over its logarithm; the long ones are odd."""
    n = max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))
    return n | 1 if n > 2048 else n


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    hq, hkv, d = rng.choice([(32, 2, 128), (32, 8, 128), (48, 2, 128), (28, 4, 128), (32, 4, 64), (20, 5, 64), (12, 12, 64), (8, 1, 256)])
    if op != "attend":
        case = {"op": op, "tokens": _spread(rng, 1, 16384), "hq": hq, "hkv": hkv, "d": d, "rot": d if rng.random() < 0.6 else d // 2,
                "interleaved": rng.random() < 0.4, "norm": rng.random() < 0.6, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                "far": _spread(rng, 256, 32768)}
        if op == "append":
            case.update(page=rng.choice([16, 16, 32, 64]), skipped=rng.choice([0.0, 0.0, 0.1]), queries=rng.random() < 0.7)
            if case["dtype"] == "fp32":
                case["dtype"] = "bf16"
        return case
    case = {"op": op, "hq": hq, "hkv": hkv, "d": d, "page": rng.choice([16, 16, 32, 64]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
            "lse": rng.random() < 0.3, "lens": rng.randrange(1 << 20)}
    kind = rng.choice(["decode", "decode", "few", "prompt"])
    if kind == "decode":  # one token per request
        case.update(requests=_spread(rng, 1, 256), q_min=1, q_max=1)
        most = max(16, min(8000, 160000 // case["requests"]))
        case["before_max"] = _spread(rng, 16, most)
    elif kind == "few":   # a few tokens to a few hundred
        case.update(requests=_spread(rng, 1, 32), q_min=1, q_max=_spread(rng, 2, 256))
        case["before_max"] = _spread(rng, 16, 500)
    else:                 # prompts
        case.update(requests=_spread(rng, 1, 8), q_min=_spread(rng, 128, 512), q_max=_spread(rng, 513, 1500))
        case["before_max"] = rng.choice([0, _spread(rng, 16, 500)])
    case["groups"] = min(case["requests"], _spread(rng, 1, 8))
    case["before_min"] = 0
    case["prefix_min"] = rng.choice([0, _spread(rng, 16, 1536)])
    case["prefix_max"] = max(case["prefix_min"], _spread(rng, 16, 8192 if kind == "decode" else 2048))
    return case


# ---------------------------------------------------------------------------------------------------------------------
# lengths of a batch: from the case alone
# ---------------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """(first request of each group and the end, prefix lengths, new tokens, own lengths with the new tokens), as lists."""
    r = random.Random(case["lens"])
    n, groups = case["requests"], case["groups"]
    cuts = [0] + sorted(r.sample(range(1, n), groups - 1)) + [n]
    prefix = [r.randint(case["prefix_min"], case["prefix_max"]) for _ in range(groups)]
    q = [r.randint(case["q_min"], case["q_max"]) for _ in range(n)]
    before = [r.randint(case["before_min"], case["before_max"]) for _ in range(n)]
    prefix[0], q[0], before[0] = case["prefix_max"], case["q_max"], case["before_max"]  # one of each is as long as may be
    return cuts, prefix, q, [a + b for a, b in zip(before, q)]


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "rotate":
        n, heads = case["tokens"], hq + hkv
        return {"bytes": n * (2 * heads * d * size + 4 * case["rot"] + 4), "flops": n * heads * d * (3 + (4 if case["norm"] else 0))}
    if case["op"] == "append":
        n = case["tokens"]
        heads, kept = hkv * 2 * (1 - case["skipped"]) + (hq if case["queries"] else 0), hkv + (hq if case["queries"] else 0)
        return {"bytes": n * (2 * heads * d * size + 4 * case["rot"] + 12), "flops": n * kept * d * (3 + (4 if case["norm"] else 0))}
    cuts, prefix, q, own_lens = _lengths(case)
    group = [g for g in range(len(prefix)) for _ in range(cuts[g + 1] - cuts[g])]
    kv = 2 * hkv * d * size
    seen = sum(n * prefix[g] + n * (length - n) + n * (n + 1) // 2 for n, length, g in zip(q, own_lens, group))
    pages = sum(-(-x // case["page"]) for x in prefix + own_lens)
    return {"bytes": kv * (sum(prefix) + sum(own_lens)) + sum(q) * hq * (2 * d * size + (4 if case["lse"] else 0)) + 4 * pages,
            "flops": 4 * d * hq * seen}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=dtype)


def _table(case):
    """Cosines, then sines, of every position up to the farthest: what a serving process makes once."""
    half = case["rot"] // 2
    freq = THETA ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) * 2 / case["rot"])
    angle = torch.arange(case["far"], device=DEVICE, dtype=torch.float64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _pool(gen, pages, page, hkv, d, dtype):
    """Keys' and values' pages of one layer, side by side in a block: two strided views [pages, page, hkv, d]."""
    blocks = _normal(gen, (pages, 2, page, hkv, d), dtype)
    return blocks[:, 0], blocks[:, 1]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, hq, hkv, d = DTYPES[case["dtype"]], case["hq"], case["hkv"], case["d"]
    s = dict(case)
    if case["op"] in ("rotate", "append"):
        n = case["tokens"]
        fused = _normal(gen, (n, hq + 2 * hkv, d), dtype)
        s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device=DEVICE, dtype=torch.int32)
        s["table"] = _table(case)
        if case["norm"]:
            s["q_weight"], s["k_weight"] = ((1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE)).to(dtype) for _ in range(2))
        else:
            s["q_weight"] = s["k_weight"] = None
        if case["op"] == "append":
            page = case["page"]
            pages = -(-n // page) + 9
            s["k_pages"], s["v_pages"] = _pool(gen, pages, page, hkv, d, dtype)
            # new tokens fill pages in any order; page 0 is nobody's
            order = 1 + torch.randperm(pages - 1, generator=gen, device=DEVICE)
            at = torch.arange(n, device=DEVICE)
            slots = order[at // page] * page + at % page
            skip = torch.rand(n, generator=gen, device=DEVICE) < case["skipped"]
            s["slots"] = torch.where(skip, torch.full_like(slots, -1), slots)
        return s
    cuts, prefix, q, own_lens = _lengths(case)
    page = case["page"]
    lens = prefix + own_lens
    counts = [-(-x // page) for x in lens]
    total = sum(counts)
    s["k_pages"], s["v_pages"] = _pool(gen, total + 5, page, hkv, d, dtype)
    order = torch.randperm(total + 5, generator=gen, device=DEVICE)[:total].to(torch.int32)

    def tables(first, counts):
        width = max(1, max(counts))
        c = torch.tensor(counts, device=DEVICE)
        begin = first + torch.cumsum(c, 0) - c
        col = torch.arange(width, device=DEVICE)
        at = (begin[:, None] + col).clamp(max=max(0, total - 1))
        held = order[at] if total else torch.zeros_like(at, dtype=torch.int32)
        return torch.where(col < c[:, None], held, torch.full_like(held, -1)).contiguous()

    n_groups = len(prefix)
    ints = dict(device=DEVICE, dtype=torch.int32)
    s["group_offsets"] = torch.tensor(cuts, **ints)
    s["prefix_tables"] = tables(0, counts[:n_groups])
    s["prefix_lens"] = torch.tensor(prefix, **ints)
    s["q_offsets"] = torch.tensor([0] + list(np.cumsum(q)), **ints)
    s["own_tables"] = tables(sum(counts[:n_groups]), counts[n_groups:])
    s["own_lens"] = torch.tensor(own_lens, **ints)
    s["q_max"] = max(q)
    fused = _normal(gen, (sum(q), hq + 2 * hkv, d), dtype)
    s["q"] = fused[:, :hq]
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------------------------------------------------
def _plain_rotate(x, weight, s):
    """Norm (where there is a weight) and rotation of heads [n, heads, d]; one rounding at the end."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    rot = s["rot"]
    half = rot // 2
    rows = s["table"][s["positions"].long()]
    cos, sin = rows[:, None, :half], rows[:, None, half:]
    z = y.clone()
    if s["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        z[..., 0:rot:2], z[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., :half], y[..., half:rot]
        z[..., :half], z[..., half:rot] = a * cos - b * sin, b * cos + a * sin
    return z.to(x.dtype)


def _plain_append(s):
    k = _plain_rotate(s["k"], s["k_weight"], s)
    kept = (s["slots"] >= 0)[:, None, None]
    page = s["page"]
    at, row = s["slots"].clamp(min=0) // page, s["slots"].clamp(min=0) % page  # page 0 is nobody's
    s["k_pages"][at, row] = torch.where(kept, k, s["k_pages"][at, row])
    s["v_pages"][at, row] = torch.where(kept, s["v"], s["v_pages"][at, row])
    return _plain_rotate(s["q"], s["q_weight"], s) if s["queries"] else None


def _plain_attend(s):
    q, page, hkv, d = s["q"], s["page"], s["hkv"], s["d"]
    total, hq = q.shape[0], q.shape[1]
    n, q_max, share = s["own_lens"].shape[0], s["q_max"], hq // hkv
    q_offsets, own_lens = s["q_offsets"].long(), s["own_lens"].long()
    request = torch.arange(n, device=q.device)
    group = torch.searchsorted(s["group_offsets"].long(), request, right=True) - 1
    # the keys and values of every request side by side: its prefix, then its own
    pages = torch.cat([s["prefix_tables"][group], s["own_tables"]], dim=1).clamp(min=0).long()
    wide = s["prefix_tables"].shape[1] * page
    col = torch.arange(pages.shape[1] * page, device=q.device)
    place = torch.where(col < wide, col, col - wide)
    prefix_lens = s["prefix_lens"].long()[group]
    held = torch.where(col < wide, place < prefix_lens[:, None], place < own_lens[:, None])            # [n, keys]
    keys = s["k_pages"][pages].reshape(n, -1, hkv, d).permute(0, 2, 1, 3).float()
    values = s["v_pages"][pages].reshape(n, -1, hkv, d).permute(0, 2, 1, 3).float()
    values = torch.where(held[:, None, :, None], values, torch.zeros((), device=q.device))
    token = torch.arange(q_max, device=q.device)
    q_lens = q_offsets[1:] - q_offsets[:-1]
    at = (q_offsets[:-1, None] + token).clamp(max=max(0, total - 1))
    rows = q[at].float().reshape(n, q_max, hkv, share, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, q_max * share, d)
    last = own_lens[:, None] - q_lens[:, None] + token                                                # [n, q_max]
    sees = held[:, None] & ((col < wide) | (place <= last[..., None]))                                # [n, q_max, keys]
    sees = sees[:, None, :, None].expand(n, 1, q_max, share, col.shape[0]).reshape(n, 1, q_max * share, col.shape[0])
    scores = torch.matmul(rows, keys.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(d))
    scores = torch.where(sees, scores, torch.full((), -math.inf, device=q.device))
    most = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    weights = torch.exp(scores - most)
    sums = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, values) / torch.where(sums > 0, sums, torch.ones((), device=q.device))
    out = out.reshape(n, hkv, q_max, share, d).permute(0, 2, 1, 3, 4).reshape(n, q_max, hq, d)
    lse = (most + torch.log(sums)).reshape(n, hkv, q_max, share).permute(0, 2, 1, 3).reshape(n, q_max, hq)
    mine = torch.searchsorted(q_offsets, torch.arange(total, device=q.device), right=True) - 1
    inside = torch.arange(total, device=q.device) - q_offsets[mine]
    out = out[mine, inside].to(q.dtype)
    return (out, lse[mine, inside]) if s["lse"] else out


def run(state):
    s = state
    if s["op"] == "rotate":
        if own:
            import paper_2511_16138_amd as lsm
            q, k = lsm.lsm_rotate_heads(s["q"], s["k"], s["positions"], s["table"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                        eps=EPS, interleaved=s["interleaved"])
        else:
            q, k = _plain_rotate(s["q"], s["q_weight"], s), _plain_rotate(s["k"], s["k_weight"], s)
        return {"q": q, "k": k}
    if s["op"] == "append":
        if own:
            import paper_2511_16138_amd as lsm
            queries = {"q": s["q"], "q_weight": s["q_weight"]} if s["queries"] else {}
            q = lsm.lsm_kv_append(s["k"], s["v"], s["positions"], s["slots"], s["k_pages"], s["v_pages"], s["table"],
                                  k_weight=s["k_weight"], eps=EPS, interleaved=s["interleaved"], **queries)
        else:
            q = _plain_append(s)
        out = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        return {**out, "q": q} if s["queries"] else out
    if own:
        import paper_2511_16138_amd as lsm
        batch = lsm.PrefixBatch(s["group_offsets"], s["prefix_tables"], s["prefix_lens"], s["q_offsets"], s["own_tables"], s["own_lens"])
        got = lsm.lsm_prefix_attention(s["q"], s["k_pages"], s["v_pages"], batch, with_lse=s["lse"])
    else:
        got = _plain_attend(s)
    return {"out": got[0], "lse": got[1]} if s["lse"] else {"out": got}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, token by token and request by request
# ---------------------------------------------------------------------------------------------------------------------
def _exact_rotate(x, weight, s):
    x = x.double()
    if weight is not None:
        x = weight.double() * x / torch.sqrt(torch.sum(x ** 2, dim=-1, keepdim=True) / x.shape[-1] + EPS)
    half = s["rot"] // 2
    angles = s["table"].double().index_select(0, s["positions"].long())
    turn = torch.complex(angles[:, :half], angles[:, half:])[:, None, :]
    if s["interleaved"]:
        first, second = slice(0, s["rot"], 2), slice(1, s["rot"], 2)
    else:
        first, second = slice(0, half), slice(half, s["rot"])
    pair = torch.complex(x[..., first], x[..., second]) * turn
    out = x.clone()
    out[..., first], out[..., second] = pair.real, pair.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "rotate":
        return {"q": _exact_rotate(s["q"], s["q_weight"], s), "k": _exact_rotate(s["k"], s["k_weight"], s)}
    if s["op"] == "append":
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        kept = torch.nonzero(s["slots"] >= 0).flatten()
        slots = s["slots"][kept]
        k_pages.view(-1, s["hkv"], s["d"])[slots] = _exact_rotate(s["k"], s["k_weight"], s)[kept]
        v_pages.view(-1, s["hkv"], s["d"])[slots] = s["v"].double()[kept]
        out = {"k_pages": k_pages, "v_pages": v_pages}
        return {**out, "q": _exact_rotate(s["q"], s["q_weight"], s)} if s["queries"] else out
    cuts, prefix, q_lens, own_lens = _lengths(case)
    share, first = s["hq"] // s["hkv"], 0
    outs, lses = [], []
    for g, length in enumerate(prefix):
        head = s["prefix_tables"][g].long()[:-(-length // s["page"])]
        head_k, head_v = (s[p][head].flatten(0, 1)[:length].double() for p in ("k_pages", "v_pages"))
        for r in range(cuts[g], cuts[g + 1]):
            n, mine = q_lens[r], own_lens[r]
            tail = s["own_tables"][r].long()[:-(-mine // s["page"])]
            keys, values = (torch.cat([h, s[p][tail].flatten(0, 1)[:mine].double()]) for h, p in ((head_k, "k_pages"), (head_v, "v_pages")))
            rows = s["q"][first:first + n].double()
            first += n
            late = torch.arange(length + mine, device=DEVICE)[None] > torch.arange(length + mine - n, length + mine, device=DEVICE)[:, None]
            out, lse = torch.empty_like(rows), torch.empty_like(rows[..., 0])
            for h in range(s["hkv"]):
                part = rows[:, h * share:(h + 1) * share].reshape(n * share, -1)
                scores = part @ keys[:, h].t().contiguous() / math.sqrt(s["d"])
                scores = scores.reshape(n, share, -1).masked_fill(late[:, None], -math.inf)
                lse[:, h * share:(h + 1) * share] = torch.logsumexp(scores, -1)
                shares = torch.softmax(scores, -1).nan_to_num(0.0).reshape(n * share, -1)
                out[:, h * share:(h + 1) * share] = (shares @ values[:, h].contiguous()).reshape(n, share, -1)
            outs.append(out)
            lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)} if s["lse"] else {"out": torch.cat(outs)}
