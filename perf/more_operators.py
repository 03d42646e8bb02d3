"""Performance cases of the attention of a decoder to its own earlier tokens: over whole prompts that lie packed one behind the
other, and of new tokens over a cache of keys and values in pages, with the operator that fills it.

Three kinds of case:
  causal  softmax(q k^T / sqrt(dim)) v over the tokens of the same sequence up to the token itself; in training with the gradients
  paged   the same for the newest tokens of each sequence, whose keys and values lie in pages that a table names
  write   keys and values of new tokens into those pages

Head counts and widths are those of the paper's model table (KAT-T / S / B: 3 / 6 / 12 heads of 64) and generic ones.  With `own` False,
run() computes the operators from elementary operations in 32 bits; with `own` True it calls the framework.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
SIZE = 2

# of the largest listed cases, which a drawn case stays below
MOST_BYTES = 5.9e8
MOST_FLOPS = 3.4e11
# pairs of a padded batch: the plain form writes that many scores in 32 bits, in training several times
MOST_PAIRS = 5.3e8


def _causal(name, dtype, sequences, longest, behind, heads, kv_heads, dim, train):
    """behind: tokens of the buffer behind the last sequence, which belong to none."""
    return {"name": name, "kind": "causal", "dtype": dtype, "sequences": sequences, "longest": longest, "behind": behind,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "train": train}


def _paged(name, dtype, sequences, tokens, longest, page, heads, kv_heads, dim):
    """tokens: new ones of each sequence; longest: the longest sequence with them."""
    return {"name": name, "kind": "paged", "dtype": dtype, "sequences": sequences, "tokens": tokens, "longest": longest, "page": page,
            "heads": heads, "kv_heads": kv_heads, "dim": dim}


def _write(name, dtype, sequences, longest, before, page, kv_heads, dim):
    """longest: new tokens of the sequence that has the most; before: tokens that the cache has already, at most."""
    return {"name": name, "kind": "write", "dtype": dtype, "sequences": sequences, "longest": longest, "before": before, "page": page,
            "kv_heads": kv_heads, "dim": dim}


def listed():
    return [
        # one short prompt of a small model: launch and host time count
        _causal("prompt, one short", "bf16", 1, 16, 0, 3, 3, 64, False),
        # the prompts of a serving batch, of different lengths, in a buffer that is not quite full
        _causal("prompts, packed", "bf16", 24, 1000, 40, 12, 12, 64, False),
        # one long prompt, shared key heads: a serving step by itself
        _causal("prompt, one long", "f16", 1, 4096, 0, 32, 8, 128, False),
        # KAT-B widths in training, texts packed to a batch
        _causal("packed training", "bf16", 16, 1500, 100, 12, 12, 64, True),
        # two long sequences in training, shared key heads
        _causal("long training", "bf16", 2, 4001, 0, 16, 4, 128, True),
        # one user: a token at a time, launch and host time count
        _paged("token, one user", "bf16", 1, 1, 500, 16, 12, 12, 64),
        # a serving batch of single tokens with long contexts
        _paged("tokens, batch", "bf16", 32, 1, 8191, 64, 32, 8, 128),
        # one user with a very long context
        _paged("token, long context", "f16", 1, 1, 100003, 128, 32, 8, 128),
        # a few proposed tokens of each sequence to be looked at together
        _paged("proposed tokens", "f16", 8, 5, 3001, 24, 12, 4, 96),
        # the new tokens of a serving step
        _write("write, single tokens", "bf16", 64, 1, 500, 16, 8, 128),
        # whole prompts into an empty cache
        _write("write, prompts", "bf16", 12, 4000, 0, 64, 8, 128),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        kind = rng.choice(["causal", "causal", "causal", "paged", "paged", "paged", "write"])
        dtype, dim, page = rng.choice(["bf16", "bf16", "f16"]), rng.choice([64, 64, 128, 128, 80, 32, 96]), rng.choice([8, 16, 16, 20, 32, 64, 128, 256])
        kv = rng.choice([1, 2, 3, 4, 6, 8, 12])
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        if kind == "causal":
            c = _causal("", dtype, _log(rng, 1, 64), _log(rng, 16, 4096), rng.choice([0, 0, _log(rng, 1, 300)]), heads, kv, dim, rng.random() < 0.5)
            if c["sequences"] * heads * c["longest"] ** 2 > MOST_PAIRS:
                continue
        elif kind == "paged":
            c = _paged("", dtype, _log(rng, 1, 128), rng.choice([1, 1, 1, _log(rng, 2, 16)]), _log(rng, 33, 100003), page, heads, kv, dim)
            # the plain form gathers all pages of the table, in 32 bits, and writes all scores
            if c["sequences"] * c["longest"] * (kv * dim + c["tokens"] * heads) > 5e8:
                continue
        else:
            c = _write("", dtype, _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 4096)]), rng.choice([0, _log(rng, 1, 2000)]), page, kv, dim)
        del c["name"]
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return c


# ------------------------------------------------------------------------------------------------ inputs
def _spread(count, longest, least, salt):
    """`count` lengths up to the longest, over their logarithm, the first the longest; now and then one is 1 and one 0."""
    rng = random.Random(1000003 * longest + 101 * count + salt)
    found = [min(longest, max(1, _log(rng, max(1.0, longest * least), longest))) for _ in range(count)]
    if count > 3:
        found[count // 2] = 0
        found[count // 3] = 1
    found[0] = longest
    return found


def _lengths(case):
    """causal: tokens of each sequence; paged: tokens in the cache, the newest among them; write: new tokens."""
    if case["kind"] == "paged":
        return _spread(case["sequences"], case["longest"], 0.25, 7)
    return _spread(case["sequences"], case["longest"], 0.06, 5)


def _offsets(lengths):
    found = [0]
    for n in lengths:
        found.append(found[-1] + n)
    return found


def _whole(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _pages(case, held, gen, rand):
    """(k_pages, v_pages, table) for that many tokens of each sequence: pages in an order of chance, some of the pool free; the table's
    entries that no sequence has reached yet name page 0."""
    page = case["page"]
    counts = [-(-n // page) for n in held]
    pool = sum(counts) + max(2, sum(counts) // 16)
    order = torch.randperm(pool, device=DEVICE, generator=gen).to(torch.int32)
    wide = max(1, max(counts))
    column = torch.arange(wide, device=DEVICE)
    first, count = _whole(_offsets(counts)[:-1]), _whole(counts)
    at = (first[:, None] + column).clamp(max=pool - 1).long()
    table = torch.where(column < count[:, None], order[at], 0).to(torch.int32).contiguous()
    return rand(pool, page, case["kv_heads"], case["dim"]), rand(pool, page, case["kv_heads"], case["dim"]), table


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    dtype, kv, dim = TYPES[case["dtype"]], case["kv_heads"], case["dim"]

    def rand(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen).to(dtype)

    s = {"case": case}
    lengths = _lengths(case)
    if case["kind"] == "causal":
        heads, tokens = case["heads"], sum(lengths) + case["behind"]
        s["lengths"], s["offsets"] = _whole(lengths), _whole(_offsets(lengths))
        # one projection's output holds queries, keys and values side by side
        qkv = rand(tokens, heads + 2 * kv, dim)
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        if case["train"]:
            s["dout"] = rand(tokens, heads, dim)
            s["leaves"] = [s[n].requires_grad_() for n in ("q", "k", "v")]
    elif case["kind"] == "paged":
        s["lengths"] = _whole(lengths)
        s["k_pages"], s["v_pages"], s["table"] = _pages(case, lengths, gen, rand)
        s["q"] = rand(case["sequences"], case["tokens"], case["heads"], dim)
    else:
        before = [min(case["before"], case["before"] * (i + 1) // case["sequences"]) for i in range(case["sequences"])]
        held = [a + b for a, b in zip(before, lengths)]
        s["lengths"], s["offsets"] = _whole(held), _whole(_offsets(lengths))
        s["k_pages"], s["v_pages"], s["table"] = _pages(case, held, gen, rand)
        kv_new = rand(sum(lengths), 2 * kv, dim)
        s["k"], s["v"] = kv_new[:, :kv], kv_new[:, kv:]
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    with torch.no_grad():
        return {"causal": _plain_causal, "paged": _plain_paged, "write": _plain_write}[case["kind"]](s, case)


def _run_own(s, case):
    from paper_2505_13813_amd import transformer

    if case["kind"] == "causal" and case["train"]:
        out = transformer.causal_attention(s["q"], s["k"], s["v"], s["offsets"])
        dq, dk, dv = torch.autograd.grad(out, s["leaves"], s["dout"])
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    with torch.no_grad():
        if case["kind"] == "causal":
            return {"out": transformer.causal_attention(s["q"], s["k"], s["v"], s["offsets"])}
        if case["kind"] == "paged":
            return {"out": transformer.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"])}
        transformer.paged_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["offsets"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ------------------------------------------------------------------------------------------------ plain forms, in 32 bits
def _softmax(score, ok):
    score = score.masked_fill(~ok, -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most > -math.inf, most, 0.0))
    del score
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, 1.0)


def _plain_causal(s, case):
    """Every sequence padded to the longest, [sequence, key head, group, token, dim]."""
    kv, tokens, scale = case["kv_heads"], s["q"].shape[0], case["dim"] ** -0.5
    at = torch.arange(case["longest"], device=DEVICE)
    there = at < s["lengths"][:, None]
    place = torch.where(there, s["offsets"][:-1, None] + at, 0).long()
    back = place[there]

    def padded(t):
        u = t.detach().float()[place] * there[:, :, None, None]
        return u.unflatten(2, (kv, -1)).permute(0, 2, 3, 1, 4).contiguous()

    def packed(t):
        out = torch.zeros(tokens, t.shape[1] * t.shape[2], case["dim"], dtype=torch.float32, device=DEVICE)
        out[back] = t.permute(0, 3, 1, 2, 4).flatten(2, 3)[there]
        return out.to(s["q"].dtype)

    q, k, v = padded(s["q"]), padded(s["k"]), padded(s["v"])
    ok = (at[None, :] <= at[:, None]) & there[:, None, None, None, :]
    p = _softmax((q @ k.transpose(-1, -2).contiguous()) * scale, ok)
    out = {"out": packed(p @ v)}
    if case["train"]:
        do = padded(s["dout"])
        out["dv"] = packed((p.transpose(-1, -2).contiguous() @ do).sum(2, keepdim=True))
        dp = do @ v.transpose(-1, -2).contiguous()
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        del dp, p
        out["dq"] = packed(ds @ k)
        out["dk"] = packed((ds.transpose(-1, -2).contiguous() @ q).sum(2, keepdim=True))
    return out


def _plain_paged(s, case):
    kv, n, scale = case["kv_heads"], case["tokens"], case["dim"] ** -0.5

    def gathered(pages):  # [sequence, key head, 1, key, dim]
        return pages[s["table"].long()].flatten(1, 2).float().permute(0, 2, 1, 3).contiguous()[:, :, None]

    q = s["q"].float().unflatten(2, (kv, -1)).permute(0, 2, 3, 1, 4).contiguous()
    k, v = gathered(s["k_pages"]), gathered(s["v_pages"])
    last = s["lengths"][:, None] - n + torch.arange(n, device=DEVICE)
    ok = torch.arange(k.shape[3], device=DEVICE) <= last[:, None, None, :, None]
    p = _softmax((q @ k.transpose(-1, -2).contiguous()) * scale, ok)
    return {"out": (p @ v).permute(0, 3, 1, 2, 4).flatten(2, 3).contiguous().to(s["q"].dtype)}


def _plain_write(s, case):
    token = torch.arange(s["k"].shape[0], device=DEVICE)
    sequence = (token[:, None] >= s["offsets"][None, 1:]).sum(1)
    position = s["lengths"].long()[sequence] - s["offsets"].long()[sequence + 1] + token
    page = s["table"].long()[sequence, position // case["page"]]
    s["k_pages"][page, position % case["page"]] = s["k"]
    s["v_pages"][page, position % case["page"]] = s["v"]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    lengths = _lengths(case)
    kv, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "write":
        return {"bytes": 4 * sum(lengths) * kv * dim * SIZE, "flops": 0}
    heads = case["heads"]
    if case["kind"] == "paged":
        n = case["tokens"]
        pairs = sum(max(0, length - i) for length in lengths for i in range(n)) * heads
        rows = 2 * case["sequences"] * n * heads * dim * SIZE
        return {"bytes": rows + 2 * sum(lengths) * kv * dim * SIZE, "flops": 4 * pairs * dim}
    tokens = sum(lengths)
    product = sum(length * (length + 1) // 2 for length in lengths) * heads * 2 * dim
    rows, keys = tokens * heads * dim * SIZE, tokens * kv * dim * SIZE
    if case["train"]:
        # forward: q, k, v, out; backward: q, k, v, out, dout, dq, dk, dv; five products beside the forward pass's two
        return {"bytes": 6 * rows + 6 * keys, "flops": 7 * product}
    return {"bytes": 2 * rows + 2 * keys, "flops": 2 * product}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        return {"causal": _exact_causal, "paged": _exact_paged, "write": _exact_write}[case["kind"]](s, case)


def _exact_causal(s, case):
    q, k, v = (s[n].detach().double() for n in ("q", "k", "v"))
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    found = {"out": torch.zeros_like(q, memory_format=torch.contiguous_format)}
    if case["train"]:
        found |= {"d" + n: torch.zeros_like(t, memory_format=torch.contiguous_format) for n, t in (("q", q), ("k", k), ("v", v))}
    start = 0
    for length in _lengths(case):
        at = slice(start, start + length)
        start += length
        later = torch.ones(length, length, dtype=torch.bool, device=DEVICE).triu(1)
        for head in range(case["heads"] if length else 0):
            kv = head // group
            Q, K, V = q[at, head], k[at, kv], v[at, kv]
            score = Q @ K.t() * scale
            score[later] = -math.inf
            P = torch.softmax(score, 1)
            found["out"][at, head] = P @ V
            if case["train"]:
                dO = s["dout"][at, head].double()
                dS = P * (dO @ V.t() - (dO * found["out"][at, head]).sum(1, keepdim=True)) * scale
                found["dq"][at, head] = dS @ K
                found["dk"][at, kv] += dS.t() @ Q
                found["dv"][at, kv] += P.t() @ dO
    return found


def _exact_paged(s, case):
    group, n, page, scale = case["heads"] // case["kv_heads"], case["tokens"], case["page"], 1.0 / math.sqrt(case["dim"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, length in enumerate(_lengths(case)):
        key = torch.arange(length, device=DEVICE)
        pages, place = s["table"][b].long()[key // page], key % page
        for kv in range(case["kv_heads"] if length else 0):
            K, V = s["k_pages"][pages, place, kv].double(), s["v_pages"][pages, place, kv].double()
            for i in range(n):
                seen = length - (n - 1 - i)
                if seen > 0:
                    Q = s["q"][b, i, kv * group:(kv + 1) * group].double()
                    out[b, i, kv * group:(kv + 1) * group] = torch.softmax(Q @ K[:seen].t() * scale, 1) @ V[:seen]
    return {"out": out}


def _exact_write(s, case):
    k_pages, v_pages, page, first = s["k_pages"].double(), s["v_pages"].double(), case["page"], 0
    for b, length in enumerate(_lengths(case)):
        position = int(s["lengths"][b]) - length + torch.arange(length, device=DEVICE)
        at, place = s["table"][b].long()[position // page], position % page
        k_pages[at, place] = s["k"][first:first + length].double()
        v_pages[at, place] = s["v"][first:first + length].double()
        first += length
    return {"k_pages": k_pages, "v_pages": v_pages}
