"""Performance cases of the operators that stand around the KAT MLP in a transformer block: root-mean-square norm with the
residual's addition (and an 8-bit output), rotary positions with several axes, and cross attention to an encoder's states.

Four kinds of case:
  norm       h = x + residual, y = h / rms(h) * weight; in training with the gradients of both
  norm8      the same with y in 8 bits (float8 e4m3) and one scale for each row
  rotary     rotation of queries and keys by the positions of their tokens along several axes; in training also back
  attention  softmax(q k^T / sqrt(D)) v over another sequence, of a length for each batch entry or under a mask; in
             training with the gradients

Sizes are those of the paper's model table (KAT-T / S / B: 192 / 384 / 768 channels in 3 / 6 / 12 heads of 64, 197 tokens,
128 images per GPU) and generic ones.  With `own` False, run() computes the operators from elementary operations in 32 bits;
with `own` True it calls the framework.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
F8_MOST = 448.0

# work of the largest listed cases: a drawn case stays below
MOST_BYTES = 6.0e8
MOST_FLOPS = 9.0e11


def _norm(name, dtype, rows, dim, residual, train):
    return {"name": name, "kind": "norm", "dtype": dtype, "rows": rows, "dim": dim, "residual": residual, "train": train}


def _norm8(name, dtype, rows, dim, residual):
    return {"name": name, "kind": "norm8", "dtype": dtype, "rows": rows, "dim": dim, "residual": residual, "train": False}


def _rotary(name, dtype, batch, grid, heads, kv_heads, dim, pairs, interleaved, train):
    """grid: extents of the tokens' axes, as text; pairs: rotated pairs of channels for each axis."""
    return {"name": name, "kind": "rotary", "dtype": dtype, "batch": batch, "grid": grid, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "pairs": pairs, "interleaved": interleaved, "train": train}


def _attention(name, dtype, batch, queries, keys, heads, kv_heads, dim, mask, train):
    """mask: "none", "lengths" (a number of keys for each batch entry) or "mask" (a truth value for each key)."""
    return {"name": name, "kind": "attention", "dtype": dtype, "batch": batch, "queries": queries, "keys": keys, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "mask": mask, "train": train}


def listed():
    return [
        # one step of a decoder serving a few sequences: launch and host time count
        _norm("norm, 8 tokens", "bf16", 8, 768, True, False),
        # KAT-B in training, 128 images per GPU, mixed precision
        _norm("norm, KAT-B training", "bf16", 128 * 197, 768, True, True),
        # an odd width in float32, without a residual, with gradients
        _norm("norm, odd width f32", "f32", 5003, 1111, False, True),
        # a prompt batch of a wide model, on its way into an 8-bit product
        _norm8("norm to 8 bits, wide", "bf16", 16384, 4096, True),
        # one image of KAT-B in inference: 14 x 14 patches, positions along height and width
        _rotary("rotary, one image", "bf16", 1, "14x14", 12, 12, 64, "16,16", False, False),
        # KAT-B in training
        _rotary("rotary, images training", "bf16", 128, "14x14", 12, 12, 64, "16,16", False, True),
        # a video: time, height, width; fewer key heads than query heads, adjacent channels as pairs
        _rotary("rotary, video", "f16", 2, "16x23x40", 16, 4, 128, "16,24,24", True, False),
        # KAT-T sized queries to one image's tokens
        _attention("attention, one image", "bf16", 1, 16, 197, 3, 3, 64, "none", False),
        # single tokens of a serving batch against long encoder states of different lengths
        _attention("attention, single tokens", "bf16", 16, 1, 8191, 32, 8, 128, "lengths", False),
        # a batch of queries to padded image tokens
        _attention("attention, images", "bf16", 64, 197, 577, 12, 12, 64, "lengths", False),
        # the same path in training, tokens dropped by a mask
        _attention("attention, images training", "bf16", 32, 256, 785, 12, 12, 64, "mask", True),
        # the largest: long sequences, shared key heads
        _attention("attention, long training", "f16", 2, 4096, 4001, 16, 4, 128, "lengths", True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "norm8", "rotary", "rotary", "attention", "attention", "attention"])
        if kind in ("norm", "norm8"):
            dim = rng.choice([_log(rng, 32, 8192), 8 * _log(rng, 8, 1024), 192, 384, 768])
            if kind == "norm":
                c = _norm("", rng.choice(["f32", "bf16", "bf16", "f16"]), _log(rng, 1, 60000), dim, rng.random() < 0.7,
                          rng.random() < 0.5)
            else:
                c = _norm8("", rng.choice(["bf16", "bf16", "f16"]), _log(rng, 1, 60000), dim, rng.random() < 0.7)
        elif kind == "rotary":
            dim = rng.choice([64, 64, 128, 80, 96])
            axes = rng.choice([2, 2, 3])
            grid = [_log(rng, 1, 48) for _ in range(axes)]
            if axes == 2:
                first = rng.randint(1, dim // 2 - 1)
                pairs = rng.choice([[dim // 4, dim // 4], [first, dim // 2 - first]])
            else:
                pairs = rng.choice([[dim // 8, dim // 16, dim // 16], [dim // 2 - 2 * (dim // 6), dim // 6, dim // 6]])
            kv = rng.choice([1, 2, 3, 4, 8, 12])
            c = _rotary("", rng.choice(["bf16", "bf16", "f16", "f32"]), _log(rng, 1, 64), "x".join(map(str, grid)),
                        kv * rng.choice([1, 1, 2, 4]), kv, dim, ",".join(map(str, pairs)), rng.random() < 0.5, rng.random() < 0.5)
        else:
            kv = rng.choice([1, 2, 3, 4, 6, 8, 12])
            train = rng.random() < 0.5
            c = _attention("", rng.choice(["bf16", "bf16", "f16"]), _log(rng, 1, 64),
                           _log(rng, 16, 4096) if train else rng.choice([1, 1, _log(rng, 1, 4096)]), _log(rng, 33, 16384),
                           kv * rng.choice([1, 1, 2, 4, 8]), kv, rng.choice([64, 64, 128, 80, 32, 96]),
                           rng.choice(["none", "lengths", "mask"]), train)
            # the plain form writes all scores in 32 bits, in training several times
            if c["batch"] * c["heads"] * c["queries"] * c["keys"] > 6e8:
                continue
        del c["name"]
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return c


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Keys of each batch entry: from a quarter of all to all, now and then none (but where there is one entry)."""
    rng = random.Random(1000003 * case["keys"] + case["batch"])
    found = [max(1, int(case["keys"] * rng.uniform(0.25, 1.0))) for _ in range(case["batch"])]
    if case["batch"] > 3:
        found[case["batch"] // 2] = 0
    found[0] = case["keys"]
    return found


def _kept(case):
    """Which keys of each batch entry the mask keeps, [batch][keys] truth values: three in four, of one entry none."""
    rng = random.Random(1000033 * case["keys"] + case["batch"])
    found = [[rng.random() < 0.75 for _ in range(case["keys"])] for _ in range(case["batch"])]
    if case["batch"] > 3:
        found[case["batch"] // 2] = [False] * case["keys"]
    return found


def _positions(grid, gen):
    """[tokens, axes]: the grid's points, in row order, from a random origin on (a crop of a larger picture)."""
    extents = [int(v) for v in grid.split("x")]
    points = torch.cartesian_prod(*(torch.arange(v) for v in extents)).reshape(-1, len(extents))
    origin = torch.randint(0, 64, (len(extents),), generator=gen, device=DEVICE)
    return (points.to(DEVICE) + origin).to(torch.int32).contiguous()


def _frequencies(pairs, theta=10000.0):
    """Radians per position step of each pair, and the axis that it turns with: a ladder of its own for each axis."""
    counts = [int(v) for v in pairs.split(",")]
    turns = torch.cat([theta ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in counts])
    axis = torch.cat([torch.full((n,), a, dtype=torch.int32) for a, n in enumerate(counts)])
    return turns.to(DEVICE), axis.to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    kind, train, dtype = case["kind"], case["train"], TYPES[case["dtype"]]

    def rand(*shape, std=1.0):
        return (torch.randn(*shape, device=DEVICE, generator=gen) * std).to(dtype)

    s = {"case": case}
    if kind in ("norm", "norm8"):
        rows, dim = case["rows"], case["dim"]
        # a residual stream: some channels larger than others
        channel = torch.exp(0.5 * torch.randn(dim, device=DEVICE, generator=gen))
        s["x"] = rand(rows, dim)
        s["residual"] = (torch.randn(rows, dim, device=DEVICE, generator=gen) * channel).to(dtype) if case["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(dim, device=DEVICE, generator=gen)).to(dtype)
        if train:
            s["dy"], s["dh"] = rand(rows, dim), rand(rows, dim) if case["residual"] else None
            s["leaves"] = [t for t in (s["x"], s["residual"], s["weight"]) if t is not None]
    elif kind == "rotary":
        positions = _positions(case["grid"], gen)
        tokens = positions.shape[0]
        s["positions"] = positions
        s["frequencies"], s["axis"] = _frequencies(case["pairs"])
        # one projection's output holds queries, keys and values side by side
        heads, kv = case["heads"], case["kv_heads"]
        qkv = rand(case["batch"], tokens, heads + 2 * kv, case["dim"])
        s["q"], s["k"] = qkv[:, :, :heads], qkv[:, :, heads:heads + kv]
        if train:
            s["dq"], s["dk"] = rand(case["batch"], tokens, heads, case["dim"]), rand(case["batch"], tokens, kv, case["dim"])
            s["leaves"] = [s["q"], s["k"]]
    else:
        batch, keys, kv = case["batch"], case["keys"], case["kv_heads"]
        s["q"] = rand(batch, case["queries"], case["heads"], case["dim"])
        # keys and values are one projection's output
        projected = rand(batch, keys, 2, kv, case["dim"])
        s["k"], s["v"] = projected[:, :, 0], projected[:, :, 1]
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE) if case["mask"] == "lengths" else None
        s["mask"] = torch.tensor(_kept(case), device=DEVICE) if case["mask"] == "mask" else None
        if train:
            s["dout"] = rand(batch, case["queries"], case["heads"], case["dim"])
            s["leaves"] = [s["q"], s["k"], s["v"]]
    for t in s.get("leaves", ()):
        t.requires_grad_()
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case, kind)
    with torch.no_grad():
        if kind == "norm":
            return _plain_norm(s, case["train"])
        if kind == "norm8":
            return _plain_norm8(s)
        return _plain_rotary(s, case) if kind == "rotary" else _plain_attention(s, case)


def _run_own(s, case, kind):
    from paper_2505_13813_amd import transformer

    if not case["train"]:
        with torch.no_grad():
            if kind == "norm":
                out = transformer.rms_norm(s["x"], s["weight"], s["residual"], eps=EPS)
                return {"y": out} if s["residual"] is None else {"y": out[0], "h": out[1]}
            if kind == "norm8":
                out = transformer.rms_norm_8bit(s["x"], s["weight"], s["residual"], eps=EPS)
                return dict(zip(("y", "scale", "h"), out))
            if kind == "rotary":
                q, k = transformer.rotary(s["q"], s["positions"], s["frequencies"], s["axis"], k=s["k"],
                                          interleaved=case["interleaved"])
                return {"q": q, "k": k}
            return {"out": transformer.cross_attention(s["q"], s["k"], s["v"], key_lengths=s["lengths"], key_mask=s["mask"])}
    if kind == "norm":
        out = transformer.rms_norm(s["x"], s["weight"], s["residual"], eps=EPS)
        if s["residual"] is None:
            dx, dw = torch.autograd.grad(out, s["leaves"], s["dy"])
            return {"y": out, "dx": dx, "dweight": dw}
        dx, dr, dw = torch.autograd.grad(out, s["leaves"], (s["dy"], s["dh"]))
        return {"y": out[0], "h": out[1], "dx": dx, "dresidual": dr, "dweight": dw}
    if kind == "rotary":
        q, k = transformer.rotary(s["q"], s["positions"], s["frequencies"], s["axis"], k=s["k"], interleaved=case["interleaved"])
        dq, dk = torch.autograd.grad((q, k), s["leaves"], (s["dq"], s["dk"]))
        return {"q": q, "k": k, "dq": dq, "dk": dk}
    out = transformer.cross_attention(s["q"], s["k"], s["v"], key_lengths=s["lengths"], key_mask=s["mask"])
    dq, dk, dv = torch.autograd.grad(out, s["leaves"], s["dout"])
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


# ------------------------------------------------------------------------------------------------ plain forms, in 32 bits
def _plain_norm(s, train):
    x, w, dtype = s["x"], s["weight"].float(), s["x"].dtype
    # the sum is kept in the residual stream's own type, and it is the kept one that is normalised
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(dtype)
    f = h.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    out = {"y": (f * r * w).to(dtype)}
    if s["residual"] is not None:
        out["h"] = h
    if train:
        dy = s["dy"].float()
        g, n = dy * w, f * r
        dx = r * (g - n * (g * n).mean(-1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["dh"].float()
        out["dx"] = dx.to(dtype)
        if s["residual"] is not None:
            out["dresidual"] = out["dx"]
        out["dweight"] = (dy * n).sum(0).to(dtype)
    return out


def _plain_norm8(s):
    x, w, dtype = s["x"], s["weight"].float(), s["x"].dtype
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(dtype)
    f = h.float()
    y = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * w
    scale = y.abs().amax(-1) / F8_MOST
    q = (y / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-F8_MOST, F8_MOST).to(torch.float8_e4m3fn)
    return {"y": q, "scale": scale} if s["residual"] is None else {"y": q, "scale": scale, "h": h}


def _turn(t, cos, sin, interleaved):
    """t [batch, tokens, heads, dim] with pair j turned by the angle of cos, sin [tokens, 1, j]; what is not in a pair stays."""
    n = cos.shape[-1]
    f = t.float()
    if interleaved:
        a, b = f[..., 0:2 * n:2], f[..., 1:2 * n:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = f[..., :n], f[..., n:2 * n]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, f[..., 2 * n:]), -1).to(t.dtype)


def _plain_rotary(s, case):
    angle = (s["positions"][:, s["axis"].long()].float() * s["frequencies"].float())[:, None, :]
    cos, sin, interleaved = angle.cos(), angle.sin(), case["interleaved"]
    out = {"q": _turn(s["q"], cos, sin, interleaved), "k": _turn(s["k"], cos, sin, interleaved)}
    if case["train"]:
        out["dq"], out["dk"] = _turn(s["dq"], cos, -sin, interleaved), _turn(s["dk"], cos, -sin, interleaved)
    return out


def _valid(s, case):
    """[batch, 1, 1, 1, keys] truth values, or None."""
    if case["mask"] == "lengths":
        ok = torch.arange(case["keys"], device=DEVICE) < s["lengths"][:, None]
    elif case["mask"] == "mask":
        ok = s["mask"]
    else:
        return None
    return ok[:, None, None, None, :]


def _by_key_head(t, kv, to):
    """[batch, tokens, heads, dim] as [batch, key head, group, tokens, dim]."""
    b, n, h, d = t.shape
    return t.to(to).reshape(b, n, kv, h // kv, d).permute(0, 2, 3, 1, 4).contiguous()


def _attend(s, case, to):
    """Cross attention and, in training, its gradients, in the type `to`."""
    kv, train = case["kv_heads"], case["train"]
    scale = case["dim"] ** -0.5
    q, k, v = (_by_key_head(s[n].detach(), kv, to) for n in ("q", "k", "v"))
    ok = _valid(s, case)
    score = (q @ k.transpose(-1, -2).contiguous()) * scale
    if ok is not None:
        score = score.masked_fill(~ok, -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most > -math.inf, most, 0.0))
    del score
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)

    def back(t):  # [batch, key head, group, tokens, dim] as it came
        return t.permute(0, 3, 1, 2, 4).flatten(2, 3).contiguous()

    out = {"out": back(p @ v)}
    if train:
        do = _by_key_head(s["dout"], kv, to)
        out["dv"] = back((p.transpose(-1, -2).contiguous() @ do).sum(2, keepdim=True))
        dp = do @ v.transpose(-1, -2).contiguous()
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        del dp
        out["dq"] = back(ds @ k)
        out["dk"] = back((ds.transpose(-1, -2).contiguous() @ q).sum(2, keepdim=True))
    return out


def _plain_attention(s, case):
    found = _attend(s, case, torch.float32)
    return {n: t.to(s["q"].dtype) for n, t in found.items()}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = SIZE[case["dtype"]]
    if case["kind"] in ("norm", "norm8"):
        n, dim = case["rows"] * case["dim"], case["dim"]
        if case["kind"] == "norm8":
            read, written = n * (2 if case["residual"] else 1) * size, n + 4 * case["rows"] + (n * size if case["residual"] else 0)
            return {"bytes": read + written + dim * size, "flops": 6 * n}
        # forward: x and the residual, y and h; backward: h (or x), dy and dh, dx (one tensor for x and the residual)
        forward = n * (4 if case["residual"] else 2) * size + dim * size
        backward = (n * (4 if case["residual"] else 3) * size + 2 * dim * size) if case["train"] else 0
        return {"bytes": forward + backward, "flops": (16 if case["train"] else 5) * n}
    if case["kind"] == "rotary":
        tokens = math.prod(int(v) for v in case["grid"].split("x"))
        n = case["batch"] * tokens * (case["heads"] + case["kv_heads"]) * case["dim"]
        axes = case["grid"].count("x") + 1
        once = 2 * n * size + 4 * axes * tokens
        times = 2 if case["train"] else 1
        return {"bytes": times * once, "flops": times * 3 * n}
    if case["mask"] == "lengths":
        attended = sum(_lengths(case))
    elif case["mask"] == "mask":
        attended = case["batch"] * case["keys"] * 3 // 4
    else:
        attended = case["batch"] * case["keys"]
    rows = case["batch"] * case["queries"] * case["heads"] * case["dim"] * size
    keys = attended * case["kv_heads"] * case["dim"] * size
    all_keys = case["batch"] * case["keys"] * case["kv_heads"] * case["dim"] * size
    product = 2 * attended * case["queries"] * case["heads"] * case["dim"]
    if case["train"]:
        # forward: q, k, v, out; backward: q, k, v, out, dout, dq, dk, dv; five products beside the forward pass's two
        return {"bytes": 2 * rows + 2 * keys + 4 * rows + 2 * keys + 2 * all_keys, "flops": 7 * product}
    return {"bytes": 2 * rows + 2 * keys, "flops": 2 * product}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        return {"norm": _exact_norm, "norm8": _exact_norm, "rotary": _exact_rotary, "attention": _exact_attention}[case["kind"]](s, case)


def _exact_norm(s, case):
    x, w = s["x"].double(), s["weight"].double()
    h = x
    if s["residual"] is not None:  # the kept sum, rounded once
        h = (x + s["residual"].double()).to(s["x"].dtype).double()
    size = torch.sqrt((h * h).sum(1) / case["dim"] + EPS)[:, None]
    y = h / size * w
    out = {}
    if case["kind"] == "norm8":
        out["scale"] = y.abs().max(1).values / F8_MOST
        out["y"] = (y / out["scale"][:, None]).to(torch.float8_e4m3fn).double()
    else:
        out["y"] = y
    if s["residual"] is not None:
        out["h"] = h
    if case["train"]:
        dy = s["dy"].double()
        # y_i = w_i h_i / size, dsize / dh_j = h_j / (dim size)
        along = (dy * w * h).sum(1, keepdim=True) / (case["dim"] * size ** 3)
        out["dx"] = dy * w / size - h * along
        if s["residual"] is not None:
            out["dx"] = out["dx"] + s["dh"].double()
            out["dresidual"] = out["dx"]
        out["dweight"] = (dy * h / size).sum(0)
    return out


def _exact_rotary(s, case):
    n, dim = s["axis"].numel(), case["dim"]
    first = torch.arange(n, device=DEVICE) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else n)
    point = torch.polar(torch.ones(1, dtype=torch.float64, device=DEVICE),
                        s["positions"].double()[:, s["axis"].long()] * s["frequencies"])[:, None]

    def turned(t, by):
        t = t.double()
        z = torch.complex(t[..., first].contiguous(), t[..., second].contiguous()) * by
        u = t.clone()
        u[..., first], u[..., second] = z.real, z.imag
        return u

    out = {"q": turned(s["q"], point), "k": turned(s["k"], point)}
    if case["train"]:
        out["dq"], out["dk"] = turned(s["dq"], point.conj()), turned(s["dk"], point.conj())
    return out


def _exact_attention(s, case):
    if case["batch"] * case["heads"] * case["queries"] * case["keys"] > 6e8:
        return None
    q, k, v = (s[n].detach().double() for n in ("q", "k", "v"))
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    out = {"out": torch.zeros_like(q)}
    if case["train"]:
        out |= {"dq": torch.zeros_like(q), "dk": torch.zeros(k.shape, dtype=k.dtype, device=DEVICE),
                "dv": torch.zeros(v.shape, dtype=v.dtype, device=DEVICE)}
    for b in range(case["batch"]):
        # only the keys that are attended to
        if case["mask"] == "lengths":
            at = torch.arange(int(s["lengths"][b]), device=DEVICE)
        elif case["mask"] == "mask":
            at = torch.nonzero(s["mask"][b])[:, 0]
        else:
            at = torch.arange(case["keys"], device=DEVICE)
        if not at.numel():
            continue
        for head in range(case["heads"]):
            Q, K, V = q[b, :, head], k[b, at, head // group], v[b, at, head // group]
            P = torch.softmax(Q @ K.t() * scale, 1)
            out["out"][b, :, head] = P @ V
            if case["train"]:
                dO = s["dout"][b, :, head].double()
                dP = dO @ V.t()
                dS = P * (dP - (dO * out["out"][b, :, head]).sum(1, keepdim=True)) * scale
                out["dq"][b, :, head] = dS @ K
                out["dk"][b, at, head // group] += dS.t() @ Q
                out["dv"][b, at, head // group] += P.t() @ dO
    return out
