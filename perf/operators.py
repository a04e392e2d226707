"""Cases of the operators around attention and the gradients: rotary positions, attention with
rules on its scores, and clipping by the global norm of many gradients.

One pass of a case is what a program asks for a batch, or for the next tokens of running sequences.
A case is a dict of plain values:
  op "rope"   B, S, Hq, Hkv, D; rot (leading part of the head that turns), interleaved, inverse (the
              backward pass), n_pos (rows of the table), layout "bhsd" | "bshd" (how the tensors lie)
  op "train"  attention forward and backward over B x S tokens, Hq query and Hkv key/value heads
  op "prompt" attention forward over the same
  op "token"  attention of the last S tokens of every sequence over its cache, room for C tokens;
              sequence lengths from `lengths` of C up to C
              mask: "causal" | "full" | "docs" (packed documents of about `doc` tokens, with padding at
              the end of a row) | "prefix" (the same, the first part of every document seen by all of it)
              cap: scores capped at +-cap (0: no cap); slopes: a bias by distance, a slope per head
  op "clip"   tensors gradients of rank-`rank` branches of a model (d, F), or of sizes lo..hi; dtype
              "mixed": bf16 and fp32; over: the norm is that many times the largest allowed
`layout_seed` draws lengths of documents, caches and tensors, so that the work of a case is known.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rope(B, S, Hq, Hkv, D, rot, dtype="bf16", interleaved=False, inverse=False, n_pos=4096, layout="bshd"):
    return {"op": "rope", "B": B, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "dtype": dtype, "interleaved": interleaved,
            "inverse": inverse, "n_pos": n_pos, "layout": layout}


def _attn(op, B, S, Hq, Hkv, D, dtype="bf16", mask="causal", cap=0.0, slopes=False, doc=0, C=0, lengths=1.0, layout="bshd",
          layout_seed=1):
    return {"op": op, "B": B, "S": S, "C": C or S, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "mask": mask, "cap": cap,
            "slopes": slopes, "doc": doc, "lengths": lengths, "layout": layout, "layout_seed": layout_seed}


def _clip(tensors, dtype, d=0, F=0, rank=0, lo=0, hi=0, over=3.0, layout_seed=1):
    return {"op": "clip", "tensors": tensors, "dtype": dtype, "d": d, "F": F, "rank": rank, "lo": lo, "hi": hi, "over": over,
            "layout_seed": layout_seed}


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # the next token of 16 running sequences: a launch, and little else
    add("rope_token", _rope(16, 1, 32, 32, 64, 64, n_pos=32768))
    # queries and keys of a training batch as the projections write them
    add("rope_6.7b", _rope(4, 2048, 32, 32, 128, 128))
    # the backward pass of neighbouring pairs on half of a head, single precision, a length that is no power of two
    add("rope_back_f32_ragged", _rope(3, 1021, 12, 12, 64, 32, dtype="f32", interleaved=True, inverse=True, layout="bhsd"))
    # a training batch packed from documents, scores falling with distance
    add("train_1.3b_packed", _attn("train", 8, 1024, 32, 32, 64, mask="docs", doc=300, slopes=True))
    # four query heads to a key/value head, capped scores
    add("train_6.7b_capped", _attn("train", 4, 2048, 32, 8, 128, cap=15.0))
    # a small model's batch of odd length: prefixes seen whole, rows of padding; half precision
    add("train_125m_prefix_f16", _attn("train", 3, 777, 12, 12, 64, dtype="f16", mask="prefix", doc=190, layout="bhsd"))
    # a long prompt before generation
    add("prompt_6.7b_long", _attn("prompt", 1, 8192, 32, 8, 128))
    # the next token of eight short sequences, lengths all different
    add("token_1.3b", _attn("token", 8, 1, 32, 32, 64, dtype="f16", slopes=True, C=1024, lengths=0.1, layout="bhsd"))
    # the next token of four long sequences with capped scores: the cache is read once
    add("token_6.7b_long", _attn("token", 4, 1, 32, 8, 128, cap=15.0, C=32768, lengths=0.3, layout="bhsd"))
    # gradients of a rank-16 branch in every layer of a small model: few and small
    add("clip_125m_lora", _clip(24, "bf16", d=768, F=4 * 768, rank=16))
    # the fp32 gradients that the low-rank calls of this package write for 24 layers
    add("clip_1.3b_lora", _clip(48, "f32", d=2048, F=8192, rank=64))
    # every weight and bias of a part of a model: many tensors, from odd small ones to whole matrices
    add("clip_many", _clip(200, "mixed", lo=64, hi=1 << 24))
    return c


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _scores(c):
    return c["B"] * c["Hq"] * c["S"] * c["C"]


def draw(rng):
    """Models of 8 to 64 heads, 1 to 8192 tokens, caches up to 32768, every type, layout and mask."""
    while True:
        op = rng.choice(["rope", "rope", "train", "train", "train", "prompt", "token", "token", "clip", "clip"])
        D = rng.choice([64, 128])
        Hkv = rng.choice([1, 2, 4, 8, 12, 16, 32])
        Hq = Hkv * rng.choice([1, 1, 2, 4, 8])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        layout = rng.choice(["bshd", "bhsd"])
        if Hq > 64:
            continue
        if op == "rope":
            D = rng.choice([64, 80, 96, 128, 256])
            rot = rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)])
            inverse = rng.random() < 0.5
            c = _rope(rng.randint(1, 16), round(_log(rng, 1, 4096)), Hq, Hkv, D, rot, dtype=rng.choice(["bf16", "f16", "f32"]),
                      interleaved=rng.random() < 0.5, inverse=inverse, n_pos=rng.choice([4096, 32768]), layout=layout)
            if 4096 * 4 * 64 * 128 < c["B"] * c["S"] * (Hq + Hkv) * D:
                continue
            return c
        if op == "clip":
            if rng.random() < 0.5:
                d = 64 * round(_log(rng, 8, 64))
                return _clip(2 * rng.randint(1, 40), rng.choice(["bf16", "f16", "f32"]), d=d, F=4 * d, rank=rng.choice([8, 16, 64]),
                             over=rng.choice([0.5, 4.0]), layout_seed=rng.randint(1, 10 ** 6))
            return _clip(round(_log(rng, 2, 300)), rng.choice(["bf16", "f16", "f32", "mixed"]), lo=rng.choice([1, 64, 1000]),
                         hi=round(_log(rng, 2000, 4000000)), over=rng.choice([0.5, 4.0]), layout_seed=rng.randint(1, 10 ** 6))
        cap = rng.choice([0.0, 0.0, 10.0, 30.0])
        slopes = rng.random() < 0.4
        if op == "token":
            c = _attn("token", rng.randint(1, 16), rng.choice([1, 1, 1, 2, 5]), Hq, Hkv, D, dtype=dtype, cap=cap, slopes=slopes,
                      C=round(_log(rng, 64, 32768)), lengths=rng.choice([0.1, 0.5, 1.0]), layout=layout, layout_seed=rng.randint(1, 10 ** 6))
            if c["B"] * Hkv * c["C"] * D > 4 * 8 * 32768 * 128 or _scores(c) > 2 ** 28:
                continue
            return c
        S = round(_log(rng, 1, 2048 if op == "train" else 8192))
        c = _attn(op, rng.randint(1, 8), S, Hq, Hkv, D, dtype=dtype, mask=rng.choice(["causal", "causal", "full", "docs", "prefix"]), cap=cap,
                  slopes=slopes, doc=round(_log(rng, 8, 1500)), layout=layout, layout_seed=rng.randint(1, 10 ** 6))
        if _scores(c) > (4 * 32 * 2048 ** 2 if op == "train" else 32 * 8192 ** 2 // 2):
            continue
        return c


def _documents(c):
    """[(begin, end, prefix)] over the flattened tokens of a packed batch; what no document holds is padding."""
    rng, out = random.Random(c["layout_seed"]), []
    for b in range(c["B"]):
        at, end = b * c["S"], (b + 1) * c["S"] - (rng.randint(0, c["S"] // 8) if rng.random() < 0.5 else 0)
        while at < end:
            n = min(end - at, 1 + int(rng.expovariate(1.0 / c["doc"])))
            out.append((at, at + n, rng.randint(0, n) if c["mask"] == "prefix" else 0))
            at += n
    return out


def _lengths(c):
    rng = random.Random(c["layout_seed"])
    low = max(c["S"], int(c["C"] * c["lengths"]))
    return [min(c["C"], max(c["S"], rng.randint(min(low, c["C"]), c["C"]))) for _ in range(c["B"])]


def _sizes(c):
    """[(dtype, size)] of a set of gradients."""
    rng = random.Random(c["layout_seed"])
    if c["rank"]:
        return [(c["dtype"], c["rank"] * (c["d"] if i % 2 == 0 else c["F"])) for i in range(c["tensors"])]
    out = []
    for i in range(c["tensors"]):
        n = round(_log(rng, c["lo"], c["hi"]))
        out.append((c["dtype"] if c["dtype"] != "mixed" else rng.choice(["bf16", "f32"]), max(1, n if rng.random() < 0.5 else n // 64 * 64)))
    return out


def _tensor(g, c, H, S, scale=1.0):
    """[B, H, S, D] in the case's layout, seeded."""
    shape = (c["B"], H, S, c["D"]) if c["layout"] == "bhsd" else (c["B"], S, H, c["D"])
    t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(_DT[c["dtype"]])
    return t if c["layout"] == "bhsd" else t.transpose(1, 2)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "rope":
        s["Q"], s["K"] = _tensor(g, c, c["Hq"], c["S"]), _tensor(g, c, c["Hkv"], c["S"])
        f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
        angle = torch.arange(c["n_pos"], dtype=torch.float64)[:, None] * f[None]
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        first = torch.randint(0, c["n_pos"] - c["S"] + 1, (c["B"], 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(c["S"], device="cuda")).to(torch.int32)
        s["Q_out"], s["K_out"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
        return s
    if c["op"] == "clip":
        sizes = _sizes(c)
        names = sorted({d for d, _ in sizes})
        total = {d: sum(n for t, n in sizes if t == d) for d in names}
        s["flat"] = {d: torch.randn(total[d], generator=g, device="cuda").mul_(0.01).to(_DT[d]) for d in names}
        s["out"] = {d: torch.empty_like(s["flat"][d]) for d in names}
        views = {d: iter(zip(s["flat"][d].split([n for t, n in sizes if t == d]), s["out"][d].split([n for t, n in sizes if t == d]))) for d in names}
        pairs = [next(views[d]) for d, _ in sizes]
        s["grads"], s["outs"] = [p[0] for p in pairs], [p[1] for p in pairs]
        s["max_norm"] = 0.01 * math.sqrt(sum(n for _, n in sizes)) / c["over"]
        s["norm"] = torch.empty(1, device="cuda")
        s["set"] = None
        return s
    # scores of standard deviation about one, two where they are capped
    s["Q"] = _tensor(g, c, c["Hq"], c["S"], 2.0 if c["cap"] else 1.0)
    s["K"], s["V"] = _tensor(g, c, c["Hkv"], c["C"]), _tensor(g, c, c["Hkv"], c["C"])
    s["O"] = torch.empty_like(s["Q"])
    s["LSE"] = torch.empty((c["B"], c["Hq"], c["S"]), device="cuda")
    s["scale"] = c["D"] ** -0.5
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device="cuda", dtype=torch.float32) / c["Hq"]) if c["slopes"] else None
    if c["op"] == "token":
        s["q_start"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda") - c["S"]
    if c["op"] == "train":
        s["dO"] = _tensor(g, c, c["Hq"], c["S"])
        s["dQ"], s["dK"], s["dV"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"]), torch.empty_like(s["V"])
    if c["mask"] in ("docs", "prefix"):
        docs = torch.tensor(_documents(c), dtype=torch.int32, device="cuda").reshape(-1, 3)
        s["doc_begin"], s["doc_end"], s["doc_prefix"] = (docs[:, i].contiguous() for i in range(3))
        s["key_lo"], s["key_hi"] = (torch.empty((c["B"], c["S"]), dtype=torch.int32, device="cuda") for _ in range(2))
    return s


# ---- plain forms: elementary operations in 32 bits -------------------------------------------------


def _plain_turn(u, s):
    c = s["case"]
    h = c["rot"] // 2
    row = s["table"][s["positions"].long()][:, None]          # [B, 1, S, rot]
    cos, sin = row[..., :h], row[..., h:]
    if c["inverse"]:
        sin = -sin
    t = u.float()
    x, y = (t[..., 0:c["rot"]:2], t[..., 1:c["rot"]:2]) if c["interleaved"] else (t[..., :h], t[..., h:c["rot"]])
    a, b = x * cos - y * sin, x * sin + y * cos
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, t[..., c["rot"]:]], -1).to(u.dtype)


def _plain_allowed(s):
    """[B, 1, S, C] truth values, and [B, 1, S, C] distances."""
    c = s["case"]
    k = torch.arange(c["C"], device="cuda")
    q = (s["q_start"].long()[:, None] if "q_start" in s else c["C"] - c["S"]) + torch.arange(c["S"], device="cuda").expand(c["B"], c["S"])
    far = (q[:, :, None] - k).abs()[:, None]
    if c["mask"] == "full":
        return torch.ones_like(far, dtype=torch.bool), far
    seen = (k <= q[:, :, None])[:, None]
    if c["mask"] == "causal":
        return seen, far
    token = torch.arange(c["B"] * c["S"], device="cuda")
    doc = torch.searchsorted(s["doc_begin"].long(), token, right=True) - 1
    at = doc.clamp(min=0)
    held = (doc >= 0) & (token < s["doc_end"].long()[at])
    doc = torch.where(held, doc, -1 - token).reshape(c["B"], c["S"])
    early = (held & (token < s["doc_begin"].long()[at] + s["doc_prefix"].long()[at])).reshape(c["B"], c["S"])
    same = (doc[:, :, None] == doc[:, None, :]) & held.reshape(c["B"], c["S"])[:, :, None]
    return (same & (seen[:, 0] | early[:, None, :]))[:, None], far


def _plain_scores(s, Q, K):
    """Masked scores after the rules on them, and the derivative by the capped score (None: 1)."""
    c = s["case"]
    allowed, far = _plain_allowed(s)
    z = torch.matmul(Q, K.transpose(-1, -2)) * s["scale"]
    slope = None
    if c["cap"]:
        t = torch.tanh(z / c["cap"])
        z, slope = t * c["cap"], 1 - t * t
    if s["slopes"] is not None:
        z = z - s["slopes"][None, :, None, None] * far
    return z.masked_fill(~allowed, -math.inf), slope


def _plain_attention(s):
    c = s["case"]
    group = c["Hq"] // c["Hkv"]
    Q, K, V = s["Q"].float(), s["K"].float().repeat_interleave(group, 1), s["V"].float().repeat_interleave(group, 1)
    z, slope = _plain_scores(s, Q, K)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    P = e / torch.where(total == 0, 1.0, total)
    O = torch.matmul(P, V)
    if c["op"] != "train":
        return O.to(s["Q"].dtype)
    dO = s["dO"].float()
    dV = torch.matmul(P.transpose(-1, -2), dO)
    dS = P * (torch.matmul(dO, V.transpose(-1, -2)) - (dO * O).sum(-1, keepdim=True)) * s["scale"]
    if slope is not None:
        dS = dS * slope
    dQ, dK = torch.matmul(dS, K), torch.matmul(dS.transpose(-1, -2), Q)
    shared = (c["B"], c["Hkv"], group, c["C"], c["D"])
    return [t.to(s["Q"].dtype) for t in (O, dQ, dK.reshape(shared).sum(2), dV.reshape(shared).sum(2))]


def _plain_clip(s):
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return {"norm": norm.reshape(1), "out": {d: (t.float() * factor).to(t.dtype) for d, t in s["flat"].items()}}


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "rope":
            return [_plain_turn(s["Q"], s), _plain_turn(s["K"], s)]
        return _plain_clip(s) if c["op"] == "clip" else _plain_attention(s)
    from paper_2510_15964_amd import lx
    if c["op"] == "rope":
        lx.lx_rope(s["Q"], s["K"], s["table"], s["positions"], s["Q_out"], s["K_out"], interleaved=c["interleaved"], inverse=c["inverse"])
        return [s["Q_out"], s["K_out"]]
    if c["op"] == "clip":
        if s["set"] is None:      # made once for the gradients of a model
            s["set"] = lx.GradSet(s["grads"], s["outs"])
        lx.lx_grad_norm_clip(s["set"], s["max_norm"], s["norm"])
        return {"norm": s["norm"], "out": s["out"]}
    rules = {"cap": c["cap"], "slopes": s["slopes"], "q_start": s.get("q_start")}
    causal = c["mask"] == "causal"
    if "key_lo" in s:
        lx.lx_attn_key_ranges(s["doc_begin"], s["doc_end"], s["doc_prefix"], True, s["key_lo"], s["key_hi"])
        rules.update(key_lo=s["key_lo"], key_hi=s["key_hi"])
    lx.lx_score_attn_fwd(s["Q"], s["K"], s["V"], s["scale"], causal, s["O"], s["LSE"], **rules)
    if c["op"] != "train":
        return s["O"]
    lx.lx_score_attn_bwd(s["Q"], s["K"], s["V"], s["O"], s["LSE"], s["dO"], s["scale"], causal, s["dQ"], s["dK"], s["dV"], **rules)
    return [s["O"], s["dQ"], s["dK"], s["dV"]]


def _pairs(c):
    """Allowed (query, key) pairs of one head, over the batch."""
    if c["op"] == "token":
        return sum(c["S"] * n - c["S"] * (c["S"] - 1) // 2 for n in _lengths(c))
    if c["mask"] == "full":
        return c["B"] * c["S"] * c["C"]
    if c["mask"] == "causal":
        return c["B"] * c["S"] * (c["S"] + 1) // 2
    return sum(p * p + ((e - b) * (e - b + 1) - p * (p + 1)) // 2 for b, e, p in _documents(c))


def work(case):
    c = case
    if c["op"] == "clip":
        sizes = _sizes(c)
        return {"bytes": sum(n * (8 if d == "f32" else 4) for d, n in sizes) + 4, "flops": sum(3 * n for _, n in sizes)}
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rope":
        rows = c["B"] * c["S"]
        n = rows * (c["Hq"] + c["Hkv"])
        return {"bytes": 2 * n * c["D"] * size + rows * 4 + min(rows, c["n_pos"]) * c["rot"] * 4, "flops": 3 * n * c["rot"]}
    q = c["B"] * c["Hq"] * c["S"] * c["D"] * size
    if c["op"] == "token":
        return {"bytes": 2 * q + 2 * sum(_lengths(c)) * c["Hkv"] * c["D"] * size, "flops": 4 * c["D"] * c["Hq"] * _pairs(c)}
    kv = c["B"] * c["Hkv"] * c["C"] * c["D"] * size
    return {"bytes": 4 * q + 4 * kv if c["op"] == "train" else 2 * q + 2 * kv, "flops": (14 if c["op"] == "train" else 4) * c["D"] * c["Hq"] * _pairs(c)}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def _exact_rope(s, u):
    c = s["case"]
    out = u.double().clone()
    h = c["rot"] // 2
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + h)
        w = torch.complex(s["table"][:, i].double(), s["table"][:, h + i].double())[s["positions"].long()][:, None]
        z = torch.complex(u[..., a].double(), u[..., b].double()) * (w.conj() if c["inverse"] else w)
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_seen(s, b):
    """[S, C]: which keys the queries of sequence b see."""
    c = s["case"]
    m = torch.zeros((c["S"], c["C"]), dtype=torch.bool)
    if c["op"] == "token":
        n = _lengths(c)[b]
        for i in range(c["S"]):
            m[i, :n - c["S"] + i + 1] = True
    elif c["mask"] == "full":
        m[:] = True
    elif c["mask"] == "causal":
        m = m.logical_not().tril()
    else:
        for x, y, p in _documents(c):
            if x // c["S"] == b:
                x, y = x - b * c["S"], y - b * c["S"]
                m[x:y, x:y] = torch.ones((y - x, y - x), dtype=torch.bool).tril()
                m[x:y, x:x + p] = True
    return m.cuda()


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "rope":
        return [_exact_rope(s, s["Q"]), _exact_rope(s, s["K"])]
    if c["op"] == "clip":
        norm = math.sqrt(sum(float(torch.dot(t.double(), t.double())) for t in s["flat"].values()))
        return {"norm": torch.tensor([norm], dtype=torch.float64),
                "out": {d: t.double() * min(1.0, s["max_norm"] / norm) for d, t in s["flat"].items()}}
    group = c["Hq"] // c["Hkv"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    dQ = torch.zeros_like(O)
    dK, dV = (torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(c["B"]):
        seen = _exact_seen(s, b)
        some = seen.any(1)
        if not bool(some.any()):
            continue
        seen = seen[some]
        place = torch.arange(c["S"], device="cuda")[some] + (_lengths(c)[b] if c["op"] == "token" else c["C"]) - c["S"]
        far = (torch.arange(c["C"], device="cuda")[None, :] - place[:, None]).abs().double()
        for h in range(c["Hq"]):
            q, k, v = s["Q"][b, h][some].double(), s["K"][b, h // group].double(), s["V"][b, h // group].double()
            z = q @ k.t().contiguous() * s["scale"]
            gain = torch.full_like(z, s["scale"])
            if c["cap"]:
                gain = gain / torch.cosh(z / c["cap"]) ** 2
                z = c["cap"] * torch.tanh(z / c["cap"])
            if c["slopes"]:
                z = z - float(s["slopes"][h]) * far
            P = torch.softmax(torch.where(seen, z, -math.inf), -1)
            o = P @ v
            O[b, h, some] = o
            if c["op"] == "train":
                do = s["dO"][b, h][some].double()
                dV[b, h // group] += P.t().contiguous() @ do
                dS = P * (do @ v.t().contiguous() - (do * o).sum(-1, keepdim=True)) * gain
                dQ[b, h, some] = dS @ k
                dK[b, h // group] += dS.t().contiguous() @ q
    return [O, dQ, dK, dV] if c["op"] == "train" else O
