"""Timed operators of a factorized Transformer's training step that stand between the layers, through the public entry points:

  experts   tokens sorted by expert for the grouped layers, dispatched and combined again, with the gradients
  qk        root-mean-square norms of queries and keys for each head with the position rotation, forward and backward
  adamw     an AdamW step over a list of tensors, with states in 32 bits or in 8

`own` selects the library's calls; otherwise `run` computes the same in elementary torch operations.  Sizes are those of the
benchmark configurations (512 wide, 8 heads of 64, 64 sequences of 128 tokens, factors at a quarter of the width, a flat buffer
of 176 tensors) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # a batch of 20 sequences that generate: one new token each, two of eight experts
        _experts("experts step", "bf16", 20, 2, 8, 512, 0, train=False),
        # the expert feed-forward layers of a Transformer block in training, 64 sequences x 128 tokens, a quarter of spare room
        _experts("experts train", "bf16", 8192, 2, 8, 512, 1.25),
        # many small experts on a ragged width in single precision, rows packed without room between experts
        _experts("experts ragged f32", "f32", 1111, 3, 61, 1500, 0),
        # a wide layer on a large batch: the largest of its kind, 42 k rows of 8 KB
        _experts("experts wide", "bf16", 16384, 2, 64, 4096, 1.25),
        # one new token for each of 20 sequences at far positions: 8 heads of 64, queries and keys read from one projection
        _qk("qk step", "bf16", 20, 8, 8, 64, 64, train=False, far=True, fused=True),
        # the same heads in training, 64 sequences x 128 tokens: forward and backward
        _qk("qk train", "bf16", 8192, 8, 8, 64, 64),
        # shared key heads, interleaved pairs, only half of a head rotated: a prompt of odd length without a gradient
        _qk("qk prompt", "bf16", 5001, 32, 4, 128, 64, train=False, pairs=True, fused=True),
        # a large batch of wide heads in training: the largest of its kind
        _qk("qk large", "bf16", 16384, 32, 8, 128, 128),
        # all factors and biases of one feed-forward block in single precision: launches and host time
        _adamw("adamw block", "f32", "f32", 6, 2048, 218000, state8=False),
        # a whole network in mixed precision: fp32 masters, tensors as views of flat buffers
        _adamw("adamw flat", "bf16", "bf16", 176, 65535, 238573, state8=False, masters=True, flat=True),
        # the same network with states in 8 bits, no masters
        _adamw("adamw 8bit", "bf16", "bf16", 176, 65536, 238573, state8=True),
        # single-precision weights and gradients with states in 8 bits, small odd tensors
        _adamw("adamw 8bit ragged", "f32", "f32", 61, 513, 66001, state8=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("experts", "experts", "qk", "qk", "adamw", "adamw"))
    if kind == "experts":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        while True:
            experts = _log(rng, 2, 256)
            k = rng.randint(1, min(8, experts))
            tokens, width = _log(rng, 1, 32768), _log(rng, 64, 4096)
            if rng.random() < 0.6:
                width = max(64, width // 32 * 32)
            room = rng.choice((0, 0, 1.0, 1.25, 2.0))
            if tokens * k * width * max(1.0, room) * _BYTES[dtype] <= 1.3e8 * 2:
                break
        c = _experts("", dtype, tokens, k, experts, width, room, train=rng.random() < 0.7)
    elif kind == "qk":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        while True:
            k_heads = rng.choice((1, 2, 4, 5, 8))
            q_heads = k_heads * rng.choice((1, 1, 2, 4, 7))
            dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 192, 256, 2 * rng.randint(9, 90)))
            rot = dim if rng.random() < 0.7 else max(2, dim // 4 * 2)
            tokens = _log(rng, 1, 32768)
            if tokens * (q_heads + k_heads) * dim * _BYTES[dtype] <= 1.6e8:
                break
        c = _qk("", dtype, tokens, q_heads, k_heads, dim, rot, train=rng.random() < 0.6, pairs=rng.random() < 0.3, far=rng.random() < 0.4,
                fused=rng.random() < 0.5)
    else:
        dtype = rng.choice(("bf16", "bf16", "f32"))
        grad = "f32" if dtype == "f32" or rng.random() < 0.3 else "bf16"
        while True:
            tensors, small = _log(rng, 2, 400), _log(rng, 64, 65536)
            large = _log(rng, small, 1 << 22)
            if tensors * (small + large) / 2 <= 26.5e6:
                break
        state8 = rng.random() < 0.5
        c = _adamw("", dtype, grad, tensors, small, large, state8=state8, masters=dtype == "bf16" and rng.random() < 0.5,
                   flat=not state8 and rng.random() < 0.4)
    del c["name"]
    return c


def _experts(name, dtype, tokens, k, experts, width, room, train=True):
    """`room`: rows of each expert as a multiple of the mean, 0 for rows without gaps."""
    return {"name": name, "kind": "experts", "dtype": dtype, "tokens": tokens, "k": k, "experts": experts, "width": width,
            "capacity": math.ceil(room * tokens * k / experts), "train": train}


def _qk(name, dtype, tokens, q_heads, k_heads, dim, rot, train=True, pairs=False, far=False, fused=False):
    return {"name": name, "kind": "qk", "dtype": dtype, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "rot": rot,
            "train": train, "pairs": pairs, "far": far, "fused": fused}


def _adamw(name, dtype, grad, tensors, small, large, state8, masters=False, flat=False):
    return {"name": name, "kind": "adamw", "dtype": dtype, "grad": grad, "tensors": tensors, "small": small, "large": large,
            "state8": state8, "masters": masters, "flat": flat}


def _sizes(c):
    """Element counts of an AdamW case's tensors."""
    return [c["large"] if i % 2 else c["small"] for i in range(c["tensors"])]


def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(_sizes(c))
        each = _BYTES[c["grad"]] + (2 + 8 if c["masters"] else 2 * _BYTES[c["dtype"]]) + (4 if c["state8"] else 16)
        return {"bytes": n * each + (n // 256 * 16 if c["state8"] else 0), "flops": n * 15}
    s = _BYTES[c["dtype"]]
    if c["kind"] == "qk":
        n = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["dim"]
        return {"bytes": n * s * (5 if c["train"] else 2) + c["tokens"] * 8, "flops": n * (25 if c["train"] else 8)}
    n, kept = c["tokens"] * c["width"], c["tokens"] * c["k"] * c["width"]
    rows = _rows(c) * c["width"]
    lists = 4 * (2 * c["tokens"] * c["k"] + _rows(c)) + 4 * c["tokens"] * c["k"]
    forward = s * (n + rows + kept + n)
    return {"bytes": lists + forward + (s * (n + kept + rows + kept + n) if c["train"] else 0), "flops": kept * (7 if c["train"] else 2)}


def _rows(c):
    return c["experts"] * c["capacity"] if c["capacity"] else c["tokens"] * c["k"]


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"experts": _prepare_experts, "qk": _prepare_qk, "adamw": _prepare_adamw}[case["kind"]](case, g)


def _normal(g, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _prepare_experts(c, g):
    T, K, E, n, dt = c["tokens"], c["k"], c["experts"], c["width"], _TORCH[c["dtype"]]
    # a router's choice: some experts are liked better by all tokens
    logits = _normal(g, (T, E)) + _normal(g, (E,), scale=0.7)
    top, ids = logits.topk(K, dim=1)
    return {"case": c, "x": _normal(g, (T, n), dt), "ids": ids.to(torch.int32).contiguous(), "weights": top.softmax(dim=1).contiguous(),
            "ys": _normal(g, (_rows(c), n), dt), "dy": _normal(g, (T, n), dt) if c["train"] else None,
            "dxs": _normal(g, (_rows(c), n), dt) if c["train"] else None}


def _prepare_qk(c, g):
    T, Hq, Hk, D, dt = c["tokens"], c["q_heads"], c["k_heads"], c["dim"], _TORCH[c["dtype"]]
    if c["fused"]:      # queries, keys and values side by side, as one projection writes them
        rows = _normal(g, (T, Hq + 2 * Hk, D), dt, 1.7)
        q, k = rows[:, :Hq], rows[:, Hq:Hq + Hk]
    else:
        q, k = _normal(g, (T, Hq, D), dt, 1.7), _normal(g, (T, Hk, D), dt, 0.4)
    if c["far"]:
        positions = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda")
    else:               # sequences of 128 tokens, one behind the other
        positions = torch.arange(T, device="cuda") % 128
    half = c["rot"] // 2
    inv_freq = (10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
    s = {"case": c, "q": q, "k": k, "positions": positions, "inv_freq": inv_freq, "wq": (1 + 0.2 * _normal(g, (D,))).to(dt),
         "wk": (1 + 0.2 * _normal(g, (D,))).to(dt), "eps": 1e-6}
    if c["train"]:
        s["dq_out"], s["dk_out"] = _normal(g, (T, Hq, D), dt), _normal(g, (T, Hk, D), dt)
    return s


def _prepare_adamw(c, g):
    """Every list is views of one buffer: without gaps (`flat`), or each tensor on a multiple of 256 elements with zeros behind it."""
    sizes, step = _sizes(c), 1 if c["flat"] else 256
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // step) * step
    real = torch.zeros(at, device="cuda")
    for b, n in zip(starts, sizes):
        real[b:b + n] = 1
    split = lambda t: [t[b:b + n] for b, n in zip(starts, sizes)]  # noqa: E731
    blocks = lambda t: [t[b // 256:b // 256 + -(-n // 256)] for b, n in zip(starts, sizes)]  # noqa: E731
    p = _normal(g, (at,), scale=0.05) * real
    scale = torch.exp(_normal(g, (at,))) * 1e-3      # gradients of a network differ in size
    grads = (_normal(g, (at,)) * scale * real).to(_TORCH[c["grad"]])
    m, v = _normal(g, (at,)) * scale * 0.3 * real, (scale * real) ** 2 * (0.5 + torch.rand(at, generator=g, device="cuda"))
    s = {"case": c, "params": p.to(_TORCH[c["dtype"]]), "grads": grads, "masters": p if c["masters"] else None,
         "hyper": {"lr": 1e-3, "betas": (0.9, 0.98), "eps": 1e-8, "weight_decay": 0.01, "step": 1000, "grad_scale": 0.5, "seed": 12345}}
    if c["state8"]:
        lengths = torch.tensor([-(-n // 256) for n in sizes], device="cuda")
        tensor = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), lengths)
        first = torch.tensor([b // 256 for b in starts], device="cuda")[tensor]
        s["tensor"], s["index"] = tensor, (torch.arange(at // 256, device="cuda") - first) * 256
        noise = _noise(s, 7)
        s["m"], s["m_scales"] = _encode(m.view(-1, 256), noise & 0xFFFF, torch.float8_e4m3fn)
        s["v"], s["v_scales"] = _encode(v.view(-1, 256), noise >> 16, torch.float8_e5m2)
        s["m"], s["v"] = s["m"].view(-1), s["v"].view(-1)
        s["lists"] = {"m_scales": blocks(s["m_scales"]), "v_scales": blocks(s["v_scales"])}
    else:
        s["m"], s["v"], s["lists"] = m, v, {}
    for name in ("params", "grads", "m", "v"):
        s["lists"][name] = split(s[name])
    if c["masters"]:
        s["lists"]["masters"] = split(s["masters"])
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2103_03936_b200 as pf
        return {"experts": _own_experts, "qk": _own_qk, "adamw": _own_adamw}[kind](pf, state)
    return {"experts": _plain_experts, "qk": _plain_qk, "adamw": _plain_adamw}[kind](state)


def _own_experts(pf, s):
    c = s["case"]
    slots, sources, counts, offsets = pf.pf_expert_sort(s["ids"], c["experts"], capacity=c["capacity"])
    out = {"slots": slots, "sources": sources, "counts": counts, "offsets": offsets,
           "xs": pf.pf_expert_dispatch_fwd(s["x"], slots, sources), "y": pf.pf_expert_combine_fwd(s["ys"], slots, s["weights"])}
    if c["train"]:
        out["dys"], out["dweights"] = pf.pf_expert_combine_bwd(s["ys"], slots, sources, s["weights"], s["dy"])
        out["dx"] = pf.pf_expert_dispatch_bwd(s["dxs"], slots)
    return out


def _own_qk(pf, s):
    style = pf.PF_ROPE_PAIRS if s["case"]["pairs"] else pf.PF_ROPE_HALVES
    rest = {"positions": s["positions"], "style": style, "eps": s["eps"]}
    out = {}
    out["q_out"], out["k_out"] = pf.pf_qk_norm_rope_fwd(s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], **rest)
    if s["case"]["train"]:
        out["dq"], out["dk"], out["dwq"], out["dwk"] = pf.pf_qk_norm_rope_bwd(s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], s["dq_out"],
                                                                               s["dk_out"], **rest)
    return out


def _own_adamw(pf, s):
    pf.pf_adamw_step(**s["lists"], **s["hyper"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {name: s[name] for name in ("params", "masters", "m", "v", "m_scales", "v_scales") if s.get(name) is not None}


# ------------------------------------------------------------------------------------ the plain forms
def _plain_experts(s):
    c, T, K, E, C = s["case"], s["case"]["tokens"], s["case"]["k"], s["case"]["experts"], s["case"]["capacity"]
    dt, device, rows = s["x"].dtype, s["x"].device, _rows(c)
    ids = s["ids"].reshape(-1).long()
    order = torch.argsort(ids, stable=True)
    counts = (ids[:, None] == torch.arange(E, device=device)).sum(dim=0)
    ends = counts.cumsum(0)
    sorted_ids = ids[order]
    rank = torch.arange(T * K, device=device) - (ends - counts)[sorted_ids]
    if C:
        offsets = torch.arange(E + 1, device=device) * C
        place = torch.where(rank < C, sorted_ids * C + rank, rows)      # `rows`: no place
    else:
        offsets = torch.cat([ends.new_zeros(1), ends])
        place = torch.arange(T * K, device=device)
    slots = torch.empty_like(ids).scatter_(0, order, place)
    sources = torch.full((rows + 1,), -1, dtype=torch.int64, device=device).scatter_(0, place, order)[:rows]
    took = slots < rows
    taken = (sources >= 0)[:, None]
    gather = sources.clamp(min=0)
    at = torch.where(took, slots, 0)
    keep = took.view(T, K, 1)
    out = {"slots": torch.where(took, slots, -1).view(T, K).to(torch.int32), "sources": sources.to(torch.int32), "counts": counts.to(torch.int32),
           "offsets": offsets.to(torch.int32)}
    out["xs"] = torch.where(taken, s["x"][gather // K], 0)
    w = s["weights"].unsqueeze(2)
    rows_of = torch.where(keep, s["ys"][at].view(T, K, -1).float(), 0)
    out["y"] = (rows_of * w).sum(dim=1).to(dt)
    if c["train"]:
        dy = s["dy"].float()
        out["dys"] = torch.where(taken, dy[gather // K] * s["weights"].reshape(-1)[gather][:, None], 0).to(dt)
        out["dweights"] = (rows_of * dy.unsqueeze(1)).sum(dim=2)
        out["dx"] = torch.where(keep, s["dxs"][at].view(T, K, -1).float(), 0).sum(dim=1).to(dt)
    return out


def _plain_turn(x, cos, sin, rot, pairs):
    """Rotates the first `rot` elements of each row by the angles of `cos` and `sin` [T, 1, rot / 2]."""
    turned, rest = x[..., :rot], x[..., rot:]
    if pairs:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _plain_qk(s):
    c = s["case"]
    rot, pairs = c["rot"], c["pairs"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()      # (far positions lose their angle in 32 bits)
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k, wq, wk = s["q"].float(), s["k"].float(), s["wq"].float(), s["wk"].float()
    rq, rk = torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]), torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"])
    nq, nk = q * rq, k * rk
    out = {"q_out": _plain_turn(nq * wq, cos, sin, rot, pairs).to(s["q"].dtype), "k_out": _plain_turn(nk * wk, cos, sin, rot, pairs).to(s["k"].dtype)}
    if c["train"]:
        eq, ek = _plain_turn(s["dq_out"].float(), cos, -sin, rot, pairs), _plain_turn(s["dk_out"].float(), cos, -sin, rot, pairs)
        dnq, dnk = eq * wq, ek * wk
        out["dq"] = (rq * (dnq - nq * (dnq * nq).mean(-1, keepdim=True))).to(s["q"].dtype)
        out["dk"] = (rk * (dnk - nk * (dnk * nk).mean(-1, keepdim=True))).to(s["k"].dtype)
        out["dwq"], out["dwk"] = (eq * nq).sum(dim=(0, 1)).to(s["wq"].dtype), (ek * nk).sum(dim=(0, 1)).to(s["wk"].dtype)
    return out


def _noise(s, seed):
    """32 random bits for each element from the seed, the tensor's place in the list and the element's in the tensor, [blocks, 256]."""
    key = (seed + (s["tensor"] + 1) * 0x9E3779B9) & 0xFFFFFFFF
    x = (s["index"][:, None] + torch.arange(256, device="cuda")) ^ key[:, None]
    x = (x * 0xA3D95FA7) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xC8B1F265) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _encode(x, noise16, dtype):
    """Blocks of 256 as 8-bit floats times a power of two for each block, rounded up with the probability of what is cut off."""
    top, cut, floor = (7, 20, 8) if dtype == torch.float8_e4m3fn else (14, 21, 16)
    bits = x.contiguous().view(torch.int32).long()
    size = bits & 0x7FFFFFFF
    field = ((size.amax(dim=1, keepdim=True) >> 23) - top).clamp(min=floor)      # exponent of the scale, as in fp32
    scaled = size + (noise16 << (cut - 16)) - ((field - (7 if top == 7 else 15)) << 23)
    least = 1 << 23                                                              # the smallest normal number of the type
    code = torch.where(scaled < least, 0, scaled >> cut)
    if dtype == torch.float8_e4m3fn:
        code = code | ((bits >> 24) & 0x80)
        code = torch.where(scaled < least, 0, code)
    else:                                                                        # a square never becomes zero by rounding
        code = torch.where((scaled < least) & (size > 0), least >> cut, code)
    return code.to(torch.uint8).view(dtype), (field << 23).to(torch.int32).view(torch.float32).view(-1)


def _plain_adamw(s):
    h, state8 = s["hyper"], s["case"]["state8"]
    b1, b2 = h["betas"]
    g = s["grads"].float() * h["grad_scale"]
    if state8:
        m = (s["m"].float().view(-1, 256) * s["m_scales"][:, None]).view(-1)
        v = (s["v"].float().view(-1, 256) * s["v_scales"][:, None]).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    p = s["masters"] if s["masters"] is not None else s["params"].float()
    update = (m / (1 - b1 ** h["step"])) / (torch.sqrt(v / (1 - b2 ** h["step"])) + h["eps"])
    p = p - h["lr"] * (h["weight_decay"] * p + update)
    if s["masters"] is not None:
        s["masters"].copy_(p)
    s["params"].copy_(p)
    if state8:
        noise = _noise(s, h["seed"])
        codes, scales = _encode(m.view(-1, 256), noise & 0xFFFF, torch.float8_e4m3fn)
        s["m"].copy_(codes.view(-1)), s["m_scales"].copy_(scales)
        codes, scales = _encode(v.view(-1, 256), noise >> 16, torch.float8_e5m2)
        s["v"].copy_(codes.view(-1)), s["v_scales"].copy_(scales)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    return _adamw_outputs(s)


# ------------------------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"experts": _exact_experts, "qk": _exact_qk, "adamw": _exact_adamw}[case["kind"]](s)


def _exact_experts(s):
    """Assignment after assignment on the host for the lists, expert after expert for the rows."""
    c = s["case"]
    T, K, E, C, rows = c["tokens"], c["k"], c["experts"], c["capacity"], _rows(c)
    ids = s["ids"].reshape(-1).tolist()
    members = [[] for _ in range(E)]
    for a, e in enumerate(ids):
        members[e].append(a)
    counts = [len(m) for m in members]
    offsets = [0]
    for e in range(E):
        offsets.append(offsets[-1] + (C if C else counts[e]))
    slots, sources = [-1] * (T * K), [-1] * rows
    for e in range(E):
        for r, a in enumerate(members[e][:C] if C else members[e]):
            slots[a] = offsets[e] + r
            sources[offsets[e] + r] = a
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    x, ys, w = s["x"], s["ys"], s["weights"].double().view(-1)
    xs, y = torch.zeros(rows, c["width"], dtype=torch.float64, device="cuda"), torch.zeros(T, c["width"], dtype=torch.float64, device="cuda")
    out = {"slots": i32(slots).view(T, K), "sources": i32(sources), "counts": i32(counts), "offsets": i32(offsets), "xs": xs, "y": y}
    if c["train"]:
        dys, dw, dx = torch.zeros_like(xs), torch.zeros(T * K, dtype=torch.float64, device="cuda"), torch.zeros_like(y)
        out["dys"], out["dweights"], out["dx"] = dys, dw.view(T, K), dx
    for e in range(E):
        a = i32(members[e][:C] if C else members[e]).long()
        if len(a) == 0:
            continue
        r, t = slice(offsets[e], offsets[e] + len(a)), a // K
        xs[r] = x[t].double()
        y.index_add_(0, t, ys[r].double() * w[a][:, None])
        if c["train"]:
            dy = s["dy"][t].double()
            dys[r] = dy * w[a][:, None]
            dw[a] = (dy * ys[r].double()).sum(dim=1)
            dx.index_add_(0, t, s["dxs"][r].double())
    return out


def _exact_qk(s):
    """Rotation as a product of complex numbers, gradients by differentiating it."""
    c, out = s["case"], {}
    rot = c["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())[:, None, :]
    for name in ("q", "k"):
        x, w = s[name].double().detach().requires_grad_(c["train"]), s["w" + name].double().detach().requires_grad_(c["train"])
        z = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + s["eps"]) * w
        pair = z[..., :rot].unflatten(-1, (rot // 2, 2) if c["pairs"] else (2, rot // 2))
        pair = pair if c["pairs"] else pair.transpose(-1, -2)
        pair = torch.view_as_real(torch.complex(pair[..., 0], pair[..., 1]) * turn)
        pair = pair if c["pairs"] else pair.transpose(-1, -2)
        y = torch.cat([pair.flatten(-2), z[..., rot:]], dim=-1)
        out[name + "_out"] = y.detach()
        if c["train"]:
            out["d" + name], out["dw" + name] = torch.autograd.grad(y, (x, w), s["d" + name + "_out"].double())
    return out


def _exact_adamw(s):
    """Block after block in 64 bits.  The 8-bit states have no such value: which way a value is rounded goes by its 32-bit form."""
    h, c = s["hyper"], s["case"]
    b1, b2 = h["betas"]
    g, p = s["grads"].double() * h["grad_scale"], (s["masters"] if c["masters"] else s["params"]).double()
    m, v = s["m"].double(), s["v"].double()
    if c["state8"]:
        m, v = m * s["m_scales"].double().repeat_interleave(256), v * s["v_scales"].double().repeat_interleave(256)
    m, v = torch.lerp(g, m, b1), torch.lerp(g * g, v, b2)
    p = p * (1 - h["lr"] * h["weight_decay"]) - h["lr"] / (1 - b1 ** h["step"]) * m / (v.sqrt() / math.sqrt(1 - b2 ** h["step"]) + h["eps"])
    out = {"params": p}
    if c["masters"]:
        out["masters"] = p
    if c["state8"]:
        return {**out, "m": None, "v": None, "m_scales": None, "v_scales": None}
    return {**out, "m": m, "v": v}
