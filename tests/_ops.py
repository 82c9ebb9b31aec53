"""Plain 64-bit forms of the operators around the layers, and the comparisons that their tests make."""
import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative


def close(got, want, slack, what):
    """|got - want| <= half a step of got's type + slack (a tensor: what fp32 arithmetic may be off by), element by element."""
    err = (got.double() - want).abs()
    allowed = U[got.dtype] * want.abs() + slack + 1e-44
    bad = ~(err <= allowed)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / allowed).max()):.3g} of what is allowed"


# ---------------------------------------------------------------------------- experts
def sort(ids, experts, capacity):
    """Lists of slots, sources, counts and offsets of assignments ids (a nested list [tokens][k])."""
    flat = [e for row in ids for e in row]
    members = [[] for _ in range(experts)]
    for a, e in enumerate(flat):
        if 0 <= e < experts:
            members[e].append(a)
    counts = [len(m) for m in members]
    offsets = [0]
    for e in range(experts):
        offsets.append(offsets[-1] + (capacity or counts[e]))
    slots, sources = [-1] * len(flat), [-1] * (experts * capacity if capacity else len(flat))
    for e in range(experts):
        for r, a in enumerate(members[e][:capacity] if capacity else members[e]):
            slots[a], sources[offsets[e] + r] = offsets[e] + r, a
    return slots, sources, counts, offsets


def rows_of(table, slots):
    """table's rows for slots [tokens, k], zeros for -1, in 64 bits."""
    keep = (slots >= 0).unsqueeze(-1)
    return torch.where(keep, table.double()[slots.clamp(min=0).long()], 0.0)


# ---------------------------------------------------------------------------- norm and rotation
def turn(x, angle, pairs):
    """x [tokens, heads, dim] with its first 2 * angle.shape[1] elements turned by angle [tokens, rot / 2]."""
    half = angle.shape[1]
    rot, c, s = 2 * half, angle.cos()[:, None], angle.sin()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :half], x[..., half:rot])
    out = x.clone()
    if pairs:
        out[..., 0:rot:2], out[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        out[..., :half], out[..., half:rot] = a * c - b * s, b * c + a * s
    return out


def other(x, half, pairs):
    """|x| with the magnitude of the other element of its pair added: what a turned element's rounding goes by."""
    x = x.abs()
    out = x.clone()
    if pairs:
        both = x[..., 0:2 * half:2] + x[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = both, both
    else:
        both = x[..., :half] + x[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = both, both
    return out


def angles(positions, inv_freq):
    """The angles [tokens, rot / 2] within a turn.  Their products have 64 bits, as far positions need: 40 of the position, 24 of the frequency."""
    a = positions.cpu().numpy().astype(np.longdouble)[:, None] * inv_freq.cpu().numpy().astype(np.longdouble)
    return torch.from_numpy(np.arctan2(np.sin(a), np.cos(a)).astype(np.float64)).to(inv_freq.device)


def norm_rope(x, w, angle, pairs, eps):
    """(output, its slack) in 64 bits.

    The sum of up to 1024 squares over the lanes of a warp adds at most 32 + 5 terms one after the other, so r is off by less than
    (37 / 2 + 3) 2^-24, z by two roundings more, sine and cosine by 2^-22: below 2^-18 of the two elements of a pair."""
    x = x.double()
    z = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    z = z if w is None else z * w.double()
    return turn(z, angle, pairs), 2.0 ** -18 * other(z, angle.shape[1], pairs)


def norm_rope_bwd(x, w, angle, pairs, eps, g):
    """(dx, its slack, dw, its slack) in 64 bits.  Slacks as for the forward; the mean of s n adds magnitudes, dw's sum those of all rows (at
    most 2^7 terms one after the other in the tests' sizes)."""
    x, g = x.double(), g.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n, e = x * r, turn(g, -angle, pairs)
    s = e if w is None else e * w.double()
    dx = r * (s - n * (s * n).mean(-1, keepdim=True))
    size = other(g, angle.shape[1], pairs)
    weighted = size if w is None else size * w.double().abs()
    slack = 2.0 ** -17 * r * (weighted + n.abs() * (weighted * n.abs()).mean(-1, keepdim=True))
    return dx, slack, (e * n).sum((0, 1)), 2.0 ** -16 * (size * n.abs()).sum((0, 1))


# ---------------------------------------------------------------------------- AdamW
def adamw(p, g, m, v, *, lr, betas, eps, weight_decay, step, grad_scale=1.0):
    """(p, its slack, m, its slack, v, its slack) after a step, in 64 bits.  Three roundings and the two of the constants in m and v (2^-22 of what
    is added); quotient and square root 2^-20 of the update."""
    p, g, m, v = p.double(), g.double() * grad_scale, m.double(), v.double()
    b1, b2 = betas
    size_m, size_v = b1 * m.abs() + (1 - b1) * g.abs(), b2 * v + (1 - b2) * g * g
    m, v = b1 * m + (1 - b1) * g, size_v
    c1, c2 = 1 - b1 ** step, 1 - b2 ** step
    denominator = torch.sqrt(v / c2) + eps
    q = p - lr * (weight_decay * p + m / c1 / denominator)
    slack = 2.0 ** -23 * p.abs() + lr * 2.0 ** -20 * (weight_decay * p.abs() + size_m / c1 / denominator)
    return q, slack, m, 2.0 ** -22 * size_m, v, 2.0 ** -22 * size_v


def noise(n, seed, tensor, start=0):
    """The 32 random bits of each element of a tensor (of n from the place `start` on, all on one side of a multiple of 2^32), as int64."""
    key = (seed + (tensor + 1) * 0x9E3779B9 + (start >> 32) * 0x9C2F1D35) & 0xFFFFFFFF
    x = (((torch.arange(n) + (start & 0xFFFFFFFF)) ^ key) * 0xA3D95FA7) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xC8B1F265) & 0xFFFFFFFF
    return x ^ (x >> 16)


def encode(x, bits16, e4m3):
    """(codes, scales) of an fp32 tensor on the host, block after block of 256."""
    top, cut, least, bias = (7, 20, 8, 7) if e4m3 else (14, 21, 16, 15)
    size = x.contiguous().view(torch.int32).long() & 0x7FFFFFFF
    codes, fields = torch.zeros_like(size), []
    for b in range(0, x.numel(), 256):
        part = size[b:b + 256]
        finite = part[part < 0x7F800000]
        field = max((int(finite.max()) >> 23 if finite.numel() else 0) - top, least)
        fields.append(field)
        moved = part + (bits16[b:b + 256] << (cut - 16)) - ((field - bias) << 23)
        code = torch.where(moved < 1 << 23, 0, moved >> cut)
        if not e4m3:
            code = torch.where((moved < 1 << 23) & (part > 0), (1 << 23) >> cut, code)
        else:
            code = torch.where(code > 0, code | torch.where(x[b:b + 256] < 0, 0x80, 0), 0)
        codes[b:b + 256] = torch.where(part >= 0x7F800000, 0x7F, code)
    scales = (torch.tensor(fields, dtype=torch.int32) << 23).view(torch.float32)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn if e4m3 else torch.float8_e5m2), scales


def decode(codes, scales):
    return codes.float() * scales.repeat_interleave(256)[:codes.numel()]


def moments32(g, m, v, betas, grad_scale=1.0):
    """m and v after a step with every product and sum rounded to fp32."""
    f = lambda x: torch.tensor(x, dtype=torch.float32)  # noqa: E731
    g = g.float() * f(grad_scale)
    return m * f(betas[0]) + g * f(1 - betas[0]), v * f(betas[1]) + (g * g) * f(1 - betas[1])
