"""The cache operators in 64 bits on the host, written from their definitions in include/lantern.h; plain loops over sequences."""
import math

import torch

F64 = torch.float64
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # largest relative error of rounding to a type
NAN_CODE = 0x7F


def decode(code):
    return code.view(torch.float8_e4m3fn).to(F64)


def e4m3(y):
    """The nearest e4m3 value (ties to even, no value above 448 comes in; NaN stays)."""
    _, e = torch.frexp(torch.where(torch.isfinite(y), y, torch.zeros_like(y)))
    step = torch.exp2((e - 4).clamp(min=-9).to(F64))
    return torch.round(y / step) * step


def scale_for(amax):
    """Least power of two 2^e, e >= -100, with amax <= 448 * 2^e."""
    e = -100
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """Values (not codes) of a paged cache, with its scales."""

    def __init__(self, k, v, k_scale, v_scale):
        self.code = [decode(k.cpu()), decode(v.cpu())]
        self.scale = [k_scale.cpu().to(F64), v_scale.cpu().to(F64)]
        self.S = k.shape[2]

    def tokens(self, which, table, first, end):
        """[end - first, heads, D]"""
        out = [self.code[which][table[i // self.S], :, i % self.S] * self.scale[which][table[i // self.S]][:, None] for i in range(first, end)]
        return torch.stack(out) if out else torch.zeros((0,) + tuple(self.code[0].shape[1::2]), dtype=F64)

    def recode(self, which, page, head, scale, held):
        old = self.scale[which][page, head].item()
        self.code[which][page, head, :held] = e4m3(self.code[which][page, head, :held] * (old / scale))
        self.scale[which][page, head] = scale

    def append(self, which, rows, table, length):
        """rows [n, heads, D] float64 (what is not finite is stored as NaN)."""
        n = rows.shape[0]
        rows = torch.where(torch.isfinite(rows), rows, torch.full_like(rows, math.nan))
        for block in range(length // self.S, -(-(length + n) // self.S) if n else 0):
            low, high = max(length, block * self.S), min(length + n, (block + 1) * self.S)
            if low >= high:
                continue
            page, held = table[block], low - block * self.S
            for head in range(rows.shape[1]):
                new = rows[low - length:high - length, head]
                scale = scale_for(new[~new.isnan()].abs().max().item() if (~new.isnan()).any() else 0.0)
                if held:
                    scale = max(scale, self.scale[which][page, head].item())
                    self.recode(which, page, head, scale, held)
                self.scale[which][page, head] = scale
                self.code[which][page, head, held:held + high - low] = e4m3(new / scale)

    def keep(self, table, length, path):
        """Token length + 1 + j becomes what token length + 1 + path[j] was."""
        for which in range(2):
            code, scale = self.code[which].clone(), self.scale[which].clone()
            moves = {}
            for j, at in enumerate(path):
                if at != j:
                    moves.setdefault((length + 1 + j) // self.S, []).append((length + 1 + j, length + 1 + at))
            for block, pairs in moves.items():
                page = table[block]
                for head in range(code.shape[1]):
                    mine = max([scale[page, head].item()] + [scale[table[source // self.S], head].item() for _, source in pairs])
                    if mine != scale[page, head].item():
                        self.recode(which, page, head, mine, self.S)
                    for to, source in pairs:
                        other = table[source // self.S]
                        self.code[which][page, head, to % self.S] = e4m3(code[other, head, source % self.S] * (scale[other, head].item() / mine))


def rotate(x, positions, inv_freq, sections, interleaved, inverse=False):
    """x [B, R, H, D] -> (rotated, sum of the magnitudes that went into each component), float64."""
    x = x.to(F64)
    y, mag = x.clone(), x.abs()
    pairs, j = sum(sections), 0
    for axis, count in enumerate(sections):
        for _ in range(count):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
            phi = positions[axis].to(F64) * float(inv_freq[j].to(F64))
            c, s = torch.cos(phi)[..., None], torch.sin(phi)[..., None] * (-1.0 if inverse else 1.0)
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
            mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
            j += 1
    return y, mag


def seen_rows(parents, r):
    """Rows of the step that row r sees."""
    if parents is None:
        return list(range(r + 1))
    out = [r]
    while r > 0:
        r = parents[r - 1] + 1
        out.append(r)
    return sorted(out)


def attention(q, cache, table, lengths, counts=None, starts=None, parents=None, scale=None):
    """q [B, R, HQ, D] -> (out, bound): float64 outputs (zeros for rows that see nothing; rows that counts leaves out are NaN) and, for
    each, what the error may be by arithmetic, without the rounding of the output."""
    B, R, HQ, D = q.shape
    H = cache.code[0].shape[1]
    G = HQ // H
    f32 = q.dtype == torch.float32
    scale = D ** -0.5 if scale is None else scale
    out = torch.full(q.shape, math.nan, dtype=F64)
    bound = torch.zeros(q.shape, dtype=F64)
    q = q.to(F64)
    for b in range(B):
        n = R if counts is None else counts[b]
        k, v = (cache.tokens(i, table[b], 0, lengths[b] + n) for i in range(2))
        vmax = cache.scale[1][table[b]].max().item() * 448.0 if len(table[b]) else 0.0
        for r in range(n):
            see = list(range(lengths[b])) + [lengths[b] + j for j in seen_rows(None if parents is None else parents[b], r)]
            see = [c for c in see if c >= (0 if starts is None else starts[b])]
            if not see:
                out[b, r] = 0.0
                continue
            for h in range(H):
                for g in range(h * G, (h + 1) * G):
                    x = scale * (k[see, h] @ q[b, r, g])
                    size = abs(scale) * (k[see, h].abs() @ q[b, r, g].abs())
                    p = torch.softmax(x, 0)
                    out[b, r, g] = p @ v[see, h]
                    # Scores: D products summed in fp32, whose every addition may drop up to a unit of the last place (2^-23) of the
                    # running sum of magnitudes; queries to 2^-17 (of the largest, as halves with a common exponent: far less) or, in
                    # fp32, 2^-22; three roundings more and those of the base-2 argument.  Numerators: exp2 2^-22, the sum of n of them
                    # 2^-24 each; as a half 2^-11 (as two 2^-22) and, below the smallest normal half 2^-14, 2^-25 of the largest value:
                    # halves there are 2^-24 apart.  What the first of two halves leaves of a numerator p < 1 is at most 2^-12, mostly below
                    # 2^-14 and so rounded by up to 2^-25 in the second, too: the term is the same for both types.
                    score = size.max().item() * ((D + 8) * 2.0 ** -23 + 2.0 ** -21)
                    rel = 2.0 * score + 2.0 ** -21 + len(see) * 2.0 ** -23 + (2.0 ** -21 if f32 else 2.0 ** -11)
                    bound[b, r, g] = rel * (p @ v[see, h].abs()) + rel * out[b, r, g].abs() + len(see) * 2.0 ** -25 * vmax
    return out, bound
