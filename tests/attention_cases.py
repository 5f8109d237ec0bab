"""Attention to the paged cache in 64 bits with a bound that follows the kernels' arithmetic term by term, and the calls that between them reach every
kernel that cache_attention() chooses from, undivided and in parts."""
import math

import torch

F64 = torch.float64


def tokens(code, scale, row, S, first, end):
    """Codes and scales of tokens [first, end) of a sequence with block table `row`: [n, heads, D], [n, heads]."""
    at = torch.arange(first, end)
    page, slot = torch.as_tensor(row, dtype=torch.long)[at // S], at % S
    return code[page, :, slot], scale[page]


def seen(parents, n, length, start):
    """[n, length + n]: which tokens row r of n sees."""
    own = torch.zeros(n, n, dtype=torch.bool)
    for r in range(n):
        own[r, r] = True
        if parents is None:
            own[r, :r] = True
        elif r:
            own[r] |= own[int(parents[r - 1]) + 1]   # (a parent has a smaller row)
    out = torch.cat([torch.ones(n, length, dtype=torch.bool), own], 1)
    out[:, :max(start, 0)] = False
    return out


def attention(q, cache, table, lengths, counts=None, starts=None, parents=None, scale=None):
    """q [B, R, HQ, D] on the host -> (out, bound): 64-bit outputs (zeros for rows that see nothing, NaN for rows that `counts` leaves out), and what a
    kernel's output may be off before it is rounded to its type:

    * Scores (natural logarithm).  D products are added in 32 bits, each addition off by a unit (2^-23) of the magnitudes added so far; a query component is
      off by 2^-22 of itself and 2^-39 of the row's largest; factors and the base-2 argument by a few times 2^-24 of the score, the argument's rounding by
      2^-24 of the score and of the row's largest.
    * Numerators.  exp2 to 2^-22; rounded once as a half, 2^-11 (bf16), or as two, 2^-22 (fp32), after a product with the value's scale (2^-23).  They are
      lifted by 2^10, so that what lies below the smallest normal half loses 2^-25 * 2^-10 of the row's largest numerator, as a factor of a code under the largest
      value scale that the row's blocks have.
    * Values become halves times 2^7 over the largest scale: off by 2^-25 * 2^-7 of it (2 where a scale's own digits are put with the numerators), and with bf16,
      where a scale is no power of two, by 2^-11 of themselves.  The factor is a half itself, whose least is 2^-24: a block whose scale is below 2^-31 of the largest
      (2^-30 where digits are put with the numerators) may be lost.
    * Sums.  The output adds up a product for each token whose value is not zero, one or two terms each, every addition off by 2^-23 of the magnitudes;
      accumulators and sums are scaled at most once per 32 tokens (2^-24); a sum takes at most a 32nd of its tokens one after the other, and what is put together
      of threads, warps and parts is below 64 additions more.
    """
    B, R, HQ, D = q.shape
    code = [t.cpu().view(torch.float8_e4m3fn).to(F64) for t in (cache.k, cache.v)]
    scales = [t.cpu().to(F64) for t in (cache.k_scale, cache.v_scale)]
    S, H = cache.page_tokens, cache.heads
    G = HQ // H
    f32 = q.dtype == torch.float32
    exact = bool((torch.frexp(scales[1])[0] == 0.5).all())
    terms, half = (2, 2.0 ** -22) if f32 else (1, 2.0 ** -11)
    scale = D ** -0.5 if scale is None else scale
    out = torch.full(q.shape, math.nan, dtype=F64)
    bound = torch.zeros(q.shape, dtype=F64)
    q = q.to(F64)
    for b in range(B):
        n = R if counts is None else counts[b]
        start = 0 if starts is None else max(starts[b], 0)
        if n == 0:
            continue
        if lengths[b] + n <= start:
            out[b, :n] = 0.0
            continue
        (kc, ks), (vc, vs) = (tokens(code[i], scales[i], table[b], S, start, lengths[b] + n) for i in range(2))
        see = seen(None if parents is None else parents[b], n, lengths[b], start)[:, start:]
        for h in range(H):
            k, v, vcode = kc[:, h].nan_to_num(0.0) * ks[:, h, None], vc[:, h].nan_to_num(0.0) * vs[:, h, None], vc[:, h].nan_to_num(0.0).abs()
            heads = slice(h * G, (h + 1) * G)
            x = q[b, :n, heads].reshape(n * G, D)
            mask = see[:, None].expand(n, G, see.shape[1]).reshape(n * G, -1)
            score = scale * (x @ k.T)
            size = abs(scale) * (x.abs() @ k.abs().T)
            most = torch.where(mask, size, 0.0).amax(1, keepdim=True)
            floor = abs(scale) * x.abs().amax(1, keepdim=True) * 2.0 ** -38 * k.abs().sum(1)[None]
            delta = size * ((D + 8) * 2.0 ** -23 + 2.0 ** -21) + most * 2.0 ** -23 + floor
            score = score.masked_fill(~mask, -math.inf)
            top = score.amax(1, keepdim=True).clamp(min=-1e300)
            p = torch.exp(score - top)
            total = p.sum(1, keepdim=True)
            p = p / total.clamp(min=1e-300)
            o = p @ v
            eps = torch.expm1(delta) + 2.0 ** -21
            count = mask.double().sum(1, keepdim=True)
            nonzero = mask.double() @ (v != 0).double()
            mag = p @ v.abs()
            err = (p * eps) @ v.abs() + (p * eps).sum(1, keepdim=True) * o.abs()
            err += (half + 2.0 ** -22 + (0.0 if f32 or exact else 2.0 ** -11)) * mag
            err += 2.0 ** -35 * vs[:, h].max() / total.clamp(min=1.0) * (mask.double() @ vcode)
            err += 2.0 ** -31 * vs[:, h].max() + p @ (v.abs() * (vs[:, h, None] < 2.0 ** -30 * vs[:, h].max()))
            err += (2 * terms * nonzero + count / 32 + 64) * 2.0 ** -23 * mag
            err += (count / 16 + 64) * 2.0 ** -24 * o.abs()
            out[b, :n, heads] = o.view(n, G, D)
            bound[b, :n, heads] = 1.01 * err.view(n, G, D)
    return out, bound


# ---- which kernel a call is given to ------------------------------------------------------------------------------------

def path_of(dtype, B, R, H, G, D, S, width, workspace_bytes):
    """(kernel, rows of a unit, components, type, divided), as the call chooses: by rows, type and the room that the table has; `workspace_bytes` says
    whether units are divided into parts."""
    rows, room, DP = R * G, width * S, 64 if D <= 64 else 128
    unit = 8 if rows <= 8 else 16 if rows <= 16 else 64 if rows <= 64 else 128
    kernel = "few" if rows <= 16 else "mid" if rows <= 64 and dtype == "bf16" and room < (2048 if DP == 64 else 1024) else "wide"
    return kernel, unit, DP, dtype, workspace_bytes > 0


def _case(lengths, R, H, G, D, S, dtype, room, **more):
    return dict(lengths=lengths, R=R, H=H, G=G, D=D, S=S, dtype=dtype, room=room, **more)


def _cases():
    out = []
    for dtype in ("bf16", "f32"):
        # up to 8 and up to 16 rows of a head; whole, in parts, and with room for parts that short contexts do not need
        for D, S in ((64, 64), (48, 16), (128, 128), (112, 32)):
            out += [_case([0, 1, 63, 300], 1, 2, 4, D, S, dtype, 384, starts=[0, 0, 60, 31]),
                    _case([900, 3, 2500], 7, 2, 1, D, S, dtype, 2560, tree=3, counts=[7, 7, 5]),
                    _case([0, 17, 400], 5, 1, 3, D, S, dtype, 512, counts=[5, 0, 4]),
                    _case([1300, 40, 0], 13, 2, 1, D, S, dtype, 4096, tree=4, starts=[700, 41, 0])]
        # 17 to 64 rows, short contexts and long ones
        for D, S, G, R, tree in ((64, 64, 1, 61, 6), (32, 16, 3, 20, 0), (128, 64, 1, 61, 6), (96, 32, 2, 31, 3)):
            out += [_case([0, 40, 131], R, 1, G, D, S, dtype, 256, tree=tree, starts=[0, 39, 5]),
                    _case([700, 250, 3], R, 2, G, D, S, dtype, 896, tree=tree, counts=[R, R - 3, 1]),
                    _case([2500, 100, 0], R, 1, G, D, S, dtype, 2688, tree=tree, starts=[1, 200, 0]),
                    _case([90, 7] * 20 + [0], R, 8, G, D, S, dtype, 2048, tree=tree)]   # as many units as places for CTAs
        # more than 64 rows
        for D, S, G, R, tree in ((64, 64, 2, 61, 6), (80, 16, 1, 150, 0), (128, 128, 5, 33, 4), (16, 32, 1, 70, 0)):
            out += [_case([0, 40, 131], R, 1, G, D, S, dtype, 384, tree=tree, starts=[0, 39, 5]),
                    _case([1500, 250, 3], R, 1, G, D, S, dtype, 2048, tree=tree, counts=[R, R - 3, 1])]
    return out


CASES = _cases()


def name_of(c):
    more = "".join(f"-{k}" for k in ("tree", "counts", "starts") if c.get(k))
    return f"{c['dtype']}-R{c['R']}-H{c['H']}x{c['G']}-D{c['D']}-S{c['S']}-room{c['room']}-{max(c['lengths'])}{more}"
