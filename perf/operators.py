"""The operators around a verification step that the cache of keys and values asks for, and the work they are measured on.

A decoding step of a target model runs the drafted rows of every sequence (the root and N drafts, a tree or a chain) through
its layers: queries and keys are rotated by the rows' positions, keys and values are appended to a paged cache held in 8 bits,
the queries attend to it, and after verification the tokens of the accepted path are kept.  A case is one call of one of the
operators (with the touched tokens read back, where the operator changes the cache).  Inputs are synthetic, made on the GPU
from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False   # True: run() calls the library; False: run() computes the operators from elementary torch operations

F8_MAX = 448.0          # largest e4m3 value
LEAST_EXPONENT = -100   # of a block's scale
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def _rotary(name=None, *, B, R, H, D, dtype, sections, interleaved, far, inverse):
    """rotary(): rows [B, R, H, D]; sections: pairs per axis; far: positions lie in [0, far); inverse: the gradient."""
    return _named(name, kind="rotary", B=B, R=R, H=H, D=D, dtype=dtype, sections=",".join(map(str, sections)),
                  interleaved=interleaved, far=far, inverse=inverse)


def _append(name=None, *, B, R, H, D, S, dtype, held, ragged, sections, interleaved):
    """cache_append() of up to R rows a sequence behind up to `held` tokens, then cache_read() of the blocks it touched."""
    return _named(name, kind="append", B=B, R=R, H=H, D=D, S=S, dtype=dtype, held=held, ragged=ragged,
                  sections=",".join(map(str, sections)), interleaved=interleaved)


def _attention(name=None, *, B, R, H, G, D, S, dtype, held, tree, ragged, left=0):
    """cache_attention(): R rows a sequence (tree: of a draft tree of that depth; 0: causal) of G heads for each of H heads of
    the cache, over up to `held` cached tokens; left: up to so many leading tokens are padding."""
    return _named(name, kind="attention", B=B, R=R, H=H, G=G, D=D, S=S, dtype=dtype, held=held, tree=tree, ragged=ragged, left=left)


def _keep(name=None, *, B, N, H, D, S, held, depth):
    """cache_keep() of accepted paths of a tree of N drafts, then cache_read() of the blocks it touched."""
    return _named(name, kind="keep", B=B, N=N, H=H, D=D, S=S, held=held, depth=depth)


def _read(name=None, *, B, R, H, D, S, dtype, held):
    """cache_read() of R tokens a sequence."""
    return _named(name, kind="read", B=B, R=R, H=H, D=D, S=S, dtype=dtype, held=held)


def _named(name, **case):
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # queries of one draft tree of 60 nodes for one image under guidance (two sequences), row and column positions: latency
        _rotary("rotary, one tree", B=2, R=61, H=20, D=64, dtype="bf16", sections=(16, 16), interleaved=True, far=32, inverse=False),
        # the gradient of a training batch's queries with time, height and width positions, an odd number of rows
        _rotary("rotary gradient", B=8, R=1021, H=32, D=128, dtype="f32", sections=(16, 24, 24), interleaved=False, far=4096, inverse=True),
        # one new token for each of 128 sequences of a serving batch, grouped heads
        _append("append, 128 tokens", B=128, R=1, H=8, D=128, S=64, dtype="bf16", held=1024, ragged=False, sections=(32, 32), interleaved=True),
        # prompts of different lengths that fill the cache
        _append("append, 32 prompts", B=32, R=1024, H=8, D=128, S=64, dtype="bf16", held=0, ragged=True, sections=(64,), interleaved=False),
        # plain decoding of one 256-pixel image under guidance: the smallest call
        _attention("one token", B=2, R=1, H=20, G=1, D=64, S=64, dtype="bf16", held=256, tree=0, ragged=False),
        # plain decoding of a serving batch, grouped heads, contexts of all lengths
        _attention("128 tokens", B=128, R=1, H=8, G=4, D=128, S=64, dtype="bf16", held=4096, tree=0, ragged=False),
        # 128 images under guidance with a 60-node draft tree each, prompts padded on the left
        _attention("256 trees", B=256, R=61, H=20, G=1, D=64, S=64, dtype="bf16", held=1144, tree=6, ragged=False, left=120),
        # one long context, a chain of seven drafts, fp32 queries
        _attention("long chain", B=1, R=8, H=4, G=8, D=128, S=128, dtype="f32", held=100003, tree=0, ragged=False),
        # the accepted paths of one image's and of a serving batch's trees
        _keep("keep, one tree", B=2, N=60, H=20, D=64, S=64, held=256, depth=6),
        _keep("keep, 256 trees", B=256, N=60, H=20, D=64, S=64, held=1144, depth=6),
        # the last block of every sequence of a small batch, and whole contexts moved to 16 bits
        _read("read, last tokens", B=16, R=37, H=8, D=96, S=16, dtype="f32", held=500),
        _read("read, contexts", B=32, R=4000, H=8, D=128, S=64, dtype="bf16", held=4100),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def _sections(rng, pairs):
    axes = rng.choice([1, 2, 3])
    cuts = sorted(rng.randrange(1, pairs) for _ in range(axes - 1)) if pairs > axes else []
    return tuple(b - a for a, b in zip([0] + cuts, cuts + [pairs]) if b > a)


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["rotary", "append", "attention", "attention", "attention", "keep", "read"])
    S = rng.choice([16, 32, 64, 128])
    D = rng.choice([64, 128, 64, 128, 16 * rng.randrange(2, 9)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    H = rng.choice([1, 2, 4, 5, 8, 16, 20, 32])
    if kind == "rotary":
        rows = _spread(rng, 8, 60_000_000 // (H * D))
        R = rng.choice([1, 8, 61, _spread(rng, 1, 2000)])
        B = max(1, rows // R)
        pairs = D // 2 if rng.random() < 0.7 else rng.randrange(3, D // 2 + 1)
        return _rotary(B=B, R=R, H=H, D=D, dtype=dtype, sections=_sections(rng, pairs), interleaved=rng.random() < 0.5,
                       far=_spread(rng, 16, 200_000), inverse=rng.random() < 0.4)
    if kind == "append":
        rows = _spread(rng, 1, 30_000_000 // (H * D))
        R = min(rows, rng.choice([1, 8, 61, _spread(rng, 1, 4000)]))
        B = max(1, min(rows // R, 1024))
        return _append(B=B, R=R, H=H, D=D, S=S, dtype=dtype, held=_spread(rng, 1, max(1, min(2000, 200_000_000 // (B * H * D)))),
                       ragged=rng.random() < 0.5, sections=_sections(rng, D // 2), interleaved=rng.random() < 0.5)
    if kind == "attention":
        G = rng.choice([1, 1, 2, 4, 5, 8])
        tree = rng.choice([0, 0, 6])
        R = rng.choice([1, 1, 1, 8, 61, _spread(rng, 1, 700)]) if not tree else rng.choice([61, 61, _spread(rng, 2, 200)])
        codes = 250_000_000 // (H * D)                          # tokens of all sequences whose codes stay below half a gigabyte
        flops = 30_000_000_000 // (4 * R * H * G * D)           # and those whose products stay below the largest listed case's
        tokens = max(1, min(codes, flops))
        B = _spread(rng, 1, max(1, min(512, tokens // (2 * R + 16))))
        held = _spread(rng, 1, max(1, min(150_000, tokens // B - R)))
        return _attention(B=B, R=R, H=H, G=G, D=D, S=S, dtype=dtype, held=held, tree=tree, ragged=rng.random() < 0.3,
                          left=rng.choice([0, 0, held // 3]))
    if kind == "keep":
        N = rng.choice([7, 60, 60, _spread(rng, 7, 200)])
        B = _spread(rng, 1, max(1, min(512, 120_000_000 // (H * D * (N + 2 * S)))))
        return _keep(B=B, N=N, H=H, D=D, S=S, held=_spread(rng, 1, max(1, min(2000, 200_000_000 // (B * H * D)))), depth=rng.choice([3, 6]))
    tokens = _spread(rng, 16, 120_000_000 // (H * D))
    R = _spread(rng, 1, min(tokens, 8000))
    return _read(B=max(1, min(512, tokens // R)), R=R, H=H, D=D, S=S, dtype=dtype, held=R + rng.randrange(0, 200))


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _tree(B, N, depth, g):
    """Parents of B trees of N drafts: a spine of `depth` nodes, then nodes below the root or any earlier node above that depth."""
    parents = torch.empty(B, N, dtype=torch.int64)
    for b in range(B):
        deep, open_nodes = [], [-1]
        picks = torch.rand(N, generator=g).tolist()
        for i in range(N):
            p = i - 1 if i < depth else open_nodes[int(picks[i] * len(open_nodes))]
            d = 1 if p < 0 else deep[p] + 1
            deep.append(d)
            if d < depth:
                open_nodes.append(i)
            parents[b, i] = p
    return parents


def _inputs(case, seed):
    """The tensors of a case (host generator for what is small, device generator for rows and codes)."""
    c, dev = case, "cuda"
    gh = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=dev).manual_seed(seed + 1)
    B, H, D = c["B"], c["H"], c["D"]
    x = {}

    def rows(*shape):   # activations: Gaussian with a spread between heads and a few strong components
        gain = torch.exp(0.3 * torch.randn(shape[-2:], generator=gd, device=dev))
        return (torch.randn(shape, generator=gd, device=dev) * gain).to(TYPES[c.get("dtype", "bf16")])

    def rotation(R):
        sections = [int(s) for s in c["sections"].split(",")]
        pairs, far = sum(sections), c.get("far", 4096)
        if c["interleaved"]:   # each axis has a ladder of its own
            freq = torch.cat([10000.0 ** (-torch.arange(s, dtype=torch.float64) / s) for s in sections])
        else:                  # one ladder, of which each axis takes a run
            freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
        x["inv_freq"] = freq.float().to(dev)
        x["sections"] = tuple(sections)
        x["positions"] = torch.randint(0, far, (len(sections), B, R), generator=gh, dtype=torch.int32).to(dev)

    if c["kind"] == "rotary":
        x["x"] = rows(B, c["R"], H, D)
        rotation(c["R"])
        return x

    S, held = c["S"], c["held"]
    R = c["N"] + 1 if c["kind"] == "keep" else c["R"]
    if c["kind"] == "read":
        lengths = torch.full((B,), max(held, R))
        x["first"] = torch.randint(0, max(held, R) - R + 1, (B,), generator=gh, dtype=torch.int32).to(dev)
        width = -(-max(held, R) // S)
    else:
        lengths = torch.randint(held // 8, held + 1, (B,), generator=gh)
        lengths[int(torch.randint(0, B, (1,), generator=gh))] = held
        if c["kind"] == "keep":   # what is kept stays within a block, so that a pass can be repeated on its own result
            lengths = lengths // S * S + (lengths % S).clamp(max=S - 1 - c["depth"])
        width = -(-(held + R) // S)
        if c.get("ragged"):
            counts = torch.randint(0, R + 1, (B,), generator=gh)
            counts[int(torch.randint(0, B, (1,), generator=gh))] = R
            x["counts"] = counts.int().to(dev)
    if c.get("left"):
        x["starts"] = torch.minimum(torch.randint(0, c["left"] + 1, (B,), generator=gh), lengths).int().to(dev)
    x["lengths"] = lengths.int().to(dev)
    pages = B * width + 1
    x["table"] = torch.randperm(pages, generator=gh)[:B * width].view(B, width).int().to(dev)
    for name in ("k", "v"):   # codes as an append leaves them, a power of two for each block and head
        exponent = torch.randint(-9, -5, (pages, H), generator=gd, device=dev).float()
        code = torch.empty(pages, H, S, D, dtype=torch.float8_e4m3fn, device=dev)
        step = max(1, 32_000_000 // (H * S * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            code[p:p + n] = (torch.randn((n, H, S, D), generator=gd, device=dev) * 90.0).clamp_(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)
        x[name + "_code"], x[name + "_scale"] = code, torch.exp2(exponent)
    if c["kind"] == "append":
        x["k"], x["v"] = rows(B, R, H, D), rows(B, R, H, D)
        rotation(R)
        x["first"] = x["lengths"] // S * S
        x["rows"] = R + S
    elif c["kind"] == "attention":
        x["q"] = rows(B, R, H * c["G"], D)
        if c["tree"]:
            x["parents"] = _tree(B, R - 1, c["tree"], gh).int().to(dev)
    elif c["kind"] == "keep":
        N = c["N"]
        parents = _tree(B, N, c["depth"], gh)
        path = torch.full((B, N), -1, dtype=torch.int64)
        accept = torch.zeros(B, dtype=torch.int64)
        ends = torch.randint(-1, N, (B,), generator=gh).tolist()
        for b in range(B):   # the path to a node drawn at random
            nodes, i = [], ends[b]
            while i >= 0:
                nodes.append(i)
                i = int(parents[b, i])
            accept[b] = len(nodes)
            path[b, :len(nodes)] = torch.tensor(nodes[::-1], dtype=torch.int64)
        x["accept_len"], x["accept_path"] = accept.int().to(dev), path.int().to(dev)
        x["first"] = x["lengths"] // S * S
        x["rows"] = c["depth"] + 1 + S
    else:
        x["rows"] = R
    return x


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    kind, dev = case["kind"], "cuda"
    B, H, D = case["B"], case["H"], case["D"]
    if kind == "rotary":
        state["out"] = torch.empty_like(state["x"])
    elif kind == "attention":
        state["out"] = torch.zeros_like(state["q"])
    else:
        dtype = TYPES[case.get("dtype", "bf16")] if kind == "read" else torch.bfloat16
        state["out"] = tuple(torch.zeros((B, state["rows"], H, D), dtype=dtype, device=dev) for _ in range(2))
    if kind == "append":
        n = state.get("counts", case["R"])
        state["read_counts"] = (state["lengths"] - state["first"] + n).int()
    if kind == "keep":
        state["read_counts"] = state["lengths"] - state["first"] + 1 + state["accept_len"]
    if own:
        import paper_2410_03355_b200 as lt
        if kind in ("rotary", "append"):
            state["rotation"] = lt.Rotation(state["inv_freq"], state["sections"], interleaved=case["interleaved"])
        if kind != "rotary":
            state["cache"] = lt.KVCache(state["k_code"], state["v_code"], state["k_scale"], state["v_scale"])
        if kind == "attention":
            need = lt.cache_attention_workspace_bytes(B, case["R"], H * case["G"], state["cache"], state["table"].shape[1],
                                                      dtype=TYPES[case["dtype"]])
            state["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        import paper_2410_03355_b200 as lt
        if kind == "rotary":
            return lt.rotary(s["x"], s["positions"], s["rotation"], inverse=c["inverse"], out=s["out"])
        if kind == "attention":
            return lt.cache_attention(s["q"], s["cache"], s["table"], s["lengths"], counts=s.get("counts"), starts=s.get("starts"),
                                      tree_parents=s.get("parents"), out=s["out"], workspace=s["workspace"])
        if kind == "read":
            return lt.cache_read(s["cache"], s["table"], s["first"], s["rows"], out=s["out"])
        if kind == "append":
            lt.cache_append(s["k"], s["v"], s["cache"], s["table"], s["lengths"], counts=s.get("counts"),
                            positions=s["positions"], rotation=s["rotation"])
            return lt.cache_read(s["cache"], s["table"], s["first"], s["rows"], counts=s["read_counts"], out=s["out"])
        lengths = lt.cache_keep(s["cache"], s["table"], s["lengths"], s["accept_len"], s["accept_path"])
        return (lengths, *lt.cache_read(s["cache"], s["table"], s["first"], s["rows"], counts=s["read_counts"], out=s["out"]))
    if kind == "rotary":
        return _plain_rotate(s["x"], s, c["interleaved"], c["inverse"]).to(s["x"].dtype)
    if kind == "attention":
        return _plain_attention(s, c)
    if kind == "read":
        return _plain_read(s, c, TYPES[c["dtype"]])
    if kind == "append":
        _plain_append(s, c)
        return _plain_read(s, c, torch.bfloat16, s["read_counts"])
    return (_plain_keep(s, c), *_plain_read(s, c, torch.bfloat16, s["read_counts"]))


def _plain_rotate(x, s, interleaved, inverse):
    """The rotated rows in 32 bits; angles in 64."""
    pairs = s["inv_freq"].numel()
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=x.device),
                                   torch.tensor(s["sections"], device=x.device), output_size=pairs)
    angle = s["positions"].double()[axis].permute(1, 2, 0) * s["inv_freq"].double()   # [B, R, pairs]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if inverse:
        sin = -sin
    y = x.float()
    if interleaved:
        a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = y[..., :pairs], y[..., pairs:2 * pairs]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, y[..., 2 * pairs:]], dim=-1)


def _slots(s, S, first, R, counts):
    """Pages [B, R], slots [B, R] and which of the R tokens from `first` on there are."""
    token = first[:, None].long() + torch.arange(R, device=first.device)
    there = torch.arange(R, device=first.device) < (torch.full_like(first, R) if counts is None else counts)[:, None]
    block = torch.clamp(token // S, max=s["table"].shape[1] - 1)
    return torch.gather(s["table"].long(), 1, block), token % S, there


def _plain_read(s, c, dtype, counts=None):
    page, slot, there = _slots(s, c["S"], s["first"], s["rows"], counts)
    out = []
    for name in ("k", "v"):
        value = s[name + "_code"].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float() * s[name + "_scale"][page][..., None]
        out.append(torch.where(there[..., None, None], value, 0.0).to(dtype))
    return tuple(out)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, e, LEAST_EXPONENT).clamp(min=LEAST_EXPONENT).float()


def _recode(s, name, page, scale, held, S):
    """Brings the first `held` slots of each listed block to a scale at least as large as its own; blocks [n], scales [n, H]."""
    old = s[name + "_scale"][page]
    new = torch.where(held[:, None] > 0, torch.maximum(old, scale), scale)
    code = s[name + "_code"].view(torch.uint8)[page]
    value = (code.view(torch.float8_e4m3fn).float() * (old / new)[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    keep = torch.arange(S, device=page.device)[None, None, :, None] < held[:, None, None, None]
    s[name + "_code"].view(torch.uint8)[page] = torch.where(keep, value, code)
    s[name + "_scale"][page] = new
    return new


def _plain_append(s, c):
    S, R, B, H = c["S"], c["R"], c["B"], c["H"]
    page, slot, there = _slots(s, S, s["lengths"], R, s.get("counts"))
    block = s["lengths"][:, None].long() // S + torch.arange(-(-R // S) + 1, device=page.device)   # blocks that may be touched
    row = s["lengths"][:, None].long() + torch.arange(R, device=page.device)
    at = row // S - block[:, :1]
    last = s["lengths"].long() + (s["counts"].long() if "counts" in s else R) - 1
    touched = (block <= last[:, None] // S) & (last >= s["lengths"])[:, None]
    b_of, j_of = torch.nonzero(touched, as_tuple=True)
    where = s["table"].long()[b_of, block[b_of, j_of]]
    held = torch.clamp(s["lengths"].long()[b_of] - block[b_of, j_of] * S, min=0)
    for name, x in (("k", _plain_rotate(s["k"], s, c["interleaved"], False)), ("v", s["v"].float())):
        amax = torch.where(there[..., None], x.abs().amax(-1), 0.0)
        most = torch.zeros(B, block.shape[1], H, device=x.device)
        most.scatter_reduce_(1, at[..., None].expand(-1, -1, H), amax, "amax")
        new = _recode(s, name, where, torch.exp2(_exponent(most[b_of, j_of])), held, S)
        scale = torch.ones(B, block.shape[1], H, device=x.device)
        scale[b_of, j_of] = new
        code = (x / torch.gather(scale, 1, at[..., None].expand(-1, -1, H))[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        bi, ri = torch.nonzero(there, as_tuple=True)
        s[name + "_code"].view(torch.uint8)[page[bi, ri], :, slot[bi, ri]] = code[bi, ri]


def _plain_keep(s, c):
    S, N = c["S"], c["N"]
    depth = min(N, c["depth"])
    j = torch.arange(depth, device=s["table"].device)
    path = s["accept_path"][:, :depth].long()
    move = (j < s["accept_len"][:, None]) & (path != j)
    source = s["lengths"][:, None].long() + 1 + torch.where(move, path, 0)
    target = s["lengths"][:, None].long() + 1 + j
    table = s["table"].long()
    page_s, page_t = torch.gather(table, 1, source // S), torch.gather(table, 1, target // S)
    b_of, j_of = torch.nonzero(move, as_tuple=True)
    blocks = torch.stack([s["lengths"].long() + 1, s["lengths"].long() + depth], 1) // S       # blocks of the first and last target
    blocks = blocks[:, :1] + torch.arange(-(-depth // S) + 1, device=path.device)
    for name in ("k", "v"):
        scale = s[name + "_scale"]
        value = s[name + "_code"].view(torch.uint8)[page_s[b_of, j_of], :, (source % S)[b_of, j_of]].view(torch.float8_e4m3fn).float() \
            * scale[page_s[b_of, j_of]][..., None]
        most = torch.zeros(*blocks.shape, c["H"], device=path.device)
        at = (target // S - blocks[:, :1])[b_of, j_of]
        flat = most.view(-1, c["H"])
        flat.scatter_reduce_(0, (b_of * blocks.shape[1] + at)[:, None].expand(-1, c["H"]), scale[page_s[b_of, j_of]], "amax")
        bt, jt = torch.nonzero(most.amax(-1) > 0, as_tuple=True)
        _recode(s, name, table[bt, blocks[bt, jt]], most[bt, jt], torch.full_like(bt, S), S)
        code = (value / scale[page_t[b_of, j_of]][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        s[name + "_code"].view(torch.uint8)[page_t[b_of, j_of], :, (target % S)[b_of, j_of]] = code
    return s["lengths"] + 1 + s["accept_len"]


def _seen(parents, R, device):
    """[.., R, R]: which of the step's rows a row sees (itself and its ancestors; without parents the rows up to it)."""
    if parents is None:
        return torch.ones(R, R, dtype=torch.bool, device=device).tril()[None]
    B = parents.shape[0]
    up = torch.cat([torch.zeros(B, 1, dtype=torch.int64, device=device), parents.long() + 1], 1)   # row of the parent; the root's is itself
    seen = torch.eye(R, dtype=torch.bool, device=device).repeat(B, 1, 1)
    for _ in range(R.bit_length() + 1):   # rows reached by up to 1, 3, 7 ... steps up
        seen = seen | torch.gather(seen, 1, up[..., None].expand(-1, -1, R))
        up = torch.gather(up, 1, up)
    return seen


def _plain_attention(s, c):
    B, R, H, G, D, S = (c[n] for n in ("B", "R", "H", "G", "D", "S"))
    dev, out = s["q"].device, torch.zeros_like(s["q"])
    width = s["table"].shape[1]
    L = width * S
    seen = _seen(s.get("parents"), R, dev)
    step = max(1, 400_000_000 // (L * H * max(D, R * G)))
    for b0 in range(0, B, step):
        b1 = min(B, b0 + step)
        n = b1 - b0
        page = s["table"][b0:b1].long()
        k, v = ((s[name + "_code"].view(torch.uint8)[page].view(torch.float8_e4m3fn).float() * s[name + "_scale"][page][..., None, None])
                .permute(0, 2, 1, 3, 4).reshape(n, H, L, D) for name in ("k", "v"))
        q = s["q"][b0:b1].float().view(n, R, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, R * G, D)
        token = torch.arange(L, device=dev)
        length = s["lengths"][b0:b1, None].long()
        inside = token < length
        row = token - length
        drafted = torch.gather((seen if seen.shape[0] == 1 else seen[b0:b1]).expand(n, -1, -1), 2,
                               row.clamp(0, R - 1)[:, None].expand(-1, R, -1)) & ((row >= 0) & (row < R))[:, None]
        see = inside[:, None] | drafted
        if "starts" in s:
            see = see & (token >= s["starts"][b0:b1, None])[:, None]
        x = (q @ k.transpose(-1, -2)) * D ** -0.5
        x = torch.where(see[:, None, :, None].expand(-1, -1, -1, G, -1).reshape(n, 1, R * G, L), x, -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
        y = (p @ torch.where(torch.isfinite(v), v, 0.0)) / p.sum(-1, keepdim=True).clamp(min=1e-37)
        y = y.view(n, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(n, R, H * G, D).to(out.dtype)
        if "counts" in s:
            y = torch.where((torch.arange(R, device=dev) < s["counts"][b0:b1, None])[..., None, None], y, torch.zeros_like(y))
        out[b0:b1] = y
    return out


# ---- work and the definitions in 64 bits -------------------------------------------------------------------------------

def work(case):
    c, H, D, B = case, case["H"], case["D"], case["B"]
    if c["kind"] == "rotary":
        n = B * c["R"] * H * D
        return {"bytes": 2 * n * SIZE[c["dtype"]] + 4 * B * c["R"] * len(c["sections"].split(",")), "flops": 3 * n}
    if c["kind"] == "read":
        n = 2 * B * c["R"] * H * D
        return {"bytes": n * (1 + SIZE[c["dtype"]]), "flops": n}
    if c["kind"] == "append":   # rows in, codes out, codes of the touched blocks in again, their values out
        rows = B * c["R"] * (0.5 if c["ragged"] else 1.0)
        held = B * min(c["held"], c["S"]) / 2
        return {"bytes": int(2 * H * D * (rows * (SIZE[c["dtype"]] + 1) + (rows + held) * 3)), "flops": int(2 * H * D * rows * 6)}
    if c["kind"] == "keep":     # about three moved tokens a sequence; the touched blocks' codes in, their values out
        rows, held = 3 * B, B * (min(c["held"], c["S"]) / 2 + 4)
        return {"bytes": int(2 * H * D * (rows * 2 + held * 3)), "flops": int(2 * H * D * held)}
    tokens = B * (c["held"] * 9 / 16 + c["R"] * (0.5 if c["ragged"] else 1.0) - c["left"] / 2)
    rows = c["R"] * (0.5 if c["ragged"] else 1.0)
    return {"bytes": int(2 * tokens * H * D + 2 * B * rows * H * c["G"] * D * SIZE[c["dtype"]]), "flops": int(4 * tokens * rows * H * c["G"] * D)}


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["kind"] == "rotary":
        return _exact_turn(x["x"].double(), x, c["interleaved"], -1.0 if c["inverse"] else 1.0)
    if c["kind"] == "attention":
        return _exact_attention(c, x)
    if c["kind"] == "append":
        return _exact_append(c, x)
    if c["kind"] == "keep":
        return _exact_keep(c, x)
    B, R, S = c["B"], c["R"], c["S"]
    out = [torch.empty(B, R, c["H"], c["D"], dtype=torch.float64, device="cuda") for _ in range(2)]
    table, first = x["table"].tolist(), x["first"].tolist()
    for b in range(B):
        k, v = _exact_tokens(x, table[b], S, first[b], first[b] + R)
        out[0][b], out[1][b] = k, v
    return tuple(out)


def _exact_turn(y, x, interleaved, sign):
    """Each pair as a complex number times e^(i angle)."""
    out, pairs, j = y.clone(), sum(x["sections"]), 0
    for axis, count in enumerate(x["sections"]):
        run = slice(j, j + count)
        angle = sign * x["positions"][axis].double()[..., None] * x["inv_freq"][run].double()
        turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
        if interleaved:
            re, im = slice(2 * j, 2 * (j + count), 2), slice(2 * j + 1, 2 * (j + count) + 1, 2)
        else:
            re, im = run, slice(pairs + j, pairs + j + count)
        z = torch.complex(y[..., re], y[..., im]) * turn
        out[..., re], out[..., im] = z.real, z.imag
        j += count
    return out


def _exact_tokens(x, table, S, first, end):
    """Keys and values [end - first, H, D] of a sequence's tokens in 64 bits."""
    blocks = torch.tensor(table[first // S:-(-end // S)], device="cuda")
    out = []
    for name in ("k", "v"):
        value = x[name + "_code"].view(torch.uint8)[blocks].view(torch.float8_e4m3fn).double() * x[name + "_scale"][blocks].double()[..., None, None]
        value = value.transpose(1, 2).flatten(0, 1)
        out.append(value[first % S:first % S + end - first])
    return out


def _exact_e4m3(value, scale):
    """value held in e4m3 with that scale: three bits behind the leading one, spacing 2^-9 below 2^-6, ties to even."""
    y = value / scale
    _, e = torch.frexp(y)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(y / step) * step * scale


def _exact_scale(amax):
    e = torch.full_like(amax, float(LEAST_EXPONENT))
    some = amax > 0
    e[some] = torch.ceil(torch.log2(amax[some] / F8_MAX)).clamp(min=LEAST_EXPONENT)
    e = torch.where(some & (amax > F8_MAX * torch.exp2(e)), e + 1, e)
    lower = some & (e > LEAST_EXPONENT) & (amax <= F8_MAX * torch.exp2(e - 1))
    return torch.exp2(torch.where(lower, e - 1, e))


def _exact_append(c, x):
    B, R, S, H, D = (c[n] for n in ("B", "R", "S", "H", "D"))
    out = [torch.zeros(B, x["rows"], H, D, dtype=torch.float64, device="cuda") for _ in range(2)]
    lengths, table = x["lengths"].tolist(), x["table"].tolist()
    counts = x["counts"].tolist() if "counts" in x else [R] * B
    if B * (R // S + 2) > 6000:
        return None
    new = (_exact_turn(x["k"].double(), x, c["interleaved"], 1.0), x["v"].double())
    for b in range(B):
        n, length = counts[b], lengths[b]
        first = length // S * S
        for which, name in enumerate(("k", "v")):
            if length > first:
                out[which][b, :length - first] = _exact_tokens(x, table[b], S, first, length)[which]
            for block in range(first, length + n, S):
                low, high = max(block, length), min(block + S, length + n)
                if low >= high:
                    continue
                fresh = new[which][b, low - length:high - length]
                scale = _exact_scale(fresh.abs().amax((0, 2)))
                if low > block:
                    scale = torch.maximum(scale, x[name + "_scale"][table[b][block // S]].double())
                    old = out[which][b, block - first:low - first]
                    out[which][b, block - first:low - first] = _exact_e4m3(old, scale[:, None])
                out[which][b, low - first:high - first] = _exact_e4m3(fresh, scale[:, None])
    for which, name in enumerate(("k", "v")):   # (without new rows the block that is read stays as it is)
        for b in range(B):
            if counts[b] == 0 and lengths[b] % S:
                first = lengths[b] // S * S
                out[which][b, :lengths[b] - first] = _exact_tokens(x, table[b], S, first, lengths[b])[which]
    return tuple(out)


def _exact_keep(c, x):
    B, N, S, H, D = (c[n] for n in ("B", "N", "S", "H", "D"))
    out = [torch.zeros(B, x["rows"], H, D, dtype=torch.float64, device="cuda") for _ in range(2)]
    lengths, table = x["lengths"].tolist(), x["table"].tolist()
    accept, paths = x["accept_len"].tolist(), x["accept_path"].tolist()
    for b in range(B):
        length, n = lengths[b], accept[b]
        first = length // S * S
        everything = _exact_tokens(x, table[b], S, first, length + 1 + N)
        for which, name in enumerate(("k", "v")):
            value = everything[which]
            kept = value[:length + 1 + n - first].clone()
            scale = {}
            for j in range(n):
                if paths[b][j] != j:
                    kept[length + 1 + j - first] = value[length + 1 + paths[b][j] - first]
                    block, source = (length + 1 + j) // S, (length + 1 + paths[b][j]) // S
                    mine = scale.get(block, x[name + "_scale"][table[b][block]].double())
                    scale[block] = torch.maximum(mine, x[name + "_scale"][table[b][source]].double())
            for block, s in scale.items():
                low, high = max(block * S - first, 0), min((block + 1) * S - first, kept.shape[0])
                kept[low:high] = _exact_e4m3(kept[low:high], s[:, None])
            out[which][b, :kept.shape[0]] = kept
    return (None, *out)


def _exact_attention(c, x):
    B, R, H, G, D, S = (c[n] for n in ("B", "R", "H", "G", "D", "S"))
    out = torch.zeros(B, R, H * G, D, dtype=torch.float64, device="cuda")
    lengths, table = x["lengths"].tolist(), x["table"].tolist()
    counts = x["counts"].tolist() if "counts" in x else [R] * B
    starts = x["starts"].tolist() if "starts" in x else [0] * B
    parents = x["parents"].tolist() if "parents" in x else None
    for b in range(B):
        n, length = counts[b], lengths[b]
        if n == 0:
            continue
        k, v = _exact_tokens(x, table[b], S, 0, length + n)
        hidden = torch.zeros(n, length + n, dtype=torch.bool)
        hidden[:, length:] = True
        for r in range(n):
            if parents is None:
                hidden[r, length:length + r + 1] = False
                continue
            at = r
            while True:
                hidden[r, length + at] = False
                if at == 0:
                    break
                at = parents[b][at - 1] + 1
        hidden[:, :starts[b]] = True
        hidden = hidden.cuda()
        for h in range(H):
            q = x["q"][b, :n, h * G:(h + 1) * G].double()
            score = torch.einsum("rgd,td->grt", q, k[:, h]) / math.sqrt(D)
            score = score.masked_fill(hidden, -math.inf)
            p = torch.softmax(score, -1).nan_to_num(0.0)   # (a row that sees nothing)
            out[b, :n, h * G:(h + 1) * G] = torch.einsum("grt,td->rgd", p, v[:, h])
    return out
