"""Performance cases of a paged cache that is held in 8 bits, and of rotary positions with several axes.

A translated context is kept in pages of 8-bit floats (1 sign, 4 exponent, 3 mantissa bits) with a scale for
each page, key/value head and K or V, a power of two: half the bytes that a decoding step reads, and room for
twice the contexts. New keys and values are rotated and rounded into the pages, attention reads them there, and
whole contexts move between pages and contiguous caches of the translation. Where a prompt holds images or
video, a row's rotation goes by several positions (time, height, width).

A page's scale is 2^e with the least e in -60 .. 60 that brings its largest value to 448 or below; where new
rows join old ones in a page, the scale never falls, and where it rises the old values are rounded again.

``run`` computes the plain form with elementary torch operations in 32 bits (angles in 64); with ``own`` set it
makes the library's calls. ``exact`` restates each operator in 64 bits. The pools are float8 tensors, the values
in units of their scales, which are outputs too.
"""
import math

import torch

own = False
DEV = "cuda"

# Query heads, key/value heads, head width and layers of the targets.
MODELS = {"opt125m": (12, 12, 64, 12), "qwen05": (14, 2, 64, 24), "qwen15": (12, 2, 128, 28),
          "qwen7": (28, 4, 128, 28)}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
F8 = torch.float8_e4m3fn
BASE, EPS = 1e6, 1e-6
AXES = 3


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(values):
    return ",".join(map(str, values))


def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly spread over their logarithm, in a mixed order."""
    at = [(i * 7919) % n / max(1, n - 1) for i in range(n)]
    return [int(round(lo * (hi / lo) ** x)) for x in at]


def listed():
    return [
        # ---- attention over 8-bit pages: lens are the positions with the new ones, chunks the new ones
        # The smallest: one token of one conversation, a short prompt behind it.
        dict(name="attn8_decode_one", kind="attn", model="qwen15", lens="517", chunks="1", page=16, dtype="bf16"),
        # One token for each of 64 conversations of very different lengths.
        dict(name="attn8_decode_64", kind="attn", model="qwen7", lens=_text(_spread(64, 100, 16384)),
             chunks=_text([1] * 64), page=64, dtype="bf16"),
        # One token for each of two very long contexts: few rows, the length is the work.
        dict(name="attn8_decode_long", kind="attn", model="qwen7", lens="131072,70001", chunks="1,1", page=128, dtype="bf16"),
        # Prompts of several sizes on translated contexts, conversations that decode among them.
        dict(name="attn8_prompts_mixed", kind="attn", model="opt125m", lens="1087,2050,513,777,64,1500",
             chunks="63,1024,1,130,64,7", page=32, dtype="bf16"),
        # The largest: a piece of 4,096 tokens of a long document on top of what is there.
        dict(name="attn8_chunk_long", kind="attn", model="qwen7", lens="32768", chunks="4096", page=64, dtype="bf16"),
        # ---- append to 8-bit pages
        # One new token for each of eight conversations, most of them in a page that has rows already.
        dict(name="append8_decode", kind="append", model="qwen15", lens="90001,517,1024,4001,333,16,12345,70", chunks=_text([1] * 8),
             page=16, rot="half", norm=False, axes="", dtype="bf16", bits=8),
        # Prompts of four conversations, keys and queries normed and rotated.
        dict(name="append8_prompts", kind="append", model="qwen7", lens="32768,2111,9000,4097", chunks="4096,2111,1999,2048",
             page=64, rot="half", norm=True, axes="", dtype="bf16", bits=8),
        # ---- a context is kept in 8-bit pages, and given back as a contiguous cache
        # A short context of the smallest target.
        dict(name="keep8_short", kind="keep", model="opt125m", lens="301", page=16, dtype="bf16"),
        # Three translated contexts of different lengths.
        dict(name="keep8_contexts", kind="keep", model="qwen7", lens="8191,4001,10240", page=64, dtype="bf16"),
        # ---- append with several axes: an image's rows share a time and have heights and widths
        # One token of text behind images.
        dict(name="axes_one", kind="append", model="qwen15", lens="9001", chunks="1", page=16, rot="half", norm=False,
             axes="sections", dtype="bf16", bits=16),
        # Prompts with images and text.
        dict(name="axes_prompts", kind="append", model="qwen7", lens="4096,2111,9000,4097", chunks="4096,2111,1999,2048",
             page=64, rot="half", norm=True, axes="turns", dtype="bf16", bits=16),
        # The same kind of prompt in the parity-precision type, each axis with frequencies of its own.
        dict(name="axes_fp32", kind="append", model="opt125m", lens="2048,700", chunks="1500,700", page=32, rot="pairs", norm=False,
             axes="own", dtype="fp32", bits=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "chunk", "chunk", "mixed", "append", "append", "keep", "axes", "axes"))
    model, page = rng.choice(sorted(MODELS)), rng.choice((16, 32, 64, 128))
    c = dict(kind="attn", model=model, page=page, dtype="bf16")
    if kind == "decode":
        n = _log(rng, 1, 128)
        lens = [_log(rng, 16, max(64, min(131072, 400000 // n))) for _ in range(n)]
        m = rng.choice((1, 1, 1, 2, 4))
        return dict(c, lens=_text(lens), chunks=_text([min(m, x) for x in lens]))
    if kind in ("chunk", "mixed"):
        n = rng.choice((1, 1, 2, 3, 5, 8))
        new = [_log(rng, 2, 3000 // n) for _ in range(n)]
        if kind == "mixed":
            new = [1 if rng.random() < 0.5 else x for x in new]
        lens = [x + (_log(rng, 1, 24000 // n) if rng.random() < 0.8 else 0) for x in new]
        return dict(c, lens=_text(lens), chunks=_text(new))
    if kind == "keep":
        return dict(c, kind="keep", lens=_text([_log(rng, 16, 8000) for _ in range(rng.choice((1, 2, 4)))]))
    n = _log(rng, 1, 64)
    new = [rng.choice((1, _log(rng, 1, max(2, 8000 // n)))) for _ in range(n)]
    lens = [x + _log(rng, 1, 100000 // n) for x in new]
    c = dict(c, kind="append", lens=_text(lens), chunks=_text(new), norm=rng.random() < 0.5)
    if kind == "append":
        return dict(c, rot=rng.choice(("half", "half", "pairs", "none")), axes="", bits=8)
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    bits = 32 if dtype == "fp32" else rng.choice((16, 8))
    return dict(c, rot=rng.choice(("half", "half", "pairs")), axes=rng.choice(("sections", "turns", "own")), dtype=dtype, bits=bits)


# ---------------------------------------------------------------- inputs

def _page_counts(case):
    return [-(-n // case["page"]) for n in _ints(case["lens"])]


def _bits(case):
    return case.get("bits", 8)


def _pool(case, gen, layers, pages):
    """Values of a pool, [layers][pages][heads][page][width]: normal draws with per-channel scales; 8 bits with
    their scales [layers][pages][heads]."""
    _, H, d, _ = MODELS[case["model"]]
    s = torch.exp(0.5 * torch.randn((H, 1, d), generator=gen, device=DEV))
    x = torch.empty((layers, pages, H, case["page"], d), dtype=F8 if _bits(case) == 8 else TYPES[case["dtype"]], device=DEV)
    scale = torch.ones((layers, pages, H), device=DEV) if _bits(case) == 8 else None
    for l in range(layers):
        y = torch.randn(x[l].shape, generator=gen, device=DEV) * s
        if scale is not None:
            scale[l] = torch.exp2(torch.ceil(torch.log2(y.abs().amax((2, 3)) / 448)))
            y /= scale[l][:, :, None, None]
        x[l] = y.to(x.dtype)
    return x, scale


def _normal(gen, case, *shape):
    return torch.randn(shape, generator=gen, device=DEV).to(TYPES[case["dtype"]])


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _axes(case):
    """Each pair's axis and its turn in radians a position: runs of pairs for time, height and width
    ("sections"; "own": with a run's own frequencies), or the axes in turn ("turns")."""
    half = MODELS[case["model"]][2] // 2
    cut = [half // 4, half // 4 + half * 3 // 8, half]
    rate = [BASE ** (-i / half) for i in range(half)]
    axis = [i % AXES if case["axes"] == "turns" else sum(i >= c for c in cut) for i in range(half)]
    if case["axes"] == "own":
        start = [0] + cut
        rate = [BASE ** (-(i - start[a]) / (cut[a] - start[a])) for i, a in enumerate(axis)]
    return axis, rate


def _positions(lens, chunks):
    """[axes][rows]: pieces of text and images in turn; text moves all axes, an image's rows have its time and
    their places in a grid 24 wide."""
    out = []
    for n, m in zip(lens, chunks):
        row, at, t = [], 0, n - m
        while len(row) < m:
            text = min(17, m - len(row))
            row += [(t + i, t + i, t + i) for i in range(text)]
            t += text
            image = min(24 * 18, m - len(row))
            row += [(t, t + i // 24, t + i % 24) for i in range(image)]
            t += 24
        out += row[:m]
    return [list(x) for x in zip(*out)]


_handles = {}


def _handle(case, layers, pages, slots, width):
    """The program's handle for caches of one form, made once and kept."""
    import paper_2607_28979_gb300.mot as M
    Hq, H, d, _ = MODELS[case["model"]]
    rot, axes, bits = case.get("rot", "none"), case.get("axes", ""), _bits(case)
    key = (Hq, H, d, layers, pages, slots, width, case["page"], case["dtype"], rot, axes, bits)
    if key not in _handles:
        cfg = M.make_paged_config(layers, Hq, H, d, case["page"], pages, slots, width, rot_dim=0 if rot == "none" else d,
                                  rot_pairs=rot == "pairs", rot_base=BASE, norm_eps=EPS, dtype=case["dtype"])
        _handles[key] = M.mot_create_paged8(cfg) if bits == 8 else M.mot_create_paged(cfg)
        if axes:
            axis, rate = _axes(case)
            M.mot_paged_set_axes(_handles[key], AXES, axis, rate if axes == "own" else None)
    return _handles[key]


def prepare(case, seed):
    Hq, H, d, L = MODELS[case["model"]]
    lens, need, kind = _ints(case["lens"]), _page_counts(case), case["kind"]
    n = len(lens)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    layers, width = L if kind == "keep" else 1, max(need)
    pages = sum(need) + max(4, sum(need) // 8)   # an eighth more: what serving pools keep free
    s = dict(case=case, kind=kind, n=n, width=width, pages=pages)
    s["k"], s["ks"] = _pool(case, gen, layers, pages)
    s["v"], s["vs"] = _pool(case, gen, layers, pages)
    s["table"] = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    s["lens"] = _i32(lens)
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    # pages lie as a pool in use has them: in no order, among free ones
    perm = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    at = 0
    for i, m in enumerate(need):
        s["table"][i, :m] = perm[at:at + m]
        at += m
    s["refs"][perm[:at].long()] = 1
    s["seqs"] = _i32(range(n))
    if kind == "keep":   # a context as the translation leaves it, and room for it where it is wanted again
        s["new"] = [_normal(gen, case, L, n, H, max(lens), d) for _ in range(2)]
        s["back"] = [torch.zeros_like(x) for x in s["new"]]
    else:
        chunks = _ints(case["chunks"])
        starts = [sum(chunks[:i]) for i in range(n + 1)]
        s.update(starts=_i32(starts), rows=starts[-1], chunk=max(chunks))
        if kind == "attn":
            s["q"] = _normal(gen, case, starts[-1], Hq, d)
        else:   # the columns of a fused projection's output
            s["qkv"] = _normal(gen, case, starts[-1], Hq + 2 * H, d)
            s["w"] = [(1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(TYPES[case["dtype"]])
                      for _ in range(2)] if case["norm"] else [None, None]
            if case["axes"]:
                s["at"] = _i32(_positions(lens, chunks)) + int(seed) % 1000
                axis, rate = _axes(case)
                s["axis"], s["rate"] = torch.tensor(axis, device=DEV), torch.tensor(rate, dtype=torch.float64, device=DEV)
        s["out"] = torch.zeros((starts[-1], Hq, d), dtype=TYPES[case["dtype"]], device=DEV)
    if own:   # the handle that a program of this form keeps
        import paper_2607_28979_gb300.mot as M
        s["h"] = _handle(case, layers, pages, n, width)
        scales = [s["ks"], s["vs"]] if _bits(case) == 8 else []
        s["cache"] = M.paged_cache(s["k"], s["v"], s["table"], s["lens"], s["refs"], *scales)
    return s


# ---------------------------------------------------------------- plain forms

def _new_rows(s):
    """Row index [n][chunk], whether there is such a row, and its position in the sequence."""
    seqs = s["seqs"].long()
    starts = s["starts"].long()
    m = starts[1:] - starts[:-1]
    r = torch.arange(s["chunk"], device=DEV)
    return (starts[:-1, None] + r).clamp_max(s["rows"] - 1), r < m[:, None], s["lens"][seqs].long()[:, None] - m[:, None] + r


def _values(x, scale, pages):
    """The pages' values in 32 bits, [..][heads][page][width]."""
    return x.view(torch.uint8)[pages].view(F8).float() * scale[pages][..., None, None]


def _plain_attention(s):
    k, v, q = s["k"][0], s["v"][0], s["q"]
    H, P, d = k.shape[1:]
    n, Hq = s["n"], q.shape[1]
    seqs = s["seqs"].long()
    at = s["table"][seqs].long().clamp_min(0)
    idx, there, pos = _new_rows(s)
    N, m, G = at.shape[1] * P, idx.shape[1], Hq // H
    K = _values(k, s["ks"][0], at).permute(0, 2, 1, 3, 4).reshape(n, H, N, d)
    V = _values(v, s["vs"][0], at).permute(0, 2, 1, 3, 4).reshape(n, H, N, d)
    key = torch.arange(N, device=DEV)
    V.masked_fill_((key >= s["lens"][seqs].long()[:, None])[:, None, :, None], 0.0)
    Q = q[idx].float().view(n, m, H, G, d).permute(0, 2, 3, 1, 4).reshape(n, H, G * m, d)
    S = torch.matmul(Q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(n, H, G, m, N)
    S.masked_fill_((key > pos[:, :, None])[:, None, None], -math.inf)
    S.sub_(S.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    total = S.sum(-1, keepdim=True).clamp_min(1e-30)
    O = torch.matmul(S.view(n, H, G * m, N), V).view(n, H, G, m, d) / total
    s["out"][idx[there]] = O.permute(0, 3, 1, 2, 4).reshape(n, m, Hq, d)[there].to(q.dtype)
    return s["out"]


def _exponent(largest):
    """The least e in -60 .. 60 with largest <= 448 * 2^e."""
    frac, e = torch.frexp(largest)
    return torch.where(largest > 0, (e - torch.where(frac <= 0.875, 9, 8)).clamp(-60, 60), -60)


def _norm_rotate(s, x, w, angle):
    """x [rows][heads][d] in 32 bits: normed per head where w is given, then rotated by its row's angles."""
    x = x.float()
    d, rot = x.shape[-1], s["case"]["rot"]
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    if rot == "none":
        return x
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., :d // 2], x[..., d // 2:]) if rot == "half" else (x[..., 0::2], x[..., 1::2])
    y = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat(y, -1) if rot == "half" else torch.stack(y, -1).flatten(-2)


def _join_pages(pool, scale, x, page, slot, first):
    """New rows x [rows][heads][d] into 8-bit pages; a page's rows below first [pages] are its old ones."""
    n, H, P, d = pool.shape
    top = torch.zeros((n, H), device=DEV).scatter_reduce_(0, page[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    touched = torch.zeros(n, dtype=torch.bool, device=DEV)
    touched[page] = True
    touched = touched.nonzero().squeeze(1)
    e, was, held = _exponent(top[touched]), scale[touched], first[touched] > 0
    to = torch.where(held[:, None], torch.maximum(torch.exp2(e.float()), was), torch.exp2(e.float()))
    scale[touched] = to
    raw = pool.view(torch.uint8)
    bits = raw[touched]
    again = (bits.view(F8).float() * (was / to)[..., None, None]).to(F8).view(torch.uint8)
    old = torch.arange(P, device=DEV) < first[touched][:, None]
    raw[touched] = torch.where(old[:, None, :, None], again, bits)
    raw[page, :, slot] = (x / scale[page][..., None]).to(F8).view(torch.uint8)


def _plain_append(s):
    k, v, x = s["k"][0], s["v"][0], s["qkv"]
    H, P = k.shape[1:3]
    Hq, d = x.shape[1] - 2 * H, x.shape[2]
    idx, there, pos = _new_rows(s)
    idx, at = idx[there], pos[there]
    seq = s["seqs"].long()[:, None].expand_as(pos)[there]
    page, slot = s["table"][seq, at // P].long(), at % P
    if s["case"]["axes"]:
        angle = s["at"][s["axis"]][:, idx].T.double() * s["rate"]
    else:
        angle = at.double()[:, None] * BASE ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
    s["out"][idx] = _norm_rotate(s, x[idx, :Hq], s["w"][0], angle).to(x.dtype)
    keys, values = _norm_rotate(s, x[idx, Hq:Hq + H], s["w"][1], angle), x[idx, Hq + H:]
    if _bits(s["case"]) != 8:
        k[page, :, slot] = keys.to(x.dtype)
        v[page, :, slot] = values
        return s["out"], s["k"], s["v"]
    first = torch.zeros(s["pages"], dtype=torch.int64, device=DEV)
    start = pos[:, 0]
    first[s["table"][s["seqs"].long(), start // P].long()] = start % P
    _join_pages(k, s["ks"][0], keys, page, slot, first)
    _join_pages(v, s["vs"][0], values.float(), page, slot, first)
    return s["out"], s["k"], s["v"], s["ks"], s["vs"]


def _plain_keep(s, pool, scale, src, back):
    P = s["case"]["page"]
    L, n, H, S, d = src.shape
    seq, j = (s["table"] >= 0).nonzero().T
    page = s["table"][seq, j].long()
    pos = j[:, None] * P + torch.arange(P, device=DEV)
    here = pos < s["lens"].long()[seq][:, None]
    at = pos.clamp_max(S - 1)
    x = src[:, seq[:, None], :, at].permute(2, 0, 3, 1, 4).float()   # [L][page][H][P][d]
    x.masked_fill_(~here[None, :, None, :, None], 0.0)
    scale[:, page] = torch.exp2(_exponent(x.abs().amax((3, 4))).float())
    raw = pool.view(torch.uint8)
    bits = (x / scale[:, page][..., None, None]).to(F8).view(torch.uint8)
    raw[:, page] = torch.where(here[None, :, None, :, None], bits, raw[:, page])
    y = (pool.view(torch.uint8)[:, page].view(F8).float() * scale[:, page][..., None, None]).to(src.dtype)
    back[:, seq[:, None].expand_as(at)[here], :, at[here]] = y.permute(1, 3, 0, 2, 4)[here]


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["kind"] == "attn":
        return _plain_attention(s)
    if s["kind"] == "append":
        return _plain_append(s)
    _plain_keep(s, s["k"], s["ks"], s["new"][0], s["back"][0])
    _plain_keep(s, s["v"], s["vs"], s["new"][1], s["back"][1])
    return [s["k"], s["v"], s["ks"], s["vs"], *s["back"]]


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2607_28979_gb300.mot as M
    h, c = s["h"], s["cache"]
    if s["kind"] == "keep":
        M.mot_paged_store(h, c, s["seqs"], s["n"], *s["new"])
        M.mot_paged_load(h, c, s["seqs"], s["n"], *s["back"])
        return [s["k"], s["v"], s["ks"], s["vs"], *s["back"]]
    b = M.paged_batch(s["seqs"], s["starts"], s["n"], s["rows"], s["chunk"])
    if s["kind"] == "attn":
        M.mot_paged_attention(h, 0, c, b, s["q"], s["out"])
        return s["out"]
    x = s["qkv"]
    H = s["k"].shape[2]
    Hq = x.shape[1] - 2 * H
    args = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], s["out"], *s["w"]
    if s["case"]["axes"]:
        M.mot_paged_append_at(h, 0, c, b, s["at"], *args)
    else:
        M.mot_paged_append(h, 0, c, b, *args)
    return (s["out"], s["k"], s["v"]) if _bits(s["case"]) != 8 else (s["out"], s["k"], s["v"], s["ks"], s["vs"])


# ---------------------------------------------------------------- work

def work(case):
    Hq, H, d, L = MODELS[case["model"]]
    es, lens, P, pages = (2 if case["dtype"] == "bf16" else 4), _ints(case["lens"]), case["page"], _page_counts(case)
    cell = _bits(case) // 8
    if case["kind"] == "keep":   # read, written in 8 bits, and both again
        return {"bytes": 2 * L * H * (d * sum(lens) * 2 * (es + 1) + 8 * sum(pages)), "flops": 0}
    chunks = _ints(case["chunks"])
    rows = sum(chunks)
    if case["kind"] == "append":
        touched = sum((n - 1) // P - (n - m) // P + 1 for n, m in zip(lens, chunks) if m) if cell == 1 else 0
        at = 4 * AXES * rows if case["axes"] else 0
        return {"bytes": d * rows * (es * 2 * (Hq + H) + 2 * H * cell) + at + 8 * H * touched, "flops": 6 * d * rows * (Hq + H)}
    keys = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, chunks))
    return {"bytes": 2 * H * (d * sum(lens) + 4 * sum(pages)) + es * d * 2 * Hq * rows, "flops": 4 * keys * Hq * d}


# ---------------------------------------------------------------- the same in 64 bits

def _rows_of(s, i, pool, scale):
    """Sequence i's positions of one layer of a pool, [heads][len][d] in 64 bits."""
    pages = [int(p) for p in s["table"][i].tolist() if p >= 0]
    return torch.cat([pool[p].double() * scale[p].double()[:, None, None] for p in pages], 1)[:, :int(s["lens"][i])]


def _exact_attention(s):
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    d = s["q"].shape[2]
    G = s["q"].shape[1] // s["k"].shape[2]
    for i, n in enumerate(lens):
        K, V = _rows_of(s, i, s["k"][0], s["ks"][0]), _rows_of(s, i, s["v"][0], s["vs"][0])
        for r0 in range(starts[i], starts[i + 1], 512):
            r1 = min(starts[i + 1], r0 + 512)
            last = torch.arange(n - starts[i + 1] + r0, n - starts[i + 1] + r1, device=DEV)[:, None]
            hide = torch.arange(n, device=DEV) > last
            for h in range(s["q"].shape[1]):
                a = s["q"][r0:r1, h].double() @ K[h // G].T / math.sqrt(d)
                out[r0:r1, h] = torch.softmax(a.masked_fill(hide, -math.inf), 1) @ V[h // G]
    return out


def _eighths(x):
    """x in 64 bits to the nearest of the 8-bit floats, ties to the even one: 3 bits behind the leading one, steps of
    2^-9 below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _least_scale(top):
    """2^e with the least e in -60 .. 60 with top <= 448 * 2^e, [heads]."""
    def one(t):
        e = -60
        if t > 0:
            e = max(-60, math.frexp(t)[1] - 12)
            while e < 60 and t > 448 * 2.0 ** e:
                e += 1
        return 2.0 ** e
    return torch.tensor([one(t) for t in top.tolist()], dtype=torch.float64, device=DEV)


def _exact_append(s):
    q, P, H = s["out"].double(), s["k"].shape[3], s["k"].shape[2]
    Hq, d, rot, eight = q.shape[1], q.shape[2], s["case"]["rot"], _bits(s["case"]) == 8
    x = s["qkv"].double()
    for i, w in ((0, s["w"][0]), (1, s["w"][1])):
        if w is not None:
            y = x[:, :Hq] if i == 0 else x[:, Hq:Hq + H]
            y.copy_(y / (y.pow(2).sum(2, keepdim=True) / d + EPS).sqrt() * w.double())
    lens, starts, table = s["lens"].tolist(), s["starts"].tolist(), s["table"].tolist()
    spans = [(n - (b - a), n) for n, a, b in zip(lens, starts, starts[1:])]
    pos = torch.cat([torch.arange(a, b) for a, b in spans]).double().to(DEV)
    if rot != "none":
        pair = torch.arange(d // 2, device=DEV, dtype=torch.float64)
        angle = pos[:, None] * torch.exp(-2 * pair / d * math.log(BASE))
        if s["case"]["axes"]:
            axis, rate = _axes(s["case"])
            angle = torch.stack([s["at"][a].double() * r for a, r in zip(axis, rate)], 1)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        y = x[:, :Hq + H]
        z = torch.complex(y[..., :d // 2], y[..., d // 2:]) if rot == "half" else torch.view_as_complex(y.reshape(*y.shape[:2], d // 2, 2).contiguous())
        z = z * turn
        y.copy_(torch.cat([z.real, z.imag], -1) if rot == "half" else torch.view_as_real(z).flatten(2))
    q.copy_(x[:, :Hq])
    pools = [s["k"].double(), s["v"].double()]
    scales = [s["ks"].double(), s["vs"].double()] if eight else []
    if not eight:
        page = torch.tensor([table[i][p // P] for i, (a, b) in enumerate(spans) for p in range(a, b)], device=DEV)
        slot = pos.long() % P
        for y, c in zip(pools, (x[:, Hq:Hq + H], x[:, Hq + H:])):
            y[0, page, :, slot] = c
        return q, *pools
    for i, (a, b) in enumerate(spans):   # page by page
        while a < b:
            to, page, slot = min(b, (a // P + 1) * P), table[i][a // P], a % P
            r = starts[i] + a - spans[i][0]
            for y, c, sc in zip(pools, (x[:, Hq:Hq + H], x[:, Hq + H:]), scales):
                rows = c[r:r + to - a].transpose(0, 1)
                new = _least_scale(rows.abs().amax((1, 2)))
                if slot:
                    new = torch.maximum(new, sc[0, page])
                    y[0, page, :, :slot] = _eighths(y[0, page, :, :slot] * (sc[0, page] / new)[:, None, None])
                sc[0, page] = new
                y[0, page, :, slot:slot + to - a] = _eighths(rows / new[:, None, None])
            a = to
    return q, *pools, *scales


def _exact_keep(s):
    P, lens, table = s["case"]["page"], s["lens"].tolist(), s["table"].tolist()
    pools, scales, back = [s["k"].double(), s["v"].double()], [s["ks"].double(), s["vs"].double()], [x.double() for x in s["back"]]
    for y, sc, src, b in zip(pools, scales, s["new"], back):
        L, _, H = src.shape[:3]
        for i, n in enumerate(lens):
            for j in range(-(-n // P)):
                m, page = min(P, n - j * P), table[i][j]
                x = src[:, i, :, j * P:j * P + m].double()
                new = _least_scale(x.abs().amax((2, 3)).flatten()).view(L, H)
                sc[:, page] = new
                y[:, page, :, :m] = _eighths(x / new[..., None, None])
                b[:, i, :, j * P:j * P + m] = y[:, page, :, :m] * new[..., None, None]
    return [*pools, *scales, *back]


def exact(case, seed):
    if work(case)["flops"] > 6e12:   # over about 20 seconds at the 64-bit rate
        return None
    s = prepare(case, seed)
    return {"attn": _exact_attention, "append": _exact_append, "keep": _exact_keep}[s["kind"]](s)
