"""Performance cases of the paged cache: its pages, the append of new keys and values, and the
attention of new tokens over it.

A target model that got its context by translation goes on from there: the translated cache is
stored into pages, forked to the branches that share it, and each step reserves room for its new
tokens, writes their keys and values (with the norms and the rotation of the model) and attends
over the pages. Head counts and widths are those of the repository's own targets.

``run`` computes the plain form with elementary torch operations in 32 bits (angles in 64); with
``own`` set it makes the library's calls. ``exact`` restates each operator in 64 bits.
"""
import math

import torch

own = False
DEV = "cuda"

# Query heads, key/value heads, head width and layers of the targets.
MODELS = {"opt125m": (12, 12, 64, 12), "qwen05": (14, 2, 64, 24), "qwen15": (12, 2, 128, 28),
          "qwen7": (28, 4, 128, 28)}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE, EPS = 1e6, 1e-6


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
        # ---- attention: lens are the positions with the new ones, chunks the new ones
        # The smallest: one token of one conversation, a short prompt behind it.
        dict(name="attn_decode_one", kind="attn", model="qwen15", lens="517", chunks="1", page=16, dtype="bf16"),
        # One token for each of 64 conversations of very different lengths.
        dict(name="attn_decode_64", kind="attn", model="qwen7", lens=_text(_spread(64, 100, 16384)),
             chunks=_text([1] * 64), page=64, dtype="bf16"),
        # One token for each of two very long contexts: few rows, the length is the work.
        dict(name="attn_decode_long", kind="attn", model="qwen7", lens="131072,70001", chunks="1,1", page=128, dtype="bf16"),
        # Prompts of several sizes on translated contexts, conversations that decode among them.
        dict(name="attn_prompts_mixed", kind="attn", model="opt125m", lens="1087,2050,513,777,64,1500",
             chunks="63,1024,1,130,64,7", page=32, dtype="bf16"),
        # The largest: a piece of 4,096 tokens of a long document on top of what is there.
        dict(name="attn_chunk_long", kind="attn", model="qwen7", lens="32768", chunks="4096", page=64, dtype="bf16"),
        # The parity-precision type: a prompt and a decoding step in 32 bits.
        dict(name="attn_fp32", kind="attn", model="opt125m", lens="1024,300", chunks="64,1", page=16, dtype="fp32"),
        # ---- append
        # One new token, at the far end of a context.
        dict(name="append_one", kind="append", model="qwen15", lens="90001", chunks="1", page=16, rot="half", norm=False, dtype="bf16"),
        # Prompts of four conversations, keys and queries normed and rotated.
        dict(name="append_prompts", kind="append", model="qwen7", lens="32768,2111,9000,4097", chunks="4096,2111,1999,2048",
             page=64, rot="half", norm=True, dtype="bf16"),
        # ---- pages
        # One branch of one short context is dropped and forked again.
        dict(name="fork_one", kind="fork", model="opt125m", lens="700", children=1, page=16, dtype="bf16"),
        # Two translated prefixes, eight agents on each.
        dict(name="fork_agents", kind="fork", model="qwen7", lens="8191,4001", children=8, page=64, dtype="bf16"),
        # A conversation ends; the pool is compacted and the next translated context takes its place.
        dict(name="admit_context", kind="admit", model="qwen7", lens="8192,5003,12001,7777,4096,10240", page=64, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "chunk", "chunk", "mixed", "fp32", "append", "append", "fork", "admit"))
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
    if kind == "fp32":
        n = rng.choice((1, 2, 4))
        new = [rng.choice((1, _log(rng, 1, 256))) for _ in range(n)]
        return dict(c, lens=_text([x + _log(rng, 1, 2000) for x in new]), chunks=_text(new), dtype="fp32")
    if kind == "append":
        n = _log(rng, 1, 64)
        new = [rng.choice((1, _log(rng, 1, max(2, 8000 // n)))) for _ in range(n)]
        lens = [x + _log(rng, 1, 100000 // n) for x in new]
        return dict(c, kind="append", lens=_text(lens), chunks=_text(new), norm=rng.random() < 0.5,
                    rot=rng.choice(("half", "half", "pairs", "none")), dtype=rng.choice(("bf16", "bf16", "fp32")))
    if kind == "fork":
        n = rng.choice((1, 1, 2, 4))
        return dict(c, kind="fork", lens=_text([_log(rng, 16, 8000) for _ in range(n)]), children=rng.choice((1, 2, 4, 8)))
    return dict(c, kind="admit", lens=_text([_log(rng, 64, 8000) for _ in range(rng.choice((2, 3, 5)))]))


# ---------------------------------------------------------------- inputs

def _page_counts(case):
    return [-(-n // case["page"]) for n in _ints(case["lens"])]


def _pool(case, gen, layers, pages):
    """Keys and values of a pool, [layers][pages][heads][page][width]: normal draws with per-channel scales."""
    _, H, d, _ = MODELS[case["model"]]
    out = []
    for _ in range(2):
        s = torch.exp(0.5 * torch.randn((H, 1, d), generator=gen, device=DEV))
        x = torch.empty((layers, pages, H, case["page"], d), dtype=TYPES[case["dtype"]], device=DEV)
        for l in range(layers):
            x[l] = torch.randn(x[l].shape, generator=gen, device=DEV) * s
        out.append(x)
    return out


def _normal(gen, case, *shape):
    return torch.randn(shape, generator=gen, device=DEV).to(TYPES[case["dtype"]])


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


_handles = {}


def _handle(case, layers, pages, slots, width):
    """The program's handle for caches of one form, made once and kept."""
    import paper_2607_28979_gb300.mot as M
    Hq, H, d, _ = MODELS[case["model"]]
    rot = case.get("rot", "none")
    key = (Hq, H, d, layers, pages, slots, width, case["page"], case["dtype"], rot)
    if key not in _handles:
        _handles[key] = M.mot_create_paged(M.make_paged_config(
            layers, Hq, H, d, case["page"], pages, slots, width, rot_dim=0 if rot == "none" else d,
            rot_pairs=rot == "pairs", rot_base=BASE, norm_eps=EPS, dtype=case["dtype"]))
    return _handles[key]


def prepare(case, seed):
    Hq, H, d, L = MODELS[case["model"]]
    lens, need, kind = _ints(case["lens"]), _page_counts(case), case["kind"]
    n = len(lens)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    layers = 1 if kind in ("attn", "append") else L
    kids = case.get("children", 0)
    slots, width = n * (1 + kids), max(need)
    # spare pages: a fork's copies, an eighth more of what serving pools keep free
    pages = sum(need) + n * kids + max(4, sum(need) // 8)
    s = dict(case=case, kind=kind, n=n, width=width, slots=slots, pages=pages)
    s["k"], s["v"] = _pool(case, gen, layers, pages)
    s["table"] = torch.full((slots, width), -1, dtype=torch.int32, device=DEV)
    s["lens"] = torch.zeros(slots, dtype=torch.int32, device=DEV)
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    # pages lie as a pool in use has them: in no order, and for an attention or an append among free ones
    among = sum(need) if kind == "admit" else pages
    perm = torch.randperm(among, generator=gen, device=DEV).to(torch.int32)
    at = 0
    for i, m in enumerate(need):
        s["table"][i, :m] = perm[at:at + m]
        s["lens"][i] = lens[i]
        at += m
    s["refs"][perm[:at].long()] = 1
    if kind in ("attn", "append"):
        chunks = _ints(case["chunks"])
        starts = [sum(chunks[:i]) for i in range(n + 1)]
        s.update(seqs=_i32(range(n)), starts=_i32(starts), rows=starts[-1], chunk=max(chunks))
        if kind == "attn":
            s["q"] = _normal(gen, case, starts[-1], Hq, d)
        else:   # the columns of a fused projection's output
            s["qkv"] = _normal(gen, case, starts[-1], Hq + 2 * H, d)
            s["w"] = [(1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(TYPES[case["dtype"]])
                      for _ in range(2)] if case["norm"] else [None, None]
        s["out"] = torch.zeros((starts[-1], Hq, d), dtype=TYPES[case["dtype"]], device=DEV)
    elif kind == "fork":
        s["src"] = _i32([i for i in range(n) for _ in range(kids)])
        s["dst"] = _i32(range(n, slots))
    else:
        s["turn"] = 0
        s["one"] = [_i32([i]) for i in range(n)]
        s["starts"] = [_i32([0, m]) for m in lens]
        s["new"] = [_normal(gen, case, L, 1, H, max(lens), d) for _ in range(2)]
        s["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if own:   # the handle that a program of this form keeps
        import paper_2607_28979_gb300.mot as M
        s["h"] = _handle(case, layers, pages, slots, width)
        s["cache"] = M.paged_cache(s["k"], s["v"], s["table"], s["lens"], s["refs"])
    return s


# ---------------------------------------------------------------- plain forms

def _new_rows(s):
    """Row index [n][chunk], whether there is such a row, and its position in the sequence."""
    seqs = s["seqs"].long()
    starts = s["starts"].long()
    m = starts[1:] - starts[:-1]
    r = torch.arange(s["chunk"], device=DEV)
    return (starts[:-1, None] + r).clamp_max(s["rows"] - 1), r < m[:, None], s["lens"][seqs].long()[:, None] - m[:, None] + r


def _plain_attention(s):
    k, v, q = s["k"][0], s["v"][0], s["q"]
    H, P, d = k.shape[1:]
    n, Hq = s["n"], q.shape[1]
    seqs = s["seqs"].long()
    at = s["table"][seqs].long().clamp_min(0)
    idx, there, pos = _new_rows(s)
    N, m, G = at.shape[1] * P, idx.shape[1], Hq // H
    K = k[at].permute(0, 2, 1, 3, 4).reshape(n, H, N, d).float()
    V = v[at].permute(0, 2, 1, 3, 4).reshape(n, H, N, d).float()
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


def _norm_rotate(s, x, w, pos):
    """x [rows][heads][d] in 32 bits: normed per head where w is given, then rotated by its position."""
    x = x.float()
    d, rot = x.shape[-1], s["case"]["rot"]
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    if rot == "none":
        return x
    inv = BASE ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
    t = pos.double()[:, None, None] * inv
    cos, sin = t.cos().float(), t.sin().float()
    a, b = (x[..., :d // 2], x[..., d // 2:]) if rot == "half" else (x[..., 0::2], x[..., 1::2])
    y = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat(y, -1) if rot == "half" else torch.stack(y, -1).flatten(-2)


def _plain_append(s):
    k, v, x = s["k"][0], s["v"][0], s["qkv"]
    H, P = k.shape[1:3]
    Hq = x.shape[1] - 2 * H
    idx, there, pos = _new_rows(s)
    idx, at = idx[there], pos[there]
    seq = s["seqs"].long()[:, None].expand_as(pos)[there]
    page, slot = s["table"][seq, at // P].long(), at % P
    s["out"][idx] = _norm_rotate(s, x[idx, :Hq], s["w"][0], at).to(x.dtype)
    k[page, :, slot] = _norm_rotate(s, x[idx, Hq:Hq + H], s["w"][1], at).to(x.dtype)
    v[page, :, slot] = x[idx, Hq + H:]
    return s["out"], s["k"], s["v"]


def _plain_free(s, seqs):
    rows = s["table"][seqs]
    used = rows[rows >= 0].long()
    s["refs"].scatter_add_(0, used, torch.full_like(used, -1, dtype=torch.int32))
    s["table"][seqs] = -1
    s["lens"][seqs] = 0


def _plain_fork(s):
    P = s["case"]["page"]
    src, dst = s["src"].long(), s["dst"].long()
    n = s["lens"][src].long()
    part = torch.nonzero(n % P).squeeze(1)
    take = torch.nonzero(s["refs"] == 0).squeeze(1)[:part.numel()]
    rows = s["table"][src]
    old = rows[part, n[part] // P].long()
    rows[part, n[part] // P] = take.to(torch.int32)
    used = rows[rows >= 0].long()
    s["refs"].scatter_add_(0, used, torch.ones_like(used, dtype=torch.int32))
    s["table"][dst] = rows
    s["lens"][dst] = n.to(torch.int32)
    filled = (torch.arange(P, device=DEV) < (n[part] % P)[:, None])[None, :, None, :, None]
    for x in (s["k"], s["v"]):
        x[:, take] = torch.where(filled, x[:, old], x[:, take])


def _plain_compact(s):
    live = s["refs"] > 0
    n = live.sum()
    page = torch.arange(s["pages"], device=DEV)
    holes, movers = torch.nonzero(~live & (page < n)).squeeze(1), torch.nonzero(live & (page >= n)).squeeze(1)
    to = page.to(torch.int32)
    to[movers] = holes.to(torch.int32)
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp_min(0).long()], -1))
    s["refs"][holes] = s["refs"][movers]
    s["refs"][movers] = 0
    for x in (s["k"], s["v"]):
        x[:, holes] = x[:, movers]
    s["live"].copy_(n)


def _plain_reserve(s, seq, starts):
    P = s["case"]["page"]
    new = starts[1:] - starts[:-1]
    count = (new + P - 1).div(P, rounding_mode="floor")
    take = torch.nonzero(s["refs"] == 0).squeeze(1)[:count.item()]
    s["table"][seq.long(), :take.numel()] = take.to(torch.int32)
    s["refs"][take] = 1
    s["lens"][seq.long()] = new


def _plain_store(s, seq, src):
    P = s["case"]["page"]
    n = s["lens"][seq.long()]
    pos = torch.arange(n.item(), device=DEV)
    page = s["table"][seq.long()[0], pos // P].long()
    for x, y in zip((s["k"], s["v"]), src):
        x[:, page, :, pos % P] = y[:, 0, :, :pos.numel()].permute(2, 0, 1, 3)


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["kind"] == "attn":
        return _plain_attention(s)
    if s["kind"] == "append":
        return _plain_append(s)
    if s["kind"] == "fork":   # the branches of the last turn end, the next ones start
        _plain_free(s, s["dst"].long())
        _plain_fork(s)
    else:
        i = s["turn"]
        s["turn"] = (i + 1) % s["n"]
        _plain_free(s, s["one"][i].long())
        _plain_compact(s)
        _plain_reserve(s, s["one"][i], s["starts"][i])
        _plain_store(s, s["one"][i], s["new"])
    return [s[x] for x in ("table", "lens", "refs", "k", "v")]


# ---------------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2607_28979_gb300.mot as M
    h, c = s["h"], s["cache"]
    if s["kind"] in ("attn", "append"):
        b = M.paged_batch(s["seqs"], s["starts"], s["n"], s["rows"], s["chunk"])
        if s["kind"] == "attn":
            M.mot_paged_attention(h, 0, c, b, s["q"], s["out"])
            return s["out"]
        x = s["qkv"]
        H = s["k"].shape[2]
        Hq = x.shape[1] - 2 * H
        M.mot_paged_append(h, 0, c, b, x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], s["out"], *s["w"])
        return s["out"], s["k"], s["v"]
    if s["kind"] == "fork":
        M.mot_paged_free(h, c, s["dst"], s["dst"].numel())
        M.mot_paged_fork(h, c, s["src"], s["dst"], s["dst"].numel())
    else:
        i = s["turn"]
        s["turn"] = (i + 1) % s["n"]
        M.mot_paged_free(h, c, s["one"][i], 1)
        M.mot_paged_compact(h, c, s["live"])
        new = _ints(s["case"]["lens"])[i]
        M.mot_paged_reserve(h, c, M.paged_batch(s["one"][i], s["starts"][i], 1, new, new))
        M.mot_paged_store(h, c, s["one"][i], 1, *s["new"])
    return [s[x] for x in ("table", "lens", "refs", "k", "v")]


# ---------------------------------------------------------------- work

def work(case):
    Hq, H, d, L = MODELS[case["model"]]
    es, lens, P = (2 if case["dtype"] == "bf16" else 4), _ints(case["lens"]), case["page"]
    if case["kind"] in ("attn", "append"):
        chunks = _ints(case["chunks"])
        rows = sum(chunks)
        if case["kind"] == "append":
            return {"bytes": es * d * rows * 2 * (Hq + 2 * H), "flops": 6 * d * rows * (Hq + H)}
        keys = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, chunks))
        return {"bytes": es * d * (2 * H * sum(n for n, m in zip(lens, chunks) if m) + 2 * Hq * rows), "flops": 4 * keys * Hq * d}
    row = L * H * d * es * 2   # a position's keys and values of every layer
    if case["kind"] == "fork":
        return {"bytes": 2 * row * case["children"] * sum(n % P for n in lens) + 8 * case["children"] * sum(_page_counts(case)), "flops": 0}
    # the first conversation's pages: those that lie below the new end are filled from above it
    c = _page_counts(case)
    return {"bytes": 2 * row * (lens[0] + P * c[0] * (1 - c[0] / sum(c))), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits

def _rows_of(s, i, pool):
    """Sequence i's positions of one layer of a pool, [heads][len][d] in 64 bits."""
    n = int(s["lens"][i])
    pages = [int(p) for p in s["table"][i].tolist() if p >= 0]
    return torch.cat([pool[p] for p in pages], 1)[:, :n].double()


def _exact_attention(s):
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    d = s["q"].shape[2]
    G = s["q"].shape[1] // s["k"].shape[2]
    for i, n in enumerate(lens):
        K, V = _rows_of(s, i, s["k"][0]), _rows_of(s, i, s["v"][0])
        for r0 in range(starts[i], starts[i + 1], 512):
            r1 = min(starts[i + 1], r0 + 512)
            last = torch.arange(n - starts[i + 1] + r0, n - starts[i + 1] + r1, device=DEV)[:, None]
            hide = torch.arange(n, device=DEV) > last
            for h in range(s["q"].shape[1]):
                a = s["q"][r0:r1, h].double() @ K[h // G].T / math.sqrt(d)
                out[r0:r1, h] = torch.softmax(a.masked_fill(hide, -math.inf), 1) @ V[h // G]
    return out


def _exact_append(s):
    k, v, q = s["k"].double(), s["v"].double(), s["out"].double()
    P, H = k.shape[3], k.shape[2]
    Hq, d, rot = q.shape[1], q.shape[2], s["case"]["rot"]
    x = s["qkv"].double()
    for i, w in ((0, s["w"][0]), (1, s["w"][1])):
        if w is not None:
            y = x[:, :Hq] if i == 0 else x[:, Hq:Hq + H]
            y.copy_(y / (y.pow(2).sum(2, keepdim=True) / d + EPS).sqrt() * w.double())
    lens, starts, table = s["lens"].tolist(), s["starts"].tolist(), s["table"].tolist()
    pos = torch.cat([torch.arange(n - (b - a), n) for n, a, b in zip(lens, starts, starts[1:])]).double().to(DEV)
    if rot != "none":
        pair = torch.arange(d // 2, device=DEV, dtype=torch.float64)
        turn = torch.polar(torch.ones_like(pos)[:, None], pos[:, None] * torch.exp(-2 * pair / d * math.log(BASE)))[:, None]
        y = x[:, :Hq + H]
        z = torch.complex(y[..., :d // 2], y[..., d // 2:]) if rot == "half" else torch.view_as_complex(y.reshape(*y.shape[:2], d // 2, 2).contiguous())
        z = z * turn
        y.copy_(torch.cat([z.real, z.imag], -1) if rot == "half" else torch.view_as_real(z).flatten(2))
    q.copy_(x[:, :Hq])
    page = torch.tensor([table[i][p // P] for i, n in enumerate(lens) for p in range(n - (starts[i + 1] - starts[i]), n)], device=DEV)
    slot = pos.long() % P
    k[0, page, :, slot], v[0, page, :, slot] = x[:, Hq:Hq + H], x[:, Hq + H:]
    return q, k, v


def _exact_pages(s):
    """The bookkeeping on lists; the pools follow page by page."""
    P, table, lens, refs = s["case"]["page"], s["table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    k, v = s["k"].clone(), s["v"].clone()

    def lowest(count):
        got = [p for p, r in enumerate(refs) if r == 0][:count]
        for p in got:
            refs[p] = 1
        return got

    def free(i):
        for p in table[i]:
            if p >= 0:
                refs[p] -= 1
        table[i], lens[i] = [-1] * len(table[i]), 0

    if s["kind"] == "fork":
        src, dst = s["src"].tolist(), s["dst"].tolist()
        for i in dst:
            free(i)
        for a, b in zip(src, dst):
            table[b], lens[b] = list(table[a]), lens[a]
            full, part = divmod(lens[a], P)
            for p in table[b][:full]:
                refs[p] += 1
            if part:
                table[b][full], = lowest(1)
                for x in (k, v):
                    x[:, table[b][full], :, :part] = x[:, table[a][full], :, :part]
    else:
        n = lens[0]
        free(0)
        live = sum(r > 0 for r in refs)
        holes = [p for p in range(live) if refs[p] == 0]
        for a, b in zip([p for p in range(live, len(refs)) if refs[p]], holes):
            refs[b], refs[a] = refs[a], 0
            table = [[b if p == a else p for p in row] for row in table]
            for x in (k, v):
                x[:, b] = x[:, a]
        got = lowest(-(-n // P))
        table[0][:len(got)], lens[0] = got, n
        for j, p in enumerate(got):
            m = min(P, n - j * P)
            for x, y in zip((k, v), s["new"]):
                x[:, p, :, :m] = y[:, 0, :, j * P:j * P + m]
    return [_i32(table), _i32(lens), _i32(refs), k, v]


def exact(case, seed):
    if work(case)["flops"] > 6e12:   # over about 20 seconds at the 64-bit rate
        return None
    s = prepare(case, seed)
    return {"attn": _exact_attention, "append": _exact_append}.get(s["kind"], _exact_pages)(s)
