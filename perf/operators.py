"""The cache operators as measurable cases: what a serving program does with a
compacted prefill buffer (positions of the kept rows, keys and values into a
paged cache, attention over the cache).

Every case goes through the public calls (``paper_2609_13804_amd.binding``)
when ``own`` is true, and through elementary torch operations in 32 bits when
it is false.  Sizes follow the settings in ``paper_2609_13804_amd/workloads.py``
(images of 256 to 4096 tokens of which about a tenth to a third is kept,
prompts of 32 to 512 rows, widths 1024 to 4096 as heads of 64 or 128) and the
usual range of a serving batch: 1 to 128 sequences, caches of one to 131072
tokens.

    own                   whether run() makes the library's calls
    listed()              the fixed cases
    draw(rng)             one more case of the same ranges
    prepare(case, seed)   inputs, the cache, outputs and workspaces on the GPU
    run(state)            one pass, its outputs
    work(case)            the bytes and operations that a pass cannot do without
    exact(case, seed)     the outputs in 64 bits, from the definitions
"""
import math
import random

import torch

own = False

PADDED, PACKED = "padded", "packed"


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # Positions of the benchmark's batch: 16 images of 576 tokens, a ninth kept, with
        # 64 prompt rows each, in a padded buffer.  Latency of one small launch.
        dict(name="positions_llava15", kind="positions", images=16, lo=576, hi=576, keep=0.111, text=64,
             axes=1, layout=PADDED),
        # Three position axes (frame, row, column) of the largest batch: 64 images of 3328
        # tokens, a tenth kept, with 512 prompt rows each, packed.
        dict(name="positions_internvl3_axes", kind="positions", images=64, lo=3328, hi=3328, keep=0.1,
             text=512, axes=3, layout=PACKED),
        # One generated token of one request, float32, width 1024: the smallest call.
        dict(name="append_one_f32", kind="append", dtype="f32", q_heads=16, kv_heads=16, head_dim=64,
             page=16, seqs=1, own_lo=640, own_hi=640, rows_lo=1, rows_hi=1, layout=PACKED, axes=0,
             rot=64, pairs="halves"),
        # One generated token for each of 128 requests, grouped heads, pages of 16, three
        # position axes: a decode step's append.
        dict(name="append_tokens", kind="append", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=16, seqs=128, own_lo=64, own_hi=1000, rows_lo=1, rows_hi=1, layout=PACKED, axes=3,
             rot=128, pairs="halves"),
        # The compacted prompts of 64 large images (333 kept tokens and 512 prompt rows on
        # average) entering the cache: the largest append.
        dict(name="append_prompts", kind="append", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=64, seqs=64, own_lo=690, own_hi=1000, rows_lo=690, rows_hi=1000, layout=PACKED, axes=1,
             rot=128, pairs="halves"),
        # One token of one float32 request over 640 rows: the smallest attention call.
        dict(name="attend_one_f32", kind="attend", dtype="f32", q_heads=16, kv_heads=16, head_dim=64,
             page=16, groups=0, seqs=1, own_lo=640, own_hi=640, rows_lo=1, rows_hi=1, layout=PACKED,
             full=False),
        # One token of one request over a compacted prompt and its answer so far, width 4096.
        dict(name="attend_one", kind="attend", dtype="bf16", q_heads=32, kv_heads=32, head_dim=128,
             page=16, groups=0, seqs=1, own_lo=707, own_hi=707, rows_lo=1, rows_hi=1, layout=PACKED,
             full=False),
        # A decode step of 128 requests of very unequal lengths, grouped heads.
        dict(name="attend_tokens", kind="attend", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=16, groups=0, seqs=128, own_lo=256, own_hi=8192, rows_lo=1, rows_hi=1, layout=PACKED,
             full=False),
        # One request with a very long cache (many images in one conversation).
        dict(name="attend_long", kind="attend", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=256, groups=0, seqs=1, own_lo=131001, own_hi=131001, rows_lo=1, rows_hi=1,
             layout=PACKED, full=False),
        # A decode step of 16 questions about each of 8 images: the images' rows are the
        # shared prefixes.
        dict(name="attend_shared", kind="attend", dtype="bf16", q_heads=32, kv_heads=32, head_dim=128,
             page=32, groups=8, seqs=128, prefix_lo=320, prefix_hi=2880, own_lo=16, own_hi=512, rows_lo=1,
             rows_hi=1, layout=PACKED, full=False),
        # 16 questions about each of 4 images, their whole prompts at once behind the shared
        # prefixes, in a padded buffer.
        dict(name="attend_questions", kind="attend", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=64, groups=4, seqs=64, prefix_lo=576, prefix_hi=2880, own_lo=24, own_hi=96, rows_lo=24,
             rows_hi=96, layout=PADDED, full=False),
        # The prompts of 8 uncompressed large images (3328 tokens and 512 prompt rows),
        # causal: the largest call.
        dict(name="attend_prompts", kind="attend", dtype="bf16", q_heads=28, kv_heads=4, head_dim=128,
             page=64, groups=0, seqs=8, own_lo=3840, own_hi=3840, rows_lo=3840, rows_hi=3840,
             layout=PACKED, full=False),
    ]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _span(rng, lo, hi):
    """Two integers in order, the upper one spread over its logarithm."""
    hi = _log(rng, lo, hi)
    return (hi if rng.random() < 0.3 else rng.randint(lo, hi)), hi


# no drawn case is larger than the largest listed one
MAX_BYTES, MAX_FLOPS, MAX_CACHE = 6.0e8, 6.0e11, 1 << 30


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS and _cache_bytes(c) <= MAX_CACHE:
            return c


def _draw(rng):
    kind = rng.choice(["positions", "append", "append", "attend", "attend", "attend", "attend"])
    layout = rng.choice([PADDED, PACKED])
    if kind == "positions":
        hi = rng.randint(256, 4096)
        return dict(kind=kind, images=_log(rng, 1, 64), lo=rng.randint(200, hi) if hi > 200 else hi, hi=hi,
                    keep=round(rng.uniform(0.02, 0.34), 3), text=_log(rng, 1, 512),
                    axes=rng.choice([1, 2, 3]), layout=layout)
    f32 = rng.random() < 0.25
    heads = rng.choice([(16, 16), (8, 1)] if f32 else [(32, 32), (16, 16), (28, 4), (32, 8), (8, 1), (40, 8)])
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", q_heads=heads[0], kv_heads=heads[1],
             head_dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128, 256]),
             seqs=_log(rng, 1, 32 if f32 else 128), layout=layout)
    if rng.random() < (0.5 if kind == "append" else 0.6):
        c["rows_lo"] = c["rows_hi"] = 1
    else:
        c["rows_lo"], c["rows_hi"] = _span(rng, 1, 200 if f32 else 2048)
    before = _log(rng, 1, 2000 if f32 else 8192)
    c["own_lo"] = c["rows_lo"] + rng.randint(0, before)
    c["own_hi"] = c["rows_hi"] + before
    if kind == "append":
        c["axes"] = rng.choice([0, 1, 2, 3])
        c["rot"] = rng.choice([c["head_dim"], c["head_dim"], c["head_dim"] // 2])
        c["pairs"] = rng.choice(["halves", "halves", "interleaved"])
        return c
    c["groups"] = 0
    c["full"] = rng.random() < 0.15
    if rng.random() < 0.5:
        c["groups"] = _log(rng, 1, max(1, c["seqs"] // 2))
        c["prefix_lo"], c["prefix_hi"] = _span(rng, 16, 1000 if f32 else 8192)
        if rng.random() < 0.5:
            c["own_hi"] = min(c["own_hi"], c["rows_hi"] + 200)
            c["own_lo"] = min(c["own_lo"], c["own_hi"])
    return c


# ---------------------------------------------------------------- sizes: the case alone decides them

def _rng(c):
    return random.Random("/".join(f"{k}={c[k]}" for k in sorted(c) if k != "name"))


def _images(c):
    """Visual tokens and kept tokens of every image."""
    r = _rng(c)
    sizes = [r.randint(c["lo"], c["hi"]) for _ in range(c["images"])]
    return sizes, [max(1, min(n, int(n * c["keep"] * r.uniform(0.7, 1.3)))) for n in sizes]


def _sequences(c):
    """New rows and cached tokens (the new ones included) of every sequence."""
    r = _rng(c)
    out = []
    for _ in range(c["seqs"]):
        n = r.randint(c["rows_lo"], c["rows_hi"])
        out.append((n, n + r.randint(c["own_lo"] - c["rows_lo"], max(c["own_lo"] - c["rows_lo"],
                                                                     c["own_hi"] - c["rows_hi"]))))
    return out


def _groups(c):
    """Sequences per group and prefix lengths."""
    if not c.get("groups"):
        return [], []
    r = random.Random(_rng(c).random())
    G, S = c["groups"], c["seqs"]
    cuts = [0] + [(g * S) // G for g in range(1, G)] + [S]
    return cuts, [r.randint(c["prefix_lo"], c["prefix_hi"]) for _ in range(G)]


def _pages_of(lens, page):
    return [-(-n // page) for n in lens]


def _cache_bytes(c):
    if c["kind"] == "positions":
        return 0
    lens = [L for _, L in _sequences(c)] + _groups(c)[1]
    return 2 * sum(_pages_of(lens, c["page"])) * c["page"] * c["kv_heads"] * c["head_dim"] * _bytes(c)


def _bytes(c):
    return 4 if c["dtype"] == "f32" else 2


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _ints(a):
    return torch.tensor(a, dtype=torch.int32).cuda()


# ---------------------------------------------------------------- inputs

class State:
    pass


def prepare(case, seed):
    s = State()
    s.c = c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = random.Random(seed)
    if c["kind"] == "positions":
        _prepare_positions(s, c, g)
    else:
        _prepare_cache(s, c, g, r)
        (_prepare_append if c["kind"] == "append" else _prepare_attend)(s, c, g, r)
    if own:
        _prepare_own(s, c)
    return s


def _prepare_positions(s, c, g):
    sizes, kept = _images(c)
    B, A = c["images"], c["axes"]
    s.sizes, s.kept, s.texts = sizes, kept, [c["text"]] * B
    s.img_off, s.text_off, s.kept_off = _ints(_offsets(sizes)), _ints(_offsets(s.texts)), _ints(_offsets(kept))
    s.kept_cnt = _ints(kept)
    s.T_vis, s.T_txt = sum(sizes), sum(s.texts)
    s.kept_idx = torch.cat([torch.sort(torch.randperm(n, generator=g, device="cuda")[:k])[0].int()
                            for n, k in zip(sizes, kept)])
    vis, txt = [], []
    for n, L in zip(sizes, s.texts):
        i = torch.arange(n, device="cuda")
        side = int(math.ceil(math.sqrt(n)))
        first = n if A == 1 else side
        shift = torch.randint(0, 8, (1,), generator=g, device="cuda")     # where a conversation stands
        vis.append((i[None] if A == 1 else torch.stack([0 * i, i // side, i % side])[3 - A:]) + shift)
        txt.append((first + shift + torch.arange(L, device="cuda"))[None].expand(A, L))
    s.vis_pos = torch.cat(vis, 1).int().contiguous()
    s.text_pos = torch.cat(txt, 1).int().contiguous()
    s.per_image = max(k + L for k, L in zip(kept, s.texts)) if c["layout"] == PADDED else 0
    s.out_rows = B * s.per_image if c["layout"] == PADDED else sum(kept) + s.T_txt
    s.pos = torch.zeros(A, s.out_rows, dtype=torch.int32, device="cuda")


def _normal(g, shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(0.0, scale, generator=g)


def _prepare_cache(s, c, g, r):
    """Rows of the batch, the runs' pages in a shuffled order, the cache."""
    seqs = _sequences(c)
    s.dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    s.n, s.len = [n for n, _ in seqs], [L for _, L in seqs]
    s.S = len(seqs)
    s.per_seq = max(s.n) if c["layout"] == PADDED else 0
    s.first = [i * s.per_seq for i in range(s.S)] if s.per_seq else _offsets(s.n)[:-1]
    s.T = s.S * s.per_seq if s.per_seq else sum(s.n)
    s.seq_info = _ints(s.n if s.per_seq else _offsets(s.n))
    s.cuts, s.prefix = _groups(c)
    counts = _pages_of(s.len, c["page"]) + _pages_of(s.prefix, c["page"])
    s.pages = sum(counts)
    order = list(range(s.pages))
    r.shuffle(order)
    tables, at = [], 0
    for k in counts:
        tables.append(order[at:at + k])
        at += k
    fill = lambda rows: _ints([t + [0] * (max(map(len, rows)) - len(t)) for t in rows])
    s.tables = fill(tables[:s.S])
    s.lens = _ints(s.len)
    if s.prefix:
        s.prefix_tables, s.prefix_lens, s.grp_off = fill(tables[s.S:]), _ints(s.prefix), _ints(s.cuts)
    shape = (s.pages, c["kv_heads"], c["page"], c["head_dim"])
    s.k_cache, s.v_cache = _normal(g, shape, s.dtype), _normal(g, shape, s.dtype)
    s.live = torch.cat([torch.arange(f, f + n) for f, n in zip(s.first, s.n)]).cuda()


def _prepare_append(s, c, g, r):
    """A fused product's q, k, v rows, and the angles of every position."""
    Hq, Hk, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    s.qkv = _normal(g, (s.T, (Hq + 2 * Hk) * D), s.dtype)
    s.q, s.k, s.v = s.qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    s.q_out = torch.zeros(s.T, Hq * D, dtype=s.dtype, device="cuda")
    pairs, axes = c["rot"] // 2, c["axes"]
    s.positions = max(s.len) + 64
    freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    ang = torch.arange(s.positions, dtype=torch.float64, device="cuda")[:, None] * freq
    s.cos_sin = torch.stack([ang.cos(), ang.sin()], dim=2).float().contiguous()
    s.sections = {0: [pairs], 1: [pairs], 2: [pairs // 2, pairs - pairs // 2],
                  3: [pairs // 4, 3 * pairs // 8, pairs - pairs // 4 - 3 * pairs // 8]}[axes]
    s.pos = None
    if axes:
        at = torch.cat([torch.arange(L - n, L) for n, L in seqs_of(s)]).cuda()
        s.pos = torch.zeros(axes, s.T, dtype=torch.int32, device="cuda")
        for a in range(axes):                       # the axes run apart by a few places
            s.pos[a, s.live] = (at + r.randint(0, 63)).int()


def seqs_of(s):
    return list(zip(s.n, s.len))


def _prepare_attend(s, c, g, r):
    Hq, D = c["q_heads"], c["head_dim"]
    s.q = _normal(g, (s.T, Hq * D), s.dtype, 2.0)    # scores of a few units: some keys stand out
    s.scale = 1.0 / math.sqrt(D)
    s.o = torch.zeros(s.T, Hq * D, dtype=s.dtype, device="cuda")
    s.lse = torch.zeros(s.T, Hq, dtype=torch.float32, device="cuda")


def _prepare_own(s, c):
    from paper_2609_13804_amd import binding as sp
    s.sp = sp
    s.layout = sp.SP_LAYOUT_PADDED if c["layout"] == PADDED else sp.SP_LAYOUT_PACKED
    nbytes = 256
    if c["kind"] != "positions":
        s.dims = sp.cache_dims(c["q_heads"], c["kv_heads"], c["head_dim"],
                               sp.SP_F32 if c["dtype"] == "f32" else sp.SP_BF16, c["page"], s.pages)
        s.rows = sp.cache_rows(s.T, s.layout, s.per_seq, s.seq_info, max(s.n))
        s.runs = sp.cache_runs(s.tables, s.lens, max(s.len))
    if c["kind"] == "append":
        s.rotation = sp.cache_rotation(s.cos_sin, c["rot"], s.pos, s.sections, c["pairs"] == "interleaved")
    if c["kind"] == "attend":
        s.shared = sp.cache_runs(s.prefix_tables, s.prefix_lens, max(s.prefix)) if s.prefix else None
        s.off = s.grp_off if s.prefix else None
        s.flags = sp.SP_ATTEND_ALL if c["full"] else 0
        nbytes = sp.stepprune_cache_workspace_bytes(s.dims, s.rows, s.runs, s.shared)
    s.ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s, s.c)
    return {"positions": _positions, "append": _append, "attend": _attend}[s.c["kind"]](s, s.c)


def _run_own(s, c):
    sp = s.sp
    if c["kind"] == "positions":
        sp.stepprune_compact_positions(s.vis_pos, s.T_vis, s.img_off, s.text_pos, s.T_txt, s.text_off, c["axes"],
                                       s.kept_idx, s.kept_off, s.kept_cnt, c["images"], s.layout, s.per_image,
                                       s.out_rows, s.pos, s.ws, s.ws.numel())
        return {"pos": s.pos}
    if c["kind"] == "append":
        sp.stepprune_cache_append(s.dims, s.q, s.q.stride(0), s.k, s.k.stride(0), s.v, s.v.stride(0), s.rows,
                                  s.runs, s.rotation, s.q_out, s.k_cache, s.v_cache, s.ws, s.ws.numel())
        return {"q": s.q_out, "k_cache": s.k_cache, "v_cache": s.v_cache}
    sp.stepprune_cache_attend(s.dims, s.q, s.q.stride(0), s.rows, s.runs, s.shared, s.off, s.scale, s.flags,
                              s.k_cache, s.v_cache, s.o, s.lse, s.ws, s.ws.numel())
    return {"o": s.o, "lse": s.lse}


def _positions(s, c):
    pos = torch.zeros_like(s.pos)
    at = img = txt = ki = 0
    for b, (n, k, L) in enumerate(zip(s.sizes, s.kept, s.texts)):
        if s.per_image:
            at = b * s.per_image
        rows = s.kept_idx[ki:ki + k].long() + img
        pos[:, at:at + k] = s.vis_pos[:, rows]
        pos[:, at + k:at + k + L] = s.text_pos[:, txt:txt + L]
        at, img, txt, ki = at + k + L, img + n, txt + L, ki + k
    return {"pos": pos}


def _rotate(x, cs, pairs):
    """x [rows, heads, D] in 32 bits, the first 2 len(cs) columns by cs [rows, pairs, (cos, sin)]."""
    half = cs.shape[1]
    c, s_ = cs[:, None, :, 0], cs[:, None, :, 1]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if pairs == "interleaved":
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * c - b * s_, b * c + a * s_], dim=-1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        head = torch.cat([a * c - b * s_, b * c + a * s_], dim=-1)
    return torch.cat([head, rest], dim=-1)


def _append(s, c):
    Hq, Hk, D, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    n = s.seq_info if s.per_seq else s.seq_info[1:] - s.seq_info[:-1]
    seq = torch.repeat_interleave(torch.arange(s.S, device="cuda"), n, output_size=s.live.numel())
    first = torch.cumsum(n, 0) - n
    slot = s.lens[seq] - n[seq] + torch.arange(seq.numel(), device="cuda") - first[seq]
    if c["axes"]:
        axis = torch.cat([torch.full((k,), a, device="cuda") for a, k in enumerate(s.sections)])
        at = s.pos[:, s.live].long()[axis].t()                                 # [rows, pairs]
        cs = s.cos_sin[at, torch.arange(axis.numel(), device="cuda")]
    else:
        cs = s.cos_sin[slot.long()]
    heads = lambda x, H: x[s.live].float().view(-1, H, D)
    s.q_out[s.live] = _rotate(heads(s.q, Hq), cs, c["pairs"]).flatten(1).to(s.dtype)
    where = s.tables[seq, slot // page].long(), slice(None), (slot % page).long()
    s.k_cache[where] = _rotate(heads(s.k, Hk), cs, c["pairs"]).to(s.dtype)
    s.v_cache[where] = heads(s.v, Hk).to(s.dtype)
    return {"q": s.q_out, "k_cache": s.k_cache, "v_cache": s.v_cache}


def _gather(cache, table, n, page):
    """The first n tokens of a run, [kv_heads, n, D] in 32 bits."""
    p = cache[table[:-(-n // page)].long()]                 # [pages, heads, page, D]
    return p.transpose(0, 1).flatten(1, 2)[:, :n].float()


def _attend(s, c):
    Hq, Hk, D, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    r = Hq // Hk
    o, lse = torch.zeros_like(s.o), torch.zeros_like(s.lse)
    grp = 0
    for i, (n, L) in enumerate(zip(s.n, s.len)):
        k, v = _gather(s.k_cache, s.tables[i], L, page), _gather(s.v_cache, s.tables[i], L, page)
        P = 0
        if s.prefix:
            while s.cuts[grp + 1] <= i:
                grp += 1
            P = s.prefix[grp]
            k = torch.cat([_gather(s.k_cache, s.prefix_tables[grp], P, page), k], 1)
            v = torch.cat([_gather(s.v_cache, s.prefix_tables[grp], P, page), v], 1)
        rows = slice(s.first[i], s.first[i] + n)
        q = s.q[rows].float().view(n, Hk, r, D).permute(1, 2, 0, 3).reshape(Hk, r * n, D)
        sc = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(s.scale).view(Hk, r, n, P + L)
        if n > 1 and not c["full"]:
            key = torch.arange(P + L, device="cuda")
            last = P + L - n + torch.arange(n, device="cuda")
            sc = sc.masked_fill(key[None, :] > last[:, None], -math.inf)
        m = sc.amax(-1, keepdim=True)
        p = torch.exp(sc - m)
        l = p.sum(-1, keepdim=True)
        out = torch.matmul(p.view(Hk, r * n, P + L), v.contiguous()).view(Hk, r, n, D) / l
        o[rows] = out.permute(2, 0, 1, 3).reshape(n, Hq * D).to(s.dtype)
        lse[rows] = (m + torch.log(l)).squeeze(-1).permute(2, 0, 1).reshape(n, Hq)
    return {"o": o, "lse": lse}


# ---------------------------------------------------------------- what a pass cannot do without

def work(c):
    if c["kind"] == "positions":
        sizes, kept = _images(c)
        rows = sum(kept) + c["images"] * c["text"]
        return {"bytes": 4 * (sum(kept) + 2 * c["axes"] * rows + 4 * c["images"]), "flops": 0}
    seqs = _sequences(c)
    e, Hq, Hk, D = _bytes(c), c["q_heads"], c["kv_heads"], c["head_dim"]
    T = sum(n for n, _ in seqs)
    if c["kind"] == "append":
        # q, k, v read and written; the positions' angles once each
        places = len({p for n, L in seqs for p in range(L - n, L)})
        return {"bytes": 2 * T * (Hq + 2 * Hk) * D * e + min(T, places) * c["rot"] * 4 + T * c["axes"] * 4,
                "flops": 3 * T * (Hq + Hk) * c["rot"]}
    cuts, prefix = _groups(c)
    keys = sum(L for _, L in seqs) + sum(prefix)
    pairs = 0
    for i, (n, L) in enumerate(seqs):
        P = next((p for g, p in enumerate(prefix) if cuts[g] <= i < cuts[g + 1]), 0)
        pairs += n * (P + L) - (0 if c["full"] else n * (n - 1) // 2)
    return {"bytes": 2 * keys * Hk * D * e + 2 * T * Hq * D * e + 4 * T * Hq, "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------- the outputs in 64 bits

def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return {"positions": _exact_positions, "append": _exact_append, "attend": _exact_attend}[c["kind"]](s, c)


def _exact_positions(s, c):
    """Row by row from the definition: a sequence's kept tokens, then its text."""
    pos = torch.zeros(s.pos.shape, dtype=torch.int64)
    vis, txt, idx = s.vis_pos.cpu(), s.text_pos.cpu(), s.kept_idx.cpu()
    io, to, ko = s.img_off.tolist(), s.text_off.tolist(), s.kept_off.tolist()
    at = 0
    for b in range(c["images"]):
        if s.per_image:
            at = b * s.per_image
        src = [vis[:, io[b] + int(idx[j])] for j in range(ko[b], ko[b] + s.kept[b])]
        src += [txt[:, t] for t in range(to[b], to[b + 1])]
        pos[:, at:at + len(src)] = torch.stack(src, 1)
        at += len(src)
    return {"pos": pos.cuda()}


def _exact_append(s, c):
    """Each pair as the complex number it is, turned by cos + i sin."""
    Hq, Hk, D, page, rot = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"], c["rot"]
    q = torch.zeros(s.T, Hq, D, dtype=torch.float64, device="cuda")
    k_cache, v_cache = s.k_cache.double(), s.v_cache.double()
    turn = torch.view_as_complex(s.cos_sin.double().contiguous())                # [positions, pairs]
    if c["pairs"] == "interleaved":
        re = torch.arange(0, rot, 2, device="cuda")
        im = re + 1
    else:
        re = torch.arange(0, rot // 2, device="cuda")
        im = re + rot // 2
    for i, (n, L) in enumerate(seqs_of(s)):
        rows = torch.arange(s.first[i], s.first[i] + n, device="cuda")
        slots = torch.arange(L - n, L, device="cuda")
        parts, p0 = [], 0
        for a, w in enumerate(s.sections):
            at = s.pos[a, rows].long() if c["axes"] else slots
            parts.append(turn[at, p0:p0 + w])
            p0 += w
        z = torch.cat(parts, 1)[:, None]                                          # [n, 1, pairs]

        def turned(x, H):
            y = x[rows].double().view(n, H, D).clone()
            w = torch.complex(y[..., re], y[..., im]) * z
            y[..., re], y[..., im] = w.real, w.imag
            return y

        q[rows] = turned(s.q, Hq)
        pg, sl = s.tables[i].long()[slots // page], slots % page
        k_cache[pg, :, sl] = turned(s.k, Hk)
        v_cache[pg, :, sl] = s.v[rows].double().view(n, Hk, D)
    return {"q": q.view(s.T, Hq * D), "k_cache": k_cache, "v_cache": v_cache}


def _exact_attend(s, c):
    """Head by head: softmax over the keys that a row sees, in blocks of rows."""
    Hq, Hk, D, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    o = torch.zeros(s.T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.T, Hq, dtype=torch.float64, device="cuda")
    for i, (n, L) in enumerate(seqs_of(s)):
        j = torch.arange(L, device="cuda")
        pages, slots, P = s.tables[i].long()[j // page], j % page, 0
        for g in range(len(s.prefix)):
            if s.cuts[g] <= i < s.cuts[g + 1]:
                P = s.prefix[g]
                j = torch.arange(P, device="cuda")
                pages = torch.cat([s.prefix_tables[g].long()[j // page], pages])
                slots = torch.cat([j % page, slots])
        for h in range(Hk):
            k = s.k_cache[pages, h, slots].double()
            v = s.v_cache[pages, h, slots].double()
            kt = k.t().contiguous()
            heads = slice(h * (Hq // Hk), (h + 1) * (Hq // Hk))
            for a in range(0, n, 512):
                e = min(n, a + 512)
                rows = slice(s.first[i] + a, s.first[i] + e)
                q = s.q[rows].double().view(e - a, Hq, D)[:, heads].reshape(-1, D)
                sc = (q @ kt * s.scale).view(e - a, -1, P + L)
                if not c["full"]:
                    sees = P + L - n + 1 + torch.arange(a, e, device="cuda")      # keys of each row
                    hide = torch.arange(P + L, device="cuda")[None] >= sees[:, None]
                    sc.masked_fill_(hide[:, None], -math.inf)
                z = torch.logsumexp(sc, -1)
                w = torch.exp(sc - z[..., None]).view(-1, P + L)
                o[rows, heads] = (w @ v).view(e - a, -1, D)
                lse[rows, heads] = z
    return {"o": o.view(s.T, Hq * D), "lse": lse}
