"""The rotation, append and 8-bit cache operators, as they are measured.

Four kinds of pass:

* ``rope``: rotary positions of a chunk's queries and keys (``rope_apply``),
  one axis or several, the first ``rot`` channels of each head;
* ``append``: one token of every sequence, its key rotated on the way into a
  paged cache and its query rotated beside it (``append_rope``);
* ``decode``: one layer's decode attention over an int8 cache, whose rows
  each carry a scale of their own (``decode_attn``);
* ``chunk``: prefill attention of one chunk over an int8 cache, and the cast
  of its output to the model's type (``prefill_attn``).

``run`` computes each in plain torch, or through the framework where ``own``
is true.  Keys, values and queries are seeded unit normals rounded to bf16,
with two outlier channels per KV head scaled by 8 where the case says so.
"""
import math
import random

import torch

own = False
DEV = "cuda"
PAGE = 256                      # token rows per page of a full unit
APPEND_CTX = 65536              # rows that a full unit of an append case may reach


def _rope(name, **kw):
    c = dict(name=name, kind="rope", n=512, hq=32, hkv=8, d=128, rot=128, sections="64", interleaved=False,
             pairing="half", theta=10000.0, far=4096, in_place=False)
    c.update(kw)
    return c


def _append(name, **kw):
    c = dict(name=name, kind="append", batch=1, g=6, hkv=4, d=256, rot=64, sections="11,11,10", interleaved=True,
             pairing="half", theta=1e7, far=114688, window=2048, full=1, sinks=4, fmt="bf16")
    c.update(kw)
    return c


def _decode(name, **kw):
    c = dict(name=name, kind="decode", batch=1, d=128, g=4, hkv=8, sinks=4, windows="", full=True, lo=1024, hi=1024,
             paged=False, outliers=False, pick=1)
    c.update(kw)
    return c


def _chunk(name, **kw):
    c = dict(name=name, kind="chunk", d=128, g=4, hkv=8, sinks=4, windows="", full=True, p0=0, n=512, paged=False,
             outliers=False, pick=1)
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token of a video model: three axes dealt out channel by
        # channel over a quarter of each head; latency
        _rope("rope_token", n=1, hq=24, hkv=4, d=256, rot=64, sections="11,11,10", interleaved=True, theta=1e7,
              far=131072),
        # an image's odd number of patches in a small model: height and width
        # in blocks of the head, adjacent channels paired, in place
        _rope("rope_image", n=2901, hq=8, hkv=2, d=64, rot=64, sections="16,16", pairing="pairs", far=64,
              in_place=True),
        # a long prompt in one piece, the whole head rotated, far positions
        _rope("rope_prompt", n=32768, hq=32, hkv=8, d=128, theta=500000.0, far=131072),
        # interactive decoding: one sequence, one full unit and three windows
        _append("append_one"),
        # a serving batch, half of the units full and paged
        _append("append_batch", batch=96, g=4, hkv=8, d=128, rot=128, sections="64", interleaved=False, theta=500000.0,
                window=1024, full=2),
        # a short chat turn in a small model: launches and latency
        _decode("decode_short", d=64, g=4, hkv=2, windows="256", lo=700, hi=700),
        # one sequence at 112K of context, per-head windows {2K, 8K, 32K, full}
        _decode("decode_112k", d=256, g=6, hkv=4, windows="2048,8192,32768", lo=114688, hi=114688, pick=0),
        # batched serving: 16 ragged sequences of 16K-64K, paged full units
        _decode("decode_batch16", batch=16, d=256, g=6, hkv=4, windows="1024,4096,16384", lo=16384, hi=65536,
                paged=True, pick=0),
        # a busy chat server: many short ragged sequences
        _decode("decode_batch48", batch=48, windows="512,1500", lo=200, hi=6000, paged=True, outliers=True),
        # the rest of a chat prompt, few tokens over few keys
        _chunk("chunk_77", d=64, g=1, hkv=8, windows="256", p0=1001, n=77),
        # chunked prefill beside decoding: a small chunk far into a long context
        _chunk("chunk_512", windows="2048,8192", p0=49152, n=512, paged=True),
        # a ragged chunk with grouped wide heads
        _chunk("chunk_2k", d=256, g=6, hkv=4, windows="1024,4096,16384", p0=30011, n=1999, outliers=True, pick=0),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _windows(rng, top):
    return ",".join(str(w) for w in sorted({_logint(rng, 64, max(65, top)) for _ in range(rng.randint(0, 3))}))


def _rotation(rng, d):
    """rot, sections, interleaved, pairing, theta of a drawn rotation."""
    rot = rng.choice([d, d, d // 2, d // 4])
    half = rot // 2
    axes = rng.choice([1, 1, 2, 3, 4])
    cuts = sorted(rng.sample(range(1, half), axes - 1))
    parts = [b - a for a, b in zip([0] + cuts, cuts + [half])]
    return dict(rot=rot, sections=",".join(map(str, parts)), interleaved=axes > 1 and rng.random() < 0.5,
                pairing=rng.choice(["half", "half", "pairs"]), theta=rng.choice([1e4, 5e5, 1e7]))


def draw(rng):
    """One more case; sizes over the whole range of the listed ones."""
    kind = rng.choice(["rope", "append", "decode", "decode", "chunk"])
    while True:
        d = rng.choice([64, 128, 128, 256])
        c = dict(kind=kind, d=d, hkv=rng.randint(1, 8))
        g = rng.choice([1, 2, 4, 6, 8])
        if kind == "rope":
            c.update(_rotation(rng, d), hq=c["hkv"] * g, n=_logint(rng, 1, 32768), far=_logint(rng, 64, 1 << 20),
                     in_place=rng.random() < 0.3)
        elif kind == "append":
            c.update(_rotation(rng, d), g=g, batch=_logint(rng, 1, 96), far=_logint(rng, 64, 1 << 20),
                     window=_logint(rng, 64, 4096), full=rng.randint(0, min(2, c["hkv"])),
                     sinks=rng.choice([0, 1, 4, 16]), fmt=rng.choice(["bf16", "bf16", "f16"]))
        else:
            c.update(g=g, sinks=rng.choice([0, 1, 4, 4, 16]), paged=rng.random() < 0.5, full=rng.random() < 0.7,
                     outliers=rng.random() < 0.3, pick=rng.randint(1, 1 << 20))
            if kind == "decode":
                hi = _logint(rng, 1, 120000)
                c.update(batch=_logint(rng, 1, 64), lo=max(1, hi // rng.randint(1, 8)), hi=hi, windows=_windows(rng, hi))
            else:
                c.update(p0=rng.choice([0, _logint(rng, 1, 50000), _logint(rng, 1, 50000)]), n=_logint(rng, 1, 2048))
                c["windows"] = _windows(rng, c["p0"] + c["n"])
            if not c["full"] and not c["windows"]:
                c["full"] = True
        w = work(c)
        most = {"rope": 6.8e8, "append": 1e9, "decode": 6e8, "chunk": 4e8}[kind]
        # (the plain form holds a padded batch, and a chunk's logits, whole)
        wide = (c["batch"] * c["hkv"] * c["hi"] * d if kind == "decode" else
                c["hkv"] * c["g"] * c["n"] * (c["p0"] + c["n"]) * 4 if kind == "chunk" else
                c["batch"] * c["full"] * APPEND_CTX * d * 4 if kind == "append" else 0)
        if w["bytes"] <= most and w["flops"] <= 5.5e11 and wide <= 6.5e9:
            return c


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
def _codebook(c):
    w = [int(x) for x in c["windows"].split(",") if x]
    return w + [0] if c["full"] or not w else w


def _levels(c):
    """Level of each KV head: head h at level h (pick 0), else drawn."""
    k = len(_codebook(c))
    flat = [h % k for h in range(c["hkv"])]
    if c["pick"]:
        random.Random(c["pick"]).shuffle(flat)
    return flat


def _lengths(c):
    r = random.Random(c["pick"] + 17)
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]


def _max_ctx(c):
    return c["hi"] + 1 if c["kind"] == "decode" else c["p0"] + c["n"]


def _held(c, w, n):
    """Positions that a unit of window w (0 = full) holds at length n."""
    return n if w == 0 or c["sinks"] + w >= _max_ctx(c) else min(n, c["sinks"] + w)


def work(c):
    d, hkv = c["d"], c["hkv"]
    if c["kind"] == "rope":
        rows = c["n"] * (c["hq"] + hkv)
        axes = len(c["sections"].split(","))
        return {"bytes": rows * d * 4.0 + c["n"] * axes * 4.0, "flops": rows * c["rot"] * 3.0}
    g = c["g"]
    if c["kind"] == "append":
        b = c["batch"]
        axes = len(c["sections"].split(","))
        # q and k read and written, v copied
        return {"bytes": b * hkv * d * (4.0 * g + 4 + 4) + b * axes * 4.0, "flops": b * hkv * (g + 1) * c["rot"] * 3.0}
    cb = _codebook(c)
    if c["kind"] == "decode":
        rows = sum(_held(c, cb[k], n) for k in _levels(c) for n in _lengths(c))
        return {"bytes": rows * 2.0 * (d + 1) + c["batch"] * hkv * g * d * 6.0, "flops": rows * g * d * 4.0}
    p0, n = c["p0"], c["n"]
    keys = sum(min(p0, _held(c, cb[k], p0 + 1)) for k in _levels(c))
    pairs = sum(_held(c, cb[k], t + 1) for k in _levels(c) for t in range(p0, p0 + n))
    return {"bytes": keys * 2.0 * (d + 1) + n * hkv * d * (4.0 + 4.0 * g), "flops": 4.0 * d * g * pairs}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Inputs:
    """Seeded inputs, drawn in a fixed order."""

    def __init__(self, c, seed):
        self.c = c
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed((int(seed) * 1000003 + 777) % (1 << 62))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=DEV).to(torch.bfloat16)

    def kv(self, n):
        """K and V of n tokens, [n, hkv, d]."""
        out = []
        for _ in range(2):
            x = torch.randn((n, self.c["hkv"], self.c["d"]), generator=self.gen, device=DEV)
            if self.c.get("outliers"):
                x[:, :, 3] *= 8.0
                x[:, :, self.c["d"] - 10] *= 8.0
            out.append(x.to(torch.bfloat16))
        return out

    def positions(self, axes, n):
        """Positions below ``far`` on each axis, int32 [axes, n]: consecutive
        ones on the first, as text has them, any on the others."""
        far = self.c["far"]
        pos = torch.randint(0, far, (axes, n), generator=self.gen, device=DEV, dtype=torch.int32)
        pos[0] = (pos[0, 0] + torch.arange(n, device=DEV, dtype=torch.int32)) % far
        return pos


def _frequencies(c):
    """Frequency and axis of each rotated pair: theta^(-2 i / rot); the axes
    take their sections in blocks, or (interleaved) pair i goes to axis
    i mod axes while that axis has pairs left, else to axis 0."""
    half = c["rot"] // 2
    sections = [int(x) for x in c["sections"].split(",")]
    freq = [c["theta"] ** (-2.0 * i / c["rot"]) for i in range(half)]
    if c["interleaved"]:
        axis = [i % len(sections) if i // len(sections) < sections[i % len(sections)] else 0 for i in range(half)]
    else:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    return freq, axis


def _quantise(x):
    """int8 codes and scale exponents of bf16 rows x [..., d]: the row's
    largest magnitude lies in [2^(e-127), 2^(e-126)), and a code counts
    2^(e-133)."""
    top = x.float().abs().amax(dim=-1)
    e = ((top.view(torch.int32) >> 23) & 255).clamp(min=1)
    step = torch.exp2((133 - e).double())[..., None]
    codes = torch.round(x.double() * step).clamp(-127, 127).to(torch.int8)
    return codes, e.to(torch.uint8)


def _values(codes, e, dtype):
    """What the codes stand for."""
    return codes.to(dtype) * torch.exp2(e.to(dtype) - 133.0)[..., None]


def _policy_cache(c, batch, fmt, **kw):
    from paper_2609_02029_amd import hwkv
    pol = hwkv.policy_set(1, c["hkv"], c["hkv"] * c["g"], c["d"], c["sinks"], _codebook(c), [_levels(c)])
    pages = None
    if c["paged"]:
        full = sum(1 for k in _levels(c) if _held(c, _codebook(c)[k], _max_ctx(c)) == _max_ctx(c))
        lens = _lengths(c) if c["kind"] == "decode" else [_max_ctx(c)]
        pages = full * sum(-(-n // PAGE) for n in lens)
    return hwkv.cache_alloc(pol, batch, _max_ctx(c), kv_format=fmt, n_pages=pages)


def prepare(c, seed):
    x = _Inputs(c, seed)
    s = {"c": c}
    if c["kind"] in ("rope", "append"):
        freq, axis = _frequencies(c)
        axes = len(c["sections"].split(","))
        n = c["n"] if c["kind"] == "rope" else c["batch"]
        hq = c["hq"] if c["kind"] == "rope" else c["hkv"] * c["g"]
        s["pos"] = x.positions(axes, n)
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device=DEV)
        s["axis"] = torch.tensor(axis, dtype=torch.int64, device=DEV)
        # q, k and v as a fused projection leaves them: slices of one row
        qkv = x.normal(n, hq + 2 * c["hkv"], c["d"])
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + c["hkv"]], qkv[:, hq + c["hkv"]:]
        if own:
            from paper_2609_02029_amd import hwkv
            s["rope"] = hwkv.rope_set(c["d"], freq, axis, n_axes=axes, pairing=c["pairing"])
        s["q_out"] = torch.empty((n, hq, c["d"]), dtype=torch.bfloat16, device=DEV)
        if c["kind"] == "rope":
            s["k_out"] = torch.empty((n, c["hkv"], c["d"]), dtype=torch.bfloat16, device=DEV)
            if c["in_place"]:
                # a pass turns what the pass before it left
                s["q_out"].copy_(s["q"])
                s["k_out"].copy_(s["k"])
                s["q"], s["k"] = s["q_out"], s["k_out"]
        else:
            _append_state(s)
        return s
    s["scale"] = 1.0 / math.sqrt(c["d"])
    if c["kind"] == "decode":
        hist = [x.kv(n) for n in _lengths(c)]
        s["q"] = x.normal(c["batch"], c["hkv"] * c["g"], c["d"])
        if own:
            from paper_2609_02029_amd import hwkv
            s["cache"] = _policy_cache(c, c["batch"], "i8")
            for b, (k, v) in enumerate(hist):
                hwkv.prefill_write(s["cache"], 0, b, 0, k, v)
            s["out"] = torch.empty(s["q"].shape, device=DEV)
            s["ws"] = torch.empty(max(1, hwkv.decode_workspace_bytes(s["cache"])), dtype=torch.uint8, device=DEV)
        else:
            _padded(s, hist)
        return s
    k0, v0 = x.kv(c["p0"])
    s["k"], s["v"] = x.kv(c["n"])
    s["q"] = x.normal(c["n"], c["hkv"] * c["g"], c["d"])
    if own:
        from paper_2609_02029_amd import hwkv
        s["cache"] = cache = _policy_cache(c, 1, "i8")
        if c["p0"]:
            hwkv.prefill_write(cache, 0, 0, 0, k0, v0)
        s["out"] = torch.empty(s["q"].shape, device=DEV)
        s["ws"] = torch.empty(max(1, hwkv.prefill_attn_workspace_bytes(cache, c["n"])), dtype=torch.uint8, device=DEV)
    else:
        s["kc"], s["ke"] = _quantise(k0)
        s["vc"], s["ve"] = _quantise(v0)
    return s


def _resident(c, w, n):
    """Positions that a unit of window w holds at length n."""
    if _held(c, w, n) == n:
        return torch.arange(n, device=DEV)
    return torch.cat([torch.arange(c["sinks"], device=DEV), torch.arange(n - w, n, device=DEV)])


def _padded(s, hist):
    """The resident rows of every (sequence, KV head), padded to the longest:
    codes [items, rows, d], exponents [items, rows], row counts [items]."""
    c = s["c"]
    cb, lv = _codebook(c), _levels(c)
    at = [[_resident(c, cb[lv[h]], n) for h in range(c["hkv"])] for n in _lengths(c)]
    most = max(len(p) for row in at for p in row)
    items = c["batch"] * c["hkv"]
    s["count"] = torch.tensor([len(p) for row in at for p in row], device=DEV)
    for name, side in (("k", 0), ("v", 1)):
        codes = torch.zeros((items, most, c["d"]), dtype=torch.int8, device=DEV)
        e = torch.ones((items, most), dtype=torch.uint8, device=DEV)
        for b, row in enumerate(at):
            for h, p in enumerate(row):
                codes[b * c["hkv"] + h, :len(p)], e[b * c["hkv"] + h, :len(p)] = _quantise(hist[b][side][p, h])
        s[name + "c"], s[name + "e"] = codes, e


def _append_shape(c):
    """(full heads, their count, window heads, their count, rows of a window
    region): the last heads are full."""
    nw = c["hkv"] - c["full"]
    cap = c["sinks"] + c["window"]
    return list(range(nw, c["hkv"])), c["full"], list(range(nw)), nw, (cap + 63) // 64 * 64


def _append_state(s):
    """An empty paged cache over a buffer of the program's own, and views of
    the two parts that hold rows: the windows' regions and the pool."""
    c = s["c"]
    _, nf, _, nw, pad = _append_shape(c)
    d, b = c["d"], c["batch"]
    regions = nw * b * pad * d * 2 * 2
    pool_at = -(-regions // 256) * 256
    pages = nf * b * (APPEND_CTX // PAGE)
    pool = pages * 2 * PAGE * d * 2
    table = nf * b * (APPEND_CTX // PAGE) * 4
    buf = torch.zeros(-(-(pool_at + pool) // 256) * 256 + table, dtype=torch.uint8, device=DEV)
    t = torch.bfloat16 if c["fmt"] == "bf16" else torch.float16
    s["windows"], s["pool"] = buf[:regions].view(t), buf[pool_at:pool_at + pool].view(t)
    s["n"] = 0
    if own:
        from paper_2609_02029_amd import hwkv
        pol = hwkv.policy_set(1, c["hkv"], c["hkv"] * c["g"], d, c["sinks"], [c["window"], 0],
                              [[0] * nw + [1] * nf])
        s["cache"] = hwkv.cache_alloc(pol, b, APPEND_CTX, dev_buf=buf, kv_format=c["fmt"], n_pages=pages)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _turn(x, cos, sin, rot, pairing):
    """The first rot channels of x [n, heads, d] turned, [n, 1, rot / 2]
    cosines and sines; the rest as they are."""
    if pairing == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _rope_plain(s, parts):
    c = s["c"]
    angle = s["pos"][s["axis"]].double() * s["freq"][:, None]          # [rot / 2, n]
    cos, sin = angle.cos().float().T[:, None], angle.sin().float().T[:, None]
    return [_turn(x.float(), cos, sin, c["rot"], c["pairing"]).to(torch.bfloat16) for x in parts]


def _store(s, k, v):
    """Rows k, v [batch, hkv, d] of position n into the cache's layout: K in
    tiles of 64 rows, [d / 8][64][8]; V row by row; a window's rows as a ring
    behind its sinks; a full unit's in pages of 256 rows taken in order."""
    c = s["c"]
    full, nf, win, nw, pad = _append_shape(c)
    d, b, n = c["d"], c["batch"], s["n"]
    seq = torch.arange(b, device=DEV)[:, None]
    ch = torch.arange(d, device=DEV)
    if nw:
        slot = n if n < c["sinks"] else c["sinks"] + (n - c["sinks"]) % c["window"]
        base = (torch.arange(nw, device=DEV)[None, :] * b + seq) * pad * d
        at = base[..., None] + slot // 64 * 64 * d + ch // 8 * 512 + slot % 64 * 8 + ch % 8
        s["windows"][at.reshape(-1)] = k[:, win].reshape(-1).to(s["windows"].dtype)
        at = nw * b * pad * d + base[..., None] + slot * d + ch
        s["windows"][at.reshape(-1)] = v[:, win].reshape(-1).to(s["windows"].dtype)
    if nf:
        r = n % PAGE
        base = (n // PAGE * b * nf + seq * nf + torch.arange(nf, device=DEV)[None, :]) * 2 * PAGE * d
        at = base[..., None] + r // 64 * 64 * d + ch // 8 * 512 + r % 64 * 8 + ch % 8
        s["pool"][at.reshape(-1)] = k[:, full].reshape(-1).to(s["pool"].dtype)
        at = base[..., None] + PAGE * d + r * d + ch
        s["pool"][at.reshape(-1)] = v[:, full].reshape(-1).to(s["pool"].dtype)


def _decode_plain(s):
    c = s["c"]
    items, g, d = c["batch"] * c["hkv"], c["g"], c["d"]
    q = s["q"].float().reshape(items, g, d)
    z = (q @ _values(s["kc"], s["ke"], torch.float32).transpose(1, 2)) * s["scale"]
    seen = torch.arange(z.shape[2], device=DEV) < s["count"][:, None]
    z = z.masked_fill(~seen[:, None], -math.inf)
    p = torch.exp(z - z.amax(dim=2, keepdim=True))
    out = (p @ _values(s["vc"], s["ve"], torch.float32)) / p.sum(dim=2, keepdim=True)
    return out.reshape(c["batch"], c["hkv"] * g, d)


def _seen(c):
    """[hkv, n, p0 + n]: whether the chunk's token sees the key."""
    cb = _codebook(c)
    top = _max_ctx(c)
    w = torch.tensor([top if _held(c, cb[k], top) == top else cb[k] for k in _levels(c)], device=DEV)[:, None, None]
    t = (c["p0"] + torch.arange(c["n"], device=DEV))[None, :, None]
    key = torch.arange(top, device=DEV)[None, None, :]
    return (key <= t) & ((key < c["sinks"]) | (key > t - w))


def _chunk_plain(s):
    c = s["c"]
    n, hkv, g, d = c["n"], c["hkv"], c["g"], c["d"]
    (kc, ke), (vc, ve) = _quantise(s["k"]), _quantise(s["v"])
    k = _values(torch.cat([s["kc"], kc]), torch.cat([s["ke"], ke]), torch.float32).permute(1, 2, 0).contiguous()
    v = _values(torch.cat([s["vc"], vc]), torch.cat([s["ve"], ve]), torch.float32).permute(1, 0, 2).contiguous()
    q = s["q"].float().reshape(n, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, n * g, d)
    z = ((q @ k) * s["scale"]).reshape(hkv, n, g, -1)
    z.masked_fill_(~_seen(c)[:, :, None], -math.inf)
    p = z.sub_(z.amax(dim=3, keepdim=True)).exp_()
    out = (p.reshape(hkv, n * g, -1) @ v).reshape(hkv, n, g, d) / p.sum(dim=3, keepdim=True)
    return out.permute(1, 0, 2, 3).reshape(n, hkv * g, d).to(torch.bfloat16)


def run(s):
    c = s["c"]
    if own:
        from paper_2609_02029_amd import hwkv
        if c["kind"] == "rope":
            hwkv.rope_apply(s["rope"], s["pos"], s["q"], s["k"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if c["kind"] == "append":
            hwkv.append_rope(s["cache"], 0, s["rope"], s["pos"], s["k"], s["v"], s["q"], s["q_out"])
            return {"q": s["q_out"], "windows": s["windows"], "pool": s["pool"]}
        if c["kind"] == "decode":
            hwkv.decode_attn(s["cache"], 0, s["q"], s["scale"], s["out"], s["ws"])
            return s["out"]
        hwkv.prefill_attn(s["cache"], 0, 0, c["p0"], s["q"], s["k"], s["v"], s["scale"], s["out"], ws=s["ws"])
        return s["out"].to(torch.bfloat16)
    if c["kind"] == "rope":
        q, k = _rope_plain(s, (s["q"], s["k"]))
        if c["in_place"]:
            q, k = s["q_out"].copy_(q), s["k_out"].copy_(k)
        return {"q": q, "k": k}
    if c["kind"] == "append":
        q, k = _rope_plain(s, (s["q"], s["k"]))
        _store(s, k, s["v"])
        s["n"] += 1
        return {"q": q, "windows": s["windows"], "pool": s["pool"]}
    return _decode_plain(s) if c["kind"] == "decode" else _chunk_plain(s)


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_rows(x):
    """bf16 rows as an int8 cache holds them, in 64 bits."""
    x = x.double()
    top = x.abs().amax(dim=-1, keepdim=True).clamp(min=2.0 ** -126)
    unit = torch.exp2(torch.frexp(top)[1].double() - 1.0)     # 2^floor(log2 top)
    return torch.round(x / unit * 64.0).clamp(-127.0, 127.0) / 64.0 * unit


def _exact_turn(c, x, pos, freq, axis):
    out = x.double().clone()
    for i in range(c["rot"] // 2):
        a = pos[axis[i]].double() * freq[i]
        lo, hi = (i, i + c["rot"] // 2) if c["pairing"] == "half" else (2 * i, 2 * i + 1)
        u, v = x[..., lo].double(), x[..., hi].double()
        out[..., lo] = u * a.cos()[:, None] - v * a.sin()[:, None]
        out[..., hi] = v * a.cos()[:, None] + u * a.sin()[:, None]
    return out


def _exact_attend(q, k, v, seen, scale):
    """q [m, d] over k, v [n, d], seen [m, n] or None."""
    z = (q @ k.T) * scale
    if seen is not None:
        z.masked_fill_(~seen, -math.inf)
    return torch.softmax(z, dim=1) @ v


def exact(c, seed):
    x = _Inputs(c, seed)
    if c["kind"] in ("rope", "append"):
        freq, axis = _frequencies(c)
        rope = c["kind"] == "rope"
        n, hq = (c["n"], c["hq"]) if rope else (c["batch"], c["hkv"] * c["g"])
        pos = x.positions(len(c["sections"].split(",")), n)
        qkv = x.normal(n, hq + 2 * c["hkv"], c["d"])
        q = _exact_turn(c, qkv[:, :hq], pos, freq, axis)
        if not rope:        # (the cache's own layout has no other definition)
            return {"q": q, "windows": None, "pool": None}
        return {"q": q, "k": _exact_turn(c, qkv[:, hq:hq + c["hkv"]], pos, freq, axis)}
    scale, g, cb, lv = 1.0 / math.sqrt(c["d"]), c["g"], _codebook(c), _levels(c)
    if c["kind"] == "decode":
        hist = [x.kv(n) for n in _lengths(c)]
        q = x.normal(c["batch"], c["hkv"] * g, c["d"]).double()
        out = torch.empty_like(q)
        for b, n in enumerate(_lengths(c)):
            for h in range(c["hkv"]):
                at = _resident(c, cb[lv[h]], n)
                k, v = (_exact_rows(t[at, h]) for t in hist[b])
                out[b, h * g:(h + 1) * g] = _exact_attend(q[b, h * g:(h + 1) * g], k, v, None, scale)
        return out
    (k0, v0), (k1, v1) = x.kv(c["p0"]), x.kv(c["n"])
    q = x.normal(c["n"], c["hkv"] * g, c["d"]).double()
    out = torch.empty_like(q)
    k, v = _exact_rows(torch.cat([k0, k1])), _exact_rows(torch.cat([v0, v1]))
    seen = _seen(c)
    for h in range(c["hkv"]):
        for i in range(0, c["n"], 256):
            part = q[i:i + 256, h * g:(h + 1) * g].reshape(-1, c["d"])
            o = _exact_attend(part, k[:, h], v[:, h], seen[h, i:i + 256].repeat_interleave(g, dim=0), scale)
            out[i:i + 256, h * g:(h + 1) * g] = o.reshape(-1, g, c["d"])
    return out
