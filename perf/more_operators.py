"""The operators of several continuations over one cache, as they are measured.

Four kinds of pass:

* ``select``: beam search's choice, over beams and vocabulary (``beam_select``);
* ``reorder``: every sequence of a paged cache becomes what its parent was
  (``cache_reorder``): forked, kept, moved or dropped;
* ``move``: a cache with holes in its pool goes into another buffer, its pages
  in order (``cache_move``);
* ``shared``: one layer's decode attention of sequences that were forked from
  one prompt and have their own last tokens (``decode_attn_shared``).

``run`` computes each in plain torch, or through the framework where ``own``
is true.  Logits are seeded normals of deviation 2.5 with a few high ones in
each row; keys, values and queries are unit normals rounded to bf16.
"""
import math
import random

import torch

own = False
DEV = "cuda"
PAGE = 256                      # token rows per page of a full unit
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _select(name, **kw):
    c = dict(name=name, kind="select", groups=1, beams=4, vocab=32000, n_out=8, dtype="bf16", first=False, allowed=1.0)
    c.update(kw)
    return c


def _reorder(name, **kw):
    c = dict(name=name, kind="reorder", layers=1, d=64, hkv=2, full=1, window=256, sinks=4, groups=1, beams=4, lo=700,
             hi=700, keep=0.3, fmt="bf16", pick=1)
    c.update(kw)
    return c


def _move(name, **kw):
    c = dict(name=name, kind="move", layers=1, d=64, hkv=2, full=1, window=256, sinks=4, groups=6, beams=1, lo=700,
             hi=700, fmt="bf16", pick=1)
    c.update(kw)
    return c


def _shared(name, **kw):
    c = dict(name=name, kind="shared", d=128, g=4, hkv=8, sinks=4, windows="", full=True, groups=1, beams=4, lo=1024,
             hi=1024, tail=64, fmt="bf16", pick=1)
    c.update(kw)
    return c


def listed():
    return [
        # one user's beam search with a small vocabulary: launches and latency
        _select("select_one"),
        # the first step of three requests (one beam alive each) under a
        # grammar that allows one token in fifty; an odd vocabulary
        _select("select_odd", groups=3, beams=5, vocab=50257, n_out=10, dtype="f16", first=True, allowed=0.02),
        # a translation service: many requests of four beams
        _select("select_batch", groups=24, vocab=131072),
        # offline generation, wide beams, fp32 logits
        _select("select_wide", groups=64, beams=8, vocab=131072, n_out=16, dtype="f32"),
        # a short chat turn with four beams in a small model: latency
        _reorder("reorder_short"),
        # one request of four beams in a deep model with wide heads, at 9K
        _reorder("reorder_beams", layers=16, d=256, hkv=4, window=2048, lo=9001, hi=9001),
        # a batch of beam searches of unequal lengths
        _reorder("reorder_batch", layers=8, d=128, hkv=8, full=2, window=1024, groups=8, lo=1500, hi=6000),
        # a small cache gets a larger pool
        _move("move_small"),
        # a serving cache after every second request has left: compaction
        _move("move_batch", layers=8, d=128, hkv=8, full=2, window=1024, groups=24, lo=1500, hi=12000),
        # two samples of a short prompt in a small model: latency
        _shared("shared_short", d=64, hkv=2, windows="256", beams=2, lo=700, hi=700, tail=9),
        # eight samples of one 112K prompt, per-head windows {2K, 8K, 32K, full}
        _shared("shared_112k", d=256, g=6, hkv=4, windows="2048,8192,32768", beams=8, lo=114688, hi=114688, tail=300,
                pick=0),
        # a batch of beam searches over ragged prompts, half of the heads full
        _shared("shared_batch", windows="1024", groups=8, lo=4000, hi=16384, tail=200, pick=0),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case; sizes over the whole range of the listed ones."""
    kind = rng.choice(["select", "select", "reorder", "move", "shared", "shared"])
    while True:
        c = dict(kind=kind, pick=rng.randint(1, 1 << 20))
        if kind == "select":
            c.update(groups=_logint(rng, 1, 64), beams=rng.choice([1, 2, 3, 4, 4, 5, 8, 16]), vocab=_logint(rng, 1000, 262144),
                     dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), first=rng.random() < 0.2,
                     allowed=rng.choice([1.0, 1.0, 0.3, 0.02]))
            c["n_out"] = rng.randint(1, 2 * c["beams"])
        else:
            c.update(d=rng.choice([64, 128, 128, 256]), hkv=rng.randint(1, 8), groups=_logint(rng, 1, 24),
                     beams=rng.randint(1 if kind == "move" else 2, 8), sinks=rng.choice([0, 1, 4, 4, 16]),
                     fmt=rng.choice(["bf16", "f16"]))
            c["hi"] = _logint(rng, 1, 120000 if kind == "shared" else 12000)
            c["lo"] = max(1, c["hi"] // rng.randint(1, 8))
            if kind == "shared":
                c.update(g=rng.choice([1, 2, 4, 6, 8]), tail=_logint(rng, 1, 600), full=rng.random() < 0.8,
                         windows=",".join(str(w) for w in sorted({_logint(rng, 64, max(65, c["hi"]))
                                                                  for _ in range(rng.randint(0, 3))})))
                c["full"] = c["full"] or not c["windows"]
            else:
                c.update(layers=_logint(rng, 1, 16), window=_logint(rng, 64, 4096), full=rng.randint(0, min(2, c["hkv"])))
                if kind == "reorder":
                    c["keep"] = rng.choice([0.0, 0.3, 0.7])
        w = work(c)
        held = 0
        if kind in ("reorder", "move"):
            held = sum(_region(c) * (c["hkv"] - c["full"]) + -(-n // PAGE) * PAGE * c["full"] for n in _lengths(c)
                       ) * c["layers"] * c["d"] * 4
        elif kind == "shared":      # (the plain form holds a padded batch)
            held = c["groups"] * c["beams"] * c["hkv"] * (c["hi"] + c["tail"]) * c["d"] * 8
        most = {"select": 2.6e8, "reorder": 9e8, "move": 1.2e9, "shared": 3e8}[kind]
        if 0 < w["bytes"] <= most and held <= (9e9 if kind == "shared" else 2e9):
            return c


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
def _lengths(c):
    """Tokens of each sequence: the beams of a group have the group's."""
    r = random.Random(c["pick"] + 17)
    return [n for n in [r.randint(c["lo"], c["hi"]) for _ in range(c["groups"])] for _ in range(c["beams"])]


def _tails(c):
    """A forked sequence's own tokens, behind its prompt."""
    r = random.Random(c["pick"] + 19)
    return [r.randint(1, c["tail"]) for _ in range(c["groups"] * c["beams"])]


def _parents(c):
    """A beam's parent is itself, or any beam of its group."""
    r = random.Random(c["pick"] + 23)
    b = c["beams"]
    got = [s if r.random() < c["keep"] else s // b * b + r.randrange(b) for s in range(c["groups"] * b)]
    if got == list(range(len(got))):     # something moves
        got[0] = b - 1
    return got


def _region(c):
    """Rows of a window's region."""
    return (c["sinks"] + c["window"] + 63) // 64 * 64


def _max_ctx(c):
    """Above every window, so that a window is one."""
    if c["kind"] == "shared":
        return c["hi"] + c["tail"] + 1
    return max(c["hi"], c["sinks"] + c["window"]) + PAGE


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


def _full_at(c, w):
    return w == 0 or c["sinks"] + w >= _max_ctx(c)


def _held(c, w, n):
    """Positions that a unit of window w (0 = full) holds at length n."""
    return n if _full_at(c, w) else min(n, c["sinks"] + w)


def _live(c):
    """Sequences that are left when a cache moves: every second request."""
    return [s for s in range(c["groups"] * c["beams"]) if s // c["beams"] % 2 == 0]


def work(c):
    if c["kind"] == "select":
        rows, size = c["groups"] * c["beams"], 4 if c["dtype"] == "f32" else 2
        # (a 64-bit exponential to 1e-11 and its sum: about a dozen multiply-adds)
        return {"bytes": rows * (c["vocab"] * size + 4.0) + c["groups"] * c["n_out"] * 12.0, "flops": rows * c["vocab"] * 26.0}
    d, row = c["d"], c["d"] * 4.0                     # bytes of a token's K and V
    if c["kind"] in ("reorder", "move"):
        nw, lens = (c["hkv"] - c["full"]) * c["layers"], _lengths(c)
        if c["kind"] == "move":
            rows = sum(nw * min(lens[s], c["sinks"] + c["window"]) + c["full"] * c["layers"] * lens[s] for s in _live(c))
            return {"bytes": 2 * rows * row, "flops": 0.0}
        par, rows = _parents(c), 0
        held = [min(n, c["sinks"] + c["window"]) for n in lens]
        rows += nw * sum(held[p] for p in {p for b, p in enumerate(par) if p != b})       # each source once,
        rows += nw * sum(held[b] for b, p in enumerate(par) if p != b)                    # and who changes
        more = [p for p in set(par) for _ in range(par.count(p) - 1)]                     # further children
        rows += c["full"] * c["layers"] * (sum(lens[p] % PAGE for p in more) + sum(lens[p] % PAGE for p in set(more)))
        return {"bytes": rows * row + len(lens) * 4.0, "flops": 0.0}
    g, cb, lens, tails, rows, pairs = c["g"], _codebook(c), _lengths(c), _tails(c), 0, 0
    for k in _levels(c):
        for s, (n, t) in enumerate(zip(lens, tails)):
            held = _held(c, cb[k], n + t)
            whole = n // PAGE * PAGE if _full_at(c, cb[k]) and s % c["beams"] else 0     # rows of shared pages
            rows += held - whole
            pairs += held
    return {"bytes": rows * row + len(lens) * c["hkv"] * g * d * 6.0, "flops": 4.0 * d * g * pairs}


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
        return [self.normal(n, self.c["hkv"], self.c["d"]) for _ in range(2)]

    def logits(self):
        """[groups, beams, vocab] and the beams' running scores."""
        c = self.c
        x = torch.randn((c["groups"], c["beams"], c["vocab"]), generator=self.gen, device=DEV) * 2.5
        at = torch.randint(0, c["vocab"], (c["groups"], c["beams"], 6), generator=self.gen, device=DEV)
        x.scatter_add_(2, at, torch.rand(at.shape, generator=self.gen, device=DEV) * 9.0)
        if c["allowed"] < 1.0:
            x.masked_fill_(torch.rand(x.shape, generator=self.gen, device=DEV) >= c["allowed"], -math.inf)
        s = -torch.rand((c["groups"], c["beams"]), generator=self.gen, device=DEV) * 20.0
        if c["first"]:
            s[:] = torch.tensor([0.0] + [-math.inf] * (c["beams"] - 1), device=DEV)
        return x.to(TYPES[c["dtype"]]), s


def prepare(c, seed):
    x = _Inputs(c, seed)
    s = {"c": c}
    if c["kind"] == "select":
        s["x"], s["scores"] = x.logits()
        if own:
            from paper_2609_02029_amd import hwkv
            out = (c["groups"], c["n_out"])
            s["out"] = (torch.empty(out, device=DEV), torch.empty(out, dtype=torch.int32, device=DEV),
                        torch.empty(out, dtype=torch.int32, device=DEV))
            s["ws"] = torch.empty(hwkv.beam_workspace_bytes(s["x"], c["n_out"]), dtype=torch.uint8, device=DEV)
    elif c["kind"] == "shared":
        _shared_state(s, x)
    else:
        _stored_state(s, x)
    return s


def _layout(c, batch):
    """(regions of windows, elements of one, element of page 0, pages)"""
    nw = (c["hkv"] - c["full"]) * c["layers"]
    region = _region(c) * c["d"]
    pool_at = -(-(2 * nw * batch * region) // 128) * 128
    pages = c["full"] * c["layers"] * sum(-(-n // PAGE) for n in _lengths(c))
    return nw, region, pool_at, pages


def _buffer(c, batch):
    """A zeroed buffer for the whole cache, and views of its windows' regions
    [K or V, unit, sequence, elements] and of its pages."""
    nw, region, pool_at, pages = _layout(c, batch)
    page = 2 * PAGE * c["d"]
    table = c["full"] * c["layers"] * batch * -(-_max_ctx(c) // PAGE) * 4
    buf = torch.zeros(-(-(pool_at + pages * page) // 128) * 256 + table, dtype=torch.uint8, device=DEV)
    flat = buf[:(pool_at + pages * page) * 2].view(TYPES[c["fmt"]])
    return buf, flat[:2 * nw * batch * region].view(2, nw, batch, region), flat[pool_at:].view(pages, page)


def _ring(c, n):
    """The positions that a window holds at length n, by slot."""
    held = min(n, c["sinks"] + c["window"])
    slot = torch.arange(held, device=DEV)
    last = n - c["window"]          # the ring holds [last, n) where it is full
    return torch.where((slot < c["sinks"]) | (n <= c["sinks"] + c["window"]), slot,
                       last + (slot - c["sinks"] - (last - c["sinks"])) % c["window"])


def _tiles(x, rows):
    """K rows x [n, heads, d] in tiles of 64 rows, [heads, rows / 64, d / 8, 64, 8]
    flattened by head; V rows are the same without the turn."""
    n, h, d = x.shape
    y = torch.zeros((rows, h, d), dtype=x.dtype, device=DEV)
    y[:n] = x
    return y.view(rows // 64, 64, h, d // 8, 8).permute(2, 0, 3, 1, 4).reshape(h, -1), y.permute(1, 0, 2).reshape(h, -1)


def _stored_state(s, x):
    """A cache that holds every sequence, and for the plain form its rows as a
    cache holds them.  The pages of a layer are taken sequence by sequence and
    head by head; a unit's last page is the one that a fork copies."""
    c = s["c"]
    lens, nf, nl = _lengths(c), c["full"], c["layers"]
    batch, nw = len(lens), c["hkv"] - nf
    s["buf"], s["windows"], s["pool"] = _buffer(c, batch)
    cache = None
    if own:
        from paper_2609_02029_amd import hwkv
        pol = hwkv.policy_set(nl, c["hkv"], c["hkv"], c["d"], c["sinks"], [c["window"], 0], [[0] * nw + [1] * nf] * nl)
        cache = s["cache"] = hwkv.cache_alloc(pol, batch, _max_ctx(c), dev_buf=s["buf"], kv_format=c["fmt"],
                                              n_pages=len(s["pool"]))
    first = torch.empty((nl * nf, batch), dtype=torch.int64)      # a unit's first page
    page = 0
    for layer in range(nl):
        for b, n in enumerate(lens):
            k, v = x.kv(n)
            per = -(-n // PAGE)
            first[layer * nf:(layer + 1) * nf, b] = page + torch.arange(nf) * per
            if own:
                hwkv.prefill_write(cache, layer, b, 0, k, v)
            else:
                k, v, at = k.to(TYPES[c["fmt"]]), v.to(TYPES[c["fmt"]]), _ring(c, n)
                unit = slice(layer * nw, (layer + 1) * nw)
                if nw:
                    s["windows"][0, unit, b] = _tiles(k[at, :nw], _region(c))[0]
                    s["windows"][1, unit, b] = _tiles(v[at, :nw], _region(c))[1]
                if nf:
                    rows = s["pool"][page:page + nf * per].view(nf, per, 2, -1)
                    rows[:, :, 0] = _tiles(k[:, nw:], per * PAGE)[0].view(nf, per, -1)
                    rows[:, :, 1] = _tiles(v[:, nw:], per * PAGE)[1].view(nf, per, -1)
            page += nf * per
    if c["kind"] == "reorder":
        s["parents"] = _parents(c)
        if not own:
            _reorder_plan(s, first, lens)
    elif own:
        for b in range(batch):
            if b not in _live(c):
                hwkv.cache_reset_seq(cache, b)
        s["other"] = _buffer(c, batch)
        s["used"] = nf * nl * sum(-(-lens[b] // PAGE) for b in _live(c))
    else:
        s["live"] = torch.tensor(_live(c), device=DEV)
        s["other"] = _buffer(c, batch)
        order = [first[u, b] + torch.arange(-(-lens[b] // PAGE)) for u in range(nl * nf) for b in _live(c)]
        s["order"] = torch.cat(order).to(DEV) if order else torch.zeros(0, dtype=torch.int64, device=DEV)


def _reorder_plan(s, first, lens):
    """Which last pages are copied where.  A parent that is its own child keeps
    its page, else its first child takes it; each further child gets a copy in
    the page of a sequence that has no child, both in order."""
    c, par = s["c"], s["parents"]
    heir = {p: p if par[p] == p else par.index(p) for p in set(par)}
    some = [b for b in range(len(par)) if lens[b] % PAGE]         # who has a partly filled page
    more = [b for b in some if heir[par[b]] != b]
    left = [b for b in some if b not in heir]
    owner = [par[b] for b in range(len(par))]                     # whose page each now has
    for b, o in zip(more, left):
        owner[b] = o
    last = first + torch.tensor([-(-n // PAGE) - 1 for n in lens])
    s["last"] = last.to(DEV)
    s["from"] = torch.tensor([par[b] for b in more], dtype=torch.int64, device=DEV)
    s["into"] = torch.tensor(left, dtype=torch.int64, device=DEV)
    s["owner"] = torch.tensor(owner, device=DEV)
    s["dst"] = torch.tensor([b for b, p in enumerate(par) if p != b], device=DEV)
    s["src"] = torch.tensor([p for b, p in enumerate(par) if p != b], device=DEV)


def _resident(c, w, n):
    """Positions that a unit of window w holds at length n."""
    if _held(c, w, n) == n:
        return torch.arange(n, device=DEV)
    return torch.cat([torch.arange(c["sinks"], device=DEV), torch.arange(n - w, n, device=DEV)])


def _histories(c, x):
    """Each sequence's prompt (one tensor for a group) and own tokens."""
    prompts = [x.kv(n) for n in _lengths(c)[::c["beams"]]]
    return [(prompts[b // c["beams"]], x.kv(t)) for b, t in enumerate(_tails(c))]


def _shared_state(s, x):
    c = s["c"]
    cb, lv, beams = _codebook(c), _levels(c), c["beams"]
    batch = c["groups"] * beams
    s["scale"] = 1.0 / math.sqrt(c["d"])
    hist = _histories(c, x)
    s["q"] = x.normal(batch, c["hkv"] * c["g"], c["d"])
    if own:
        from paper_2609_02029_amd import hwkv
        full = sum(_full_at(c, cb[k]) for k in lv)
        pages = full * (sum(-(-n // PAGE) for n in _lengths(c)[::beams]) + batch * (c["tail"] // PAGE + 2))
        pol = hwkv.policy_set(1, c["hkv"], c["hkv"] * c["g"], c["d"], c["sinks"], cb, [lv])
        cache = s["cache"] = hwkv.cache_alloc(pol, batch, _max_ctx(c), kv_format=c["fmt"], n_pages=pages)
        for b in range(0, batch, beams):
            hwkv.prefill_write(cache, 0, b, 0, *hist[b][0])
        hwkv.cache_reorder(cache, [b // beams * beams for b in range(batch)])
        for b, (prompt, tail) in enumerate(hist):
            hwkv.prefill_write(cache, 0, b, len(prompt[0]), *tail)
        s["out"] = torch.empty(s["q"].shape, device=DEV)
        s["ws"] = torch.empty(max(1, hwkv.decode_shared_workspace_bytes(cache)), dtype=torch.uint8, device=DEV)
        return
    # the resident rows of every (sequence, KV head), padded to the longest
    lens = [n + t for n, t in zip(_lengths(c), _tails(c))]
    s["count"] = torch.tensor([_held(c, cb[k], n) for n in lens for k in lv], device=DEV)
    most = int(s["count"].max())
    s["k"], s["v"] = (torch.zeros((batch * c["hkv"], most, c["d"]), dtype=TYPES[c["fmt"]], device=DEV) for _ in range(2))
    for b, (prompt, tail) in enumerate(hist):
        for side, to in enumerate((s["k"], s["v"])):
            rows = torch.cat([prompt[side], tail[side]])
            for h, k in enumerate(lv):
                at = _resident(c, cb[k], lens[b])
                to[b * c["hkv"] + h, :len(at)] = rows[at, h].to(to.dtype)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _select_plain(s):
    """In 64 bits, since the order of two beams' tokens hangs on their sums."""
    c = s["c"]
    x = s["x"].double()
    top = x.amax(dim=2, keepdim=True)
    lse = top + (x - top).exp().sum(dim=2, keepdim=True).log()
    score = (s["scores"].double()[..., None] + (x - lse)).nan_to_num_(nan=-math.inf).flatten(1)
    n = min(c["n_out"], score.shape[1])
    least = score.topk(n, dim=1).values[:, -1:]
    above, at = score > least, score == least
    taken = above | (at & (at.cumsum(dim=1, dtype=torch.int32) <= n - above.sum(dim=1, keepdim=True)))
    flat = taken.nonzero()[:, 1].view(-1, n)                      # rising, so that ties stay in order
    val, by = score.gather(1, flat).sort(dim=1, descending=True, stable=True)
    flat = flat.gather(1, by)
    group = torch.arange(c["groups"], device=DEV)[:, None] * c["beams"]
    none = val == -math.inf
    parent = (group + flat // c["vocab"]).masked_fill(none, -1)
    token = (flat % c["vocab"]).masked_fill(none, -1)
    pad = c["n_out"] - n
    return {"scores": torch.nn.functional.pad(val.float(), (0, pad), value=-math.inf),
            "parents": torch.nn.functional.pad(parent.int(), (0, pad), value=-1),
            "tokens": torch.nn.functional.pad(token.int(), (0, pad), value=-1)}


def _reorder_plain(s):
    s["windows"][:, :, s["dst"]] = s["windows"][:, :, s["src"]]
    s["pool"][s["last"][:, s["into"]]] = s["pool"][s["last"][:, s["from"]]]
    s["last"] = s["last"][:, s["owner"]]


def _move_plain(s):
    buf, windows, pool = s["other"]
    windows[:, :, s["live"]] = s["windows"][:, :, s["live"]]
    pool[:len(s["order"])] = s["pool"][s["order"]]
    s["other"] = s["buf"], s["windows"], s["pool"]
    s["buf"], s["windows"], s["pool"] = buf, windows, pool
    s["order"] = torch.arange(len(s["order"]), device=DEV)


def _shared_plain(s):
    c = s["c"]
    batch = c["groups"] * c["beams"]
    q = s["q"].float().reshape(batch * c["hkv"], c["g"], c["d"])
    z = (q @ s["k"].float().transpose(1, 2)) * s["scale"]
    seen = torch.arange(z.shape[2], device=DEV) < s["count"][:, None]
    z = z.masked_fill(~seen[:, None], -math.inf)
    p = torch.exp(z - z.amax(dim=2, keepdim=True))
    out = (p @ s["v"].float()) / p.sum(dim=2, keepdim=True)
    return out.reshape(batch, c["hkv"] * c["g"], c["d"])


def _rows_of(s, used):
    """What the cache holds, as bits: rows are copied, not computed."""
    return {"windows": s["windows"].view(torch.int16), "pool": s["pool"][:used].view(torch.int16)}


def run(s):
    c = s["c"]
    if c["kind"] == "select":
        if own:
            from paper_2609_02029_amd import hwkv
            hwkv.beam_select(s["x"], s["scores"], *s["out"], s["ws"])
            return dict(zip(("scores", "parents", "tokens"), s["out"]))
        return _select_plain(s)
    if c["kind"] == "reorder":
        if own:
            from paper_2609_02029_amd import hwkv
            hwkv.cache_reorder(s["cache"], s["parents"])
        else:
            _reorder_plain(s)
        return _rows_of(s, len(s["pool"]))
    if c["kind"] == "move":
        if own:
            from paper_2609_02029_amd import hwkv
            buf, windows, pool = s["other"]
            hwkv.cache_move(s["cache"], len(pool), buf)
            s["other"] = s["buf"], s["windows"], s["pool"]
            s["buf"], s["windows"], s["pool"] = buf, windows, pool
            return _rows_of(s, s["used"])
        _move_plain(s)
        return _rows_of(s, len(s["order"]))
    if own:
        from paper_2609_02029_amd import hwkv
        hwkv.decode_attn_shared(s["cache"], 0, s["q"], s["scale"], s["out"], s["ws"])
        return s["out"]
    return _shared_plain(s)


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    """(Rows that are copied have no other definition than their bits.)"""
    x = _Inputs(c, seed)
    if c["kind"] == "select":
        z, scores = x.logits()
        out = torch.full((c["groups"], c["n_out"]), -math.inf, dtype=torch.float64, device=DEV)
        for g in range(c["groups"]):
            got = []
            for b in range(c["beams"]):
                if scores[g, b] > -math.inf and z[g, b].max() > -math.inf:
                    row = z[g, b].double()
                    got.append(scores[g, b].double() + row - torch.logsumexp(row, 0))
            if got:
                best = torch.cat(got).sort(descending=True).values[:c["n_out"]]
                out[g, :len(best)] = best
        return {"scores": out, "parents": None, "tokens": None}
    if c["kind"] != "shared":
        return None
    scale, g, cb, lv = 1.0 / math.sqrt(c["d"]), c["g"], _codebook(c), _levels(c)
    hist = _histories(c, x)
    q = x.normal(c["groups"] * c["beams"], c["hkv"] * g, c["d"]).double()
    out = torch.empty_like(q)
    for b, (prompt, tail) in enumerate(hist):
        n = len(prompt[0]) + len(tail[0])
        for h in range(c["hkv"]):
            at = _resident(c, cb[lv[h]], n)
            k, v = (torch.cat([p[:, h], t[:, h]])[at].to(TYPES[c["fmt"]]).double() for p, t in zip(prompt, tail))
            z = (q[b, h * g:(h + 1) * g] @ k.T) * scale
            out[b, h * g:(h + 1) * g] = torch.softmax(z, dim=1) @ v
    return out
