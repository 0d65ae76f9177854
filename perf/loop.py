"""Calls one operator over and over, for a profiler or a clock.

    python3 perf/loop.py WORKLOAD CALLS

WORKLOAD: a case of ``perf/operators.py`` (its own inputs and call), or

* ``layers:CASE``, ``fused:CASE``: a decode case over a cache of 16 layers taken in
  turn, as a model's step has them (the rows of one layer alone may stay in the
  last-level cache), with ``decode_attn`` or ``append_decode_attn``;
* ``append:FORMAT``: ``append_rope`` of the case ``append_batch`` into a cache of
  that format;
* ``write``: ``prefill_write`` of 32,768 tokens of 8 KV heads of 128 into an int8
  cache;
* ``replay:FORMAT``: the calibration replay of 64 rows over 32,768 tokens, 24 query
  and 4 KV heads of 256, four windows.

Copies 512 MiB three times (counters are scaled by them), then makes CALLS calls,
and again CALLS calls against the clock.
"""
import math
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

import perf.operators as ops  # noqa: E402
from paper_2609_02029_amd import hwkv  # noqa: E402

DEV = "cuda"
LAYERS = 16


def _normal(*shape):
    return torch.randn(shape, device=DEV).to(torch.bfloat16)


def _layers(case, fused, calls):
    c = next(x for x in ops.listed() if x["name"] == case)
    lens, x = ops._lengths(c), ops._Inputs(c, 1)
    hkv, d, hq = c["hkv"], c["d"], c["hkv"] * c["g"]
    pol = hwkv.policy_set(LAYERS, hkv, hq, d, c["sinks"], ops._codebook(c), [ops._levels(c)] * LAYERS)
    top = max(lens) + 2 * calls // LAYERS + 2
    pages = LAYERS * hkv * sum(-(-top // ops.PAGE) for _ in lens) if c["paged"] else None
    cache = hwkv.cache_alloc(pol, c["batch"], top, kv_format="i8", n_pages=pages)
    for b, n in enumerate(lens):
        k, v = x.kv(n)
        for layer in range(LAYERS):
            hwkv.prefill_write(cache, layer, b, 0, k, v)
    q, kn, vn = _normal(c["batch"], hq, d), _normal(c["batch"], hkv, d), _normal(c["batch"], hkv, d)
    out = torch.empty(q.shape, device=DEV)
    ws = torch.empty(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    scale = 1 / math.sqrt(d)
    if fused:
        return lambda i: hwkv.append_decode_attn(cache, i % LAYERS, kn, vn, q, scale, out, ws)
    return lambda i: hwkv.decode_attn(cache, i % LAYERS, q, scale, out, ws)


def _append(fmt):
    c = next(x for x in ops.listed() if x["name"] == "append_batch")
    hkv, d, b, hq = c["hkv"], c["d"], c["batch"], c["hkv"] * c["g"]
    freq, axis = ops._frequencies(c)
    pol = hwkv.policy_set(1, hkv, hq, d, c["sinks"], [c["window"], 0], [[0] * (hkv - c["full"]) + [1] * c["full"]])
    cache = hwkv.cache_alloc(pol, b, 16384, kv_format=fmt, n_pages=c["full"] * b * 64)
    rope = hwkv.rope_set(d, freq, axis)
    row, pos = _normal(b, hq + 2 * hkv, d), torch.arange(b, dtype=torch.int32, device=DEV)
    q, k, v = row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
    out = torch.empty((b, hq, d), dtype=torch.bfloat16, device=DEV)
    return lambda i: hwkv.append_rope(cache, 0, rope, pos, k, v, q, out)


def _write():
    # eight layers and prompts in turn: one prompt's 134 MB would stay in the
    # last-level cache
    pol = hwkv.policy_set(8, 8, 8, 128, 0, [0], [[0] * 8] * 8)
    cache = hwkv.cache_alloc(pol, 1, 32768, kv_format="i8")
    kv = [(_normal(32768, 8, 128), _normal(32768, 8, 128)) for _ in range(8)]

    def call(i):
        if i % 8 == 0:
            hwkv.cache_reset_seq(cache, 0)
        hwkv.prefill_write(cache, i % 8, 0, 0, *kv[i % 8])
    return call


def _replay(fmt):
    n, rows, hkv, hq, d, windows = 32768, 64, 4, 24, 256, [1024, 4096, 16384]
    k, v, q = _normal(n, hkv, d), _normal(n, hkv, d), _normal(rows, hq, d)
    at = [n // rows * (i + 1) - 1 for i in range(rows)]
    ws = torch.empty(hwkv.calib_workspace_bytes(hq, d, 4, n, rows, n_kv_heads=hkv, kv_format=fmt), dtype=torch.uint8,
                     device=DEV)
    outs = torch.empty((len(windows) + 1, rows, hq, d), device=DEV)
    scores, means = torch.empty((len(windows), rows, hq), device=DEV), torch.empty((len(windows), hkv), device=DEV)
    return lambda i: hwkv.calib_replay(k, v, at, q, windows, 4, 1 / math.sqrt(d), outs, scores, means, ws,
                                       kv_format=fmt)


def workload(name, calls):
    kind, _, rest = name.partition(":")
    if kind in ("layers", "fused"):
        return _layers(rest, kind == "fused", calls)
    if kind == "append":
        return _append(rest)
    if kind == "write":
        return _write()
    if kind == "replay":
        return _replay(rest)
    ops.own = True
    state = ops.prepare(next(c for c in ops.listed() if c["name"] == name), 1)
    return lambda i: ops.run(state)


def main():
    name, calls = sys.argv[1], int(sys.argv[2])
    a = torch.empty(512 << 20, dtype=torch.uint8, device=DEV).random_()
    b = torch.empty_like(a)
    for _ in range(3):
        b.copy_(a)
    call = workload(name, calls)
    for i in range(calls):
        call(i)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for i in range(calls):
        call(i)
    torch.cuda.synchronize()
    print(f"{name}: {calls} calls, {(time.perf_counter() - t) / calls * 1e6:.2f} us a call", flush=True)


if __name__ == "__main__":
    main()
