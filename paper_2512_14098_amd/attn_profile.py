"""Measured attention time of an LLM executor's iterations on a workload's own requests.

The planner prices an iteration by a latency model: a prefill (k0 + k1 X) + k2 n for X tokens of
n requests, a decode step d0 + d1 n.  What such a model cannot be fitted to without a
card is the part that depends on context lengths, the attention over the cache, one share of what
an executor's profile (Sec. 5.1) holds.  This module measures it: requests come from the workload's trace, an executor admits them in batches of the
batch knob, and each iteration runs the calls that a serving step makes - cf_kv_map for the step,
cf_kv_write and cf_attn_paged for each layer on one cf_attn_plan, cf_attn_prompt for an encoder's
batch.  With --rope queries and keys are turned by their positions in every layer (cf_rope), with
--cache8 the caches hold e4m3 codes: cf_kv_write8 or, with both, cf_rope_write8 for each layer, cf_attn_paged8,
and the hand-over of the prefilled requests to another executor (cf_kv_read8).  Keys, values and queries are random.  Layers and heads are the caller's: no workload holds
them, so the seconds stand beside the latency model's and are no share of it.

Layers have caches of their own, as many as make one pass over the layers read PASS_BYTES, twice
what the last-level cache holds, before it comes back to the first: with one cache for all
layers, small batches would be read from there, which no executor's are (16 requests of c1, 32 layers:
a decode step of 1.35 ms, 1.31 with one cache).  Times are those of the calls in a row: where the kernels
are shorter than the calls (4 requests: 0.70 ms for 65 of them), the calls'.

    python -m paper_2512_14098_amd.attn_profile --config c1 --batch 64 --layers 32 [--rope] [--cache8]
"""
import argparse

import numpy as np
import torch

from . import cf
from .inputs import load_config

FRAME_MS, WINDOW = 20, 4096  # an audio encoder's frames, and the most it attends over at once
PASS_BYTES = 512 << 20
PATCH_FIELD = 3  # of the trace's random numbers
ATTRS = ("prompt", "out", "patches", "aud_in_ms", "aud_out_ms", "aud_in_tok", "aud_out_tok")


def _component_requests(model, trace, component):
    """The requests of a host trace whose type runs the component, their X and output lengths."""
    comp = next(c for c in model["components"] if c["name"] == component)
    runs = np.array([component in t["comps"] for t in model["types"]])
    t = {a: np.asarray(trace[a], np.int64) for a in ATTRS if a in trace}
    t["aud_in_tok"], t["aud_out_tok"] = -(-t["aud_in_ms"] // 80), -(-t["aud_out_ms"] // 80)
    x = sum(t[a] for a in comp["x"])
    keep = runs[np.asarray(trace["type"])] & (x > 0)
    return np.flatnonzero(keep), x[keep], np.maximum(t[comp.get("n_out", "out")][keep], 1)


def component_tokens(model, trace, component):
    """Input tokens X of each request of a host trace whose type runs the component."""
    return _component_requests(model, trace, component)[1:]


def image_patches(model, trace, seed, requests, device="cuda"):
    """Patches of every image of the requests, in order.  A trace holds a request's sum; its
    images are words 0, 1, ... of the request's block of random numbers, uniform integers."""
    requests = np.asarray(requests, np.int64)
    ctr, key = np.zeros((len(requests), 4), np.int64), np.zeros((len(requests), 2), np.int64)
    ctr[:, 0], ctr[:, 1], key[:, 0] = requests, PATCH_FIELD, np.uint64(seed).view(np.int64)
    x = cf.cf_philox_eval(torch.from_numpy(ctr).to(device), torch.from_numpy(key).to(device)).cpu().numpy()
    lo, hi = model.get("patches_per_image", [256, 1024])
    per = lo + ((x.view(np.uint64) >> np.uint64(32)) * np.uint64(hi - lo + 1) >> np.uint64(32)).astype(np.int64)
    n = np.asarray(trace["n_img"], np.int64)[requests]
    out = [per[i, :k] for i, k in enumerate(n)]
    if [int(p.sum()) for p in out] != np.asarray(trace["patches"], np.int64)[requests].tolist():
        raise cf.CfError("the trace's patches are not those of seed %d" % seed)
    return np.concatenate(out) if out else np.zeros(0, np.int64)


def encoder_sequences(model, trace, component, seed, requests, device="cuda"):
    """Lengths of the sequences that an encoder attends over for some requests: each image on its
    own, audio in windows of WINDOW frames, other tokens request by request."""
    comp = next(c for c in model["components"] if c["name"] == component)
    out = []
    for a in comp["x"]:
        if a == "patches":
            out += image_patches(model, trace, seed, requests, device).tolist()
            continue
        ms = np.asarray(trace[a.replace("_tok", "_ms")], np.int64)[requests]
        for n in (-(-ms // 80) if a.endswith("_tok") else -(-ms // FRAME_MS) if a.endswith("_ms") else ms).tolist():
            out += [n] if not a.endswith("_ms") else [WINDOW] * (n // WINDOW) + [n % WINDOW]
    return [n for n in out if n > 0]


class PagedExecutor:
    """One executor's paged cache and the attention of its iterations.  tokens: those that a step
    reads of each layer's cache (all that it holds if not given), for the number of caches.  rope: the base of
    the rotary frequencies, by which queries and keys are turned (None: not at all).  cache8: e4m3
    caches, each a triple of codes of keys and of values and exponents."""

    def __init__(self, slots, longest, layers, heads, kv_heads, dim, page=16, dtype=torch.bfloat16, device="cuda",
                 tokens=None, rope=None, cache8=False):
        self.layers, self.heads, self.kv_heads, self.dim, self.page = layers, heads, kv_heads, dim, page
        rows = -(-longest // page)
        n_pages = slots * rows
        self.table = torch.full((slots, rows), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.head = torch.zeros(1, dtype=torch.int32, device=device)
        shape = (n_pages, kv_heads, page, dim)
        row = 2 * kv_heads * (dim + 1 if cache8 else dim * dtype.itemsize)
        read = (n_pages * page if tokens is None else max(int(tokens), 1)) * row
        self.cache8, self.freq = cache8, None
        if rope is not None:
            self.freq = torch.from_numpy(float(rope) ** (-np.arange(dim // 2) / (dim // 2))).to(device)
        self.caches = [self._cache8(shape, device) if cache8 else
                       tuple(torch.randn(shape, dtype=dtype, device=device) for _ in range(2))
                       for _ in range(max(1, min(layers, -(-PASS_BYTES // read))))]
        self.qkv = torch.empty((0, heads + 2 * kv_heads, dim), dtype=dtype, device=device)

    @staticmethod
    def _cache8(shape, device):
        codes = [torch.randint(0, 127, shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
                 for _ in range(2)]
        exps = torch.full((shape[0], shape[1], 2, shape[2]), 120, dtype=torch.uint8, device=device)
        return codes[0], codes[1], exps

    def step(self, ctx_len, new_len, n_tok, max_new):
        """One iteration: returns its attention output (the last layer's) and the status words."""
        if self.qkv.shape[0] < n_tok:
            self.qkv = torch.randn((n_tok,) + tuple(self.qkv.shape[1:]), dtype=self.qkv.dtype, device=self.qkv.device)
        x, h, g = self.qkv[:n_tok], self.heads, self.kv_heads
        q_start, kv_len, slots, pos, head, status = cf.cf_kv_map(ctx_len, new_len, self.table, self.page, self.free,
                                                                 self.head, n_tok)
        self.head = head
        plan = cf.cf_attn_plan(q_start, kv_len, n_tok, max_new, h, g, self.dim)
        for layer in range(self.layers):
            cache = self.caches[layer % len(self.caches)]
            q, k, v = x[:, :h], x[:, h:h + g], x[:, h + g:]
            if self.cache8:
                if self.freq is None:
                    cf.cf_kv_write8(k, v, *cache, slots)
                else:
                    q = cf.cf_rope_write8(q, k, v, pos, self.freq, None, *cache, slots)
                out = cf.cf_attn_paged8(plan, q, *cache, self.table)
            else:
                if self.freq is not None:
                    q, k = cf.cf_rope(q, k, pos, self.freq)
                cf.cf_kv_write(k, v, *cache, slots)
                out = cf.cf_attn_paged(plan, q, *cache, self.table)
        return out, status

    def hand_over(self, lens, n_tok):
        """Every layer's cached tokens of the requests, lens int32 [slots] of them, as packed 16-bit rows: the
        last layer's keys and values and the starts."""
        start = torch.zeros(len(lens) + 1, dtype=torch.int32, device=lens.device)
        torch.cumsum(lens, 0, dtype=torch.int32, out=start[1:])
        for layer in range(self.layers):
            k, v = cf.cf_kv_read8(*self.caches[layer % len(self.caches)], self.table, start, n_tok, self.qkv.dtype)
        return k, v, start


def _timed(fn):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    out = fn()
    b.record()
    b.synchronize()
    return out, a.elapsed_time(b) * 1e-3


def profile(config, component=None, batch=64, layers=32, heads=32, kv_heads=8, dim=128, page=16, decode_steps=4,
            n_req=1000, seed=0, device="cuda", rope=None, cache8=False):
    """Attention seconds of one prefill and of decode steps of ``batch`` requests of the
    workload's first LLM (or ``component``), beside the latency model's seconds; for each
    encoder, the attention of a batch of its inputs.  rope, cache8: as PagedExecutor takes them; an
    8-bit cache's rows have one more, the hand-over of the prefilled requests."""
    cfg = load_config(config) if isinstance(config, str) else config
    model = cfg["model"]
    desc = cf.model_desc(model)
    trace, _ = cf.cf_trace_gen(desc, [seed], n_req, device)
    host = trace.to_numpy()
    llm = component or next(c["name"] for c in model["components"] if c["kind"] == "LLM")
    comp = next(c for c in model["components"] if c["name"] == llm)
    x, out = component_tokens(model, host, llm)
    x, out = x[:batch], out[:batch]
    n = len(x)
    if n == 0:
        raise cf.CfError("no request of the trace runs " + llm)
    more = dict(rope=rope, cache8=cache8) if rope is not None or cache8 else {}
    ex = PagedExecutor(n, int(x.max()) + decode_steps + 1, layers, heads, kv_heads, dim, page, device=device,
                       tokens=int(x.sum()), **more)
    rows = []
    ctx = torch.zeros(n, dtype=torch.int32, device=device)
    new = torch.as_tensor(x.astype(np.int32)).to(device)
    ones = torch.ones(n, dtype=torch.int32, device=device)
    k0, k1, k2 = comp["k"]
    d0, d1 = comp.get("decode", (0.0, 0.0))
    (_, status), _ = _timed(lambda: ex.step(ctx, new, int(x.sum()), int(x.max())))  # the first call builds buffers
    ex.head.zero_()
    (_, status), s = _timed(lambda: ex.step(ctx, new, int(x.sum()), int(x.max())))
    if int(status.sum()):
        raise cf.CfError("the cache does not hold the batch")
    rows.append(dict(step="prefill", component=llm, requests=n, tokens=int(x.sum()), attention_s=s,
                     model_s=k0 + k1 * float(x.sum()) + k2 * n))
    if cache8:
        run = lambda: ex.hand_over(new, int(x.sum()))
        _timed(run)
        rows.append(dict(step="hand over", component=llm, requests=n, tokens=int(x.sum()), attention_s=_timed(run)[1],
                         model_s=0.0))
    ctx = new.clone()
    for i in range(decode_steps):
        (_, status), s = _timed(lambda: ex.step(ctx, ones, n, 1))
        ctx = ctx + ones
        rows.append(dict(step="decode %d" % i, component=llm, requests=n, tokens=int(x.sum()) + n * (i + 1),
                         attention_s=s, model_s=d0 + d1 * n))
    for c in model["components"]:
        if c["kind"] != "ENC":
            continue
        ids, x, _ = _component_requests(model, host, c["name"])
        ids, x = ids[:batch], x[:batch]
        if len(x) == 0:
            continue
        e = encoder_sequences(model, host, c["name"], seed, ids, device)
        starts = torch.as_tensor(np.concatenate([[0], np.cumsum(e)]).astype(np.int32)).to(device)
        y = torch.randn((sum(e), 3 * 16, 64), dtype=torch.bfloat16, device=device)
        run = lambda: [cf.cf_attn_prompt(y[:, :16], y[:, 16:32], y[:, 32:], starts, causal=False)
                       for _ in range(layers)]
        _timed(run)
        _, s = _timed(run)
        rows.append(dict(step="encode", component=c["name"], requests=len(x), tokens=sum(e), attention_s=s,
                         model_s=c["k"][0] + c["k"][1] * float(x.sum()) + c["k"][2] * len(x)))
    return rows


def main(argv=None):
    p = argparse.ArgumentParser(description="attention time of an LLM executor's iterations on this GPU")
    p.add_argument("--config", default="c1")
    p.add_argument("--component")
    for name, value in (("batch", 64), ("layers", 32), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("page", 16)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--rope", type=float, nargs="?", const=10000.0, help="turn queries and keys; the frequencies' base")
    p.add_argument("--cache8", action="store_true", help="e4m3 caches")
    a = p.parse_args(argv)
    for r in profile(a.config, a.component, a.batch, a.layers, a.heads, a.kv_heads, a.dim, a.page, rope=a.rope,
                     cache8=a.cache8):
        print("%-10s %-8s %4d requests %8d tokens  attention %9.3f ms  latency model %9.3f ms"
              % (r["step"], r["component"], r["requests"], r["tokens"], r["attention_s"] * 1e3, r["model_s"] * 1e3))


if __name__ == "__main__":
    main()
