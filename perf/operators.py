"""The 4-bit cache and the eviction by attention weight, as cases that can be timed and checked.

Four kinds of pass, each one thing a program does through the Python binding:

`compact_q4`  the compaction of a finished prefill into 4-bit rows, and those rows read back as bf16;
`decode_q4`   a generation loop over a 4-bit cache, with or without the rows' attention weights;
`decode`      the same loop over a bf16 cache, with the rows' attention weights;
`evict`       the rows of least weight dropped, the others moved to another cache (bf16 or 4-bit rows),
              after a prompt together with the prefill's key weights.

A 4-bit row holds blocks of 32 values along the head: a power of two 2^e, e the smallest integer in
[-127, 125] with max|x| <= 7 * 2^e, and per value the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} to x / 2^e, ties
to the even code (a code is 8 * sign + index; the even element of a byte is in its low half).

`listed()` names the cases, `draw(rng)` gives another one of the same ranges, `prepare` builds what a program
holds before the call, `run` is one pass (in plain torch operations, or with `own` in this library's calls),
`work` counts what a pass cannot do without, and `exact` computes the outputs in 64 bits.
"""
import random

import numpy as np
import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TEXT, CURRENT = 1, 3   # roles: history text, which the compaction drops, and any other


# ------------------------------------------------------------------ the cases
def listed():
    llama = dict(q_heads=32, kv_heads=8, head_dim=128)
    qwen = dict(q_heads=28, kv_heads=4, head_dim=128)
    tiny = dict(q_heads=4, kv_heads=2, head_dim=64)
    return [
        # the compaction after the prompt of eight eight-turn conversations
        dict(name="compact_q4_8b", kind="compact_q4", batch=8, ctx_min=5424, ctx_max=5424, keep_pct=24, ragged=0, **llama),
        # the same after four 32-turn conversations of 40k tokens
        dict(name="compact_q4_long", kind="compact_q4", batch=4, ctx_min=40320, ctx_max=40320, keep_pct=19, ragged=0, **qwen),
        # a first short conversation: the latency of a step
        dict(name="decode_q4_tiny", kind="decode_q4", batch=1, ctx_min=120, ctx_max=120, ragged=0, steps=16, weights=False,
             **tiny),
        # generation for eight conversations compressed to 1.3k rows each
        dict(name="decode_q4_8b", kind="decode_q4", batch=8, ctx_min=1328, ctx_max=1328, ragged=0, steps=16, weights=False,
             **llama),
        # late in four very long conversations whose cache will be cut: the weights are kept
        dict(name="decode_q4_long", kind="decode_q4", batch=4, ctx_min=7552, ctx_max=7552, ragged=0, steps=8, weights=True,
             **qwen),
        # a full server: 64 conversations of uneven length
        dict(name="decode_q4_uneven", kind="decode_q4", batch=64, ctx_min=180, ctx_max=4300, ragged=5, steps=4, weights=False,
             **llama),
        # one conversation with a book in its cache, an odd number of rows
        dict(name="decode_q4_one", kind="decode_q4", batch=1, ctx_min=100001, ctx_max=100001, ragged=0, steps=4, weights=False,
             **llama),
        # the bf16 cache of the eight conversations, with weights
        dict(name="decode_weighted_8b", kind="decode", batch=8, ctx_min=1328, ctx_max=1328, ragged=0, steps=16, weights=True,
             **llama),
        # the bf16 cache of a full server, with weights
        dict(name="decode_weighted_uneven", kind="decode", batch=64, ctx_min=180, ctx_max=4300, ragged=5, steps=4, weights=True,
             **llama),
        # after a prompt: its key weights carried over, half of the rows dropped, system prompt and query kept
        dict(name="evict_prompt", kind="evict", rows="bf16", prompt=True, batch=8, ctx_min=1328, ctx_max=1328, budget_pct=50,
             head=256, tail=256, ragged=0, **llama),
        # the long conversations' 4-bit rows cut to a quarter
        dict(name="evict_long_q4", kind="evict", rows="q4", prompt=False, batch=4, ctx_min=7552, ctx_max=7552, budget_pct=25,
             head=512, tail=512, ragged=0, **qwen),
        # a full server making room: 64 uneven conversations cut to half of the longest but for their first and last rows
        dict(name="evict_uneven", kind="evict", rows="bf16", prompt=False, batch=64, ctx_min=100, ctx_max=8192, budget_pct=50,
             head=64, tail=100, ragged=7, **llama),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (4, 2, 64), (8, 8, 128), (8, 1, 64), (16, 2, 128), (5, 5, 64),
                             (40, 8, 64), (21, 7, 128)])
    case = dict(kind=rng.choice(["compact_q4", "decode_q4", "decode_q4", "decode_q4", "decode", "decode", "evict", "evict"]),
                batch=_log(rng, 1, 64), ragged=rng.randint(1, 1000), q_heads=hq, kv_heads=hkv, head_dim=d)
    rows = 90_000_000 // (hkv * d)          # of all requests, so that no draw is larger than the listed cases
    top = max(1, min(100_000, rows // case["batch"]))
    if case["kind"] == "compact_q4":
        case["ctx_max"] = _log(rng, 16, max(16, min(40_000, top)))
        case["keep_pct"] = rng.choice([1, 5, 20, 33, 50, 100])
    elif case["kind"] == "evict":
        case["ctx_max"] = _log(rng, 1, top)
        case.update(rows=rng.choice(["bf16", "q4"]), prompt=rng.random() < 0.4, budget_pct=rng.choice([0, 1, 10, 25, 50, 75, 99, 120]),
                    head=_log(rng, 1, 500) - 1, tail=_log(rng, 1, 500) - 1)
    else:
        case["ctx_max"] = _log(rng, 1, max(1, top // 4))
        case.update(steps=rng.randint(1, 16) if case["ctx_max"] * case["batch"] < 20_000 else rng.randint(1, 4),
                    weights=case["kind"] == "decode" or rng.random() < 0.4)
    case["ctx_min"] = max(1, case["ctx_max"] // rng.choice([1, 2, 24]))
    return case


def _lengths(case):
    """Rows of each request before the call."""
    r = random.Random(case["ragged"])
    lo, hi = case["ctx_min"], case["ctx_max"]
    return [hi if lo == hi else _log(r, lo, hi) for _ in range(case["batch"])]


def _kept(case):
    """Rows that each request of an eviction keeps."""
    budget = case["ctx_max"] * case["budget_pct"] // 100
    got = []
    for n in _lengths(case):
        h = min(case["head"], n)
        t = min(case["tail"], n - h)
        got.append(n if n <= budget else h + t + min(max(budget - h - t, 0), n - h - t))
    return got


def _starts(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, np.int64))])[:-1].astype(np.int64)


def _ints(a, dtype=torch.int32):
    return torch.tensor([int(x) for x in a], dtype=dtype, device="cuda")


# ------------------------------------------------------------------ 4-bit rows, plain form
def _block_exponents(x):
    """[..., d / 32] the exponent of each block's scale; 128 for a block with an infinity or a NaN."""
    top = x.unflatten(-1, (-1, 32)).abs().amax(-1)
    bits = top.view(torch.int16).int()
    e = (((bits + 31) >> 7) - 129).clamp(-127, 125)
    return torch.where(bits >= 0x7F80, 128, e)


def _codes(x):
    """bf16 [..., d] -> (codes uint8 [..., d / 2], two a byte; scale bytes uint8 [..., d / 32])."""
    e = _block_exponents(x)
    u = x.unflatten(-1, (-1, 32)).float() * torch.ldexp(torch.ones((), device=x.device), -e.clamp(max=125))[..., None]
    a = u.abs().clamp(max=6.0)
    a = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2))
    index = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))
    code = torch.where((e == 128)[..., None], 0, index).to(torch.uint8) | (torch.signbit(u).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The values that 4-bit rows stand for, in 32 bits."""
    table = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    pair = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    scale = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    scale = torch.where(scales == 255, torch.nan, scale)
    return (pair.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


# ------------------------------------------------------------------ inputs
class _Normals:
    """bf16 tensors of normal values, from a seed, drawn on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def __call__(self, *shape, scale=1.0):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        rows = max(1, (1 << 27) // max(1, int(np.prod(shape[1:]))))
        for i in range(0, shape[0], rows):
            part = torch.randn((min(rows, shape[0] - i),) + shape[1:], generator=self.gen, device="cuda")
            x[i:i + rows] = part * scale
        return x

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device="cuda")

    def channels(self, heads, d):
        """Magnitudes of a head's channels: a few stand out, as a model's keys have them."""
        return torch.exp(0.6 * torch.randn((heads, d), generator=self.gen, device="cuda")) * (0.5 + self.uniform(heads, 1))


def _weights(draw_, n):
    """Attention weights of n rows: most of them small, some exactly zero."""
    w = torch.exp(2.0 * torch.randn(n, generator=draw_.gen, device="cuda")) / max(n, 1)
    return torch.where(draw_.uniform(n) < 0.1, 0.0, w)


def _rows_in_4_bits(x):
    """A bf16 tensor of rows as (codes, scale bytes), made in parts."""
    n, h, d = x.shape
    codes = torch.empty((n, h, d // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, h, d // 32), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (h * d))
    for i in range(0, n, step):
        codes[i:i + step], scales[i:i + step] = _codes(x[i:i + step])
    return codes, scales


def _inputs(case, seed):
    kind, b, hq, hkv, d = (case[n] for n in ("kind", "batch", "q_heads", "kv_heads", "head_dim"))
    draw_ = _Normals(seed)
    lens = _lengths(case)
    s = dict(case=case, lens=lens)
    sk, sv = draw_.channels(hkv, d), draw_.channels(hkv, d)
    if kind == "compact_q4":
        # kept rows come in runs, as a prompt's roles do: system prompt, Nexus rows, current rows
        s["cu_host"] = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        period = 100
        keep = case["keep_pct"] * period // 100
        role = np.concatenate([np.where((np.arange(n) % period < keep) | (np.arange(n) == n - 1), CURRENT, TEXT) for n in lens])
        s["kept"] = [int(np.sum(role[a:a + n] != TEXT)) for a, n in zip(s["cu_host"], lens)]
        s["role"] = torch.from_numpy(role.astype(np.uint8)).cuda()
        s["k"], s["v"] = draw_(sum(lens), hkv, d, scale=sk), draw_(sum(lens), hkv, d, scale=sv)
        s["off"], s["rows"] = _starts(s["kept"]), sum(s["kept"])
        return s
    if kind == "evict":
        s["kept"] = _kept(case)
        s["off"], s["rows"] = _starts(lens), sum(lens)
        s["out_off"], s["out_rows"] = _starts(s["kept"]), sum(s["kept"])
        if case["prompt"]:
            # the cache of a prompt: every request's prompt was up to twice as long as what was kept
            s["prompt"] = [2 * n for n in lens]
            s["cu_host"] = np.concatenate([[0], np.cumsum(s["prompt"])]).astype(np.int32)
            index = torch.empty(s["rows"], dtype=torch.int32, device="cuda")
            for o, n in zip(s["off"], lens):
                index[o:o + n] = 2 * torch.arange(n, device="cuda") + (draw_.uniform(n) < 0.5).int()
            s["index"] = index
            s["key_weight"] = _weights(draw_, int(s["cu_host"][-1]))
        else:
            s["weight"] = _weights(draw_, s["rows"])
    else:
        n = case["steps"]
        cap = [x + n for x in lens]
        s["cap"], s["off"], s["rows"] = cap, _starts(cap), sum(cap)
        s["dq"] = draw_(n, b, hq, d)
        s["dk"], s["dv"] = draw_(n, b, hkv, d, scale=sk), draw_(n, b, hkv, d, scale=sv)
        if case["weights"]:
            s["weight0"] = _weights(draw_, s["rows"])
    for name, scale in (("k", sk), ("v", sv)):
        x = draw_(s["rows"], hkv, d, scale=scale)
        if kind == "decode_q4" or case.get("rows") == "q4":
            s[name], s[name + "s"] = _rows_in_4_bits(x)
        else:
            s[name] = x
    return s


# ------------------------------------------------------------------ prepare
def _capture(call):
    """`call` as a graph, as a program replays a fixed loop; called once before, so that everything is loaded."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    return g


def _like(s, name, rows):
    return torch.zeros((rows,) + s[name].shape[1:], dtype=s[name].dtype, device="cuda")


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2601_21927_amd import sonic
    kind, b, hq, hkv, d = (case[n] for n in ("kind", "batch", "q_heads", "kv_heads", "head_dim"))
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["row_off"] = _ints(s["off"], torch.int64)
    s["zero"] = _ints([0] * b)

    def bf16(rows):
        return torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device="cuda")

    def q4(rows):
        return [torch.zeros((rows, hkv, d // w), dtype=torch.uint8, device="cuda") for w in (2, 32, 2, 32)]

    if kind == "compact_q4":
        s["cu"], s["cap_dev"] = _ints(s["cu_host"]), _ints(s["kept"])
        s["planes"], s["length"] = q4(s["rows"]), _ints([0] * b)
        s["keep_idx"] = torch.zeros(s["rows"], dtype=torch.int32, device="cuda")
        s["ko"], s["vo"] = bf16(s["rows"]), bf16(s["rows"])
    elif kind == "evict":
        n = max(s["lens"])
        s["length"], s["max_rows"] = _ints(s["lens"]), n
        s["head"], s["tail"] = _ints([case["head"]] * b), _ints([case["tail"]] * b)
        s["budget"] = _ints([case["ctx_max"] * case["budget_pct"] // 100] * b)
        s["ws"] = torch.zeros(sonic.cache_evict_workspace_bytes(b, n), dtype=torch.uint8, device="cuda")
        s["out"] = {name: _like(s, name, s["out_rows"]) for name in ("k", "v", "ks", "vs") if name in s}
        s["out_row_off"], s["out_cap"], s["out_len"] = _ints(s["out_off"], torch.int64), _ints(s["kept"]), _ints([0] * b)
        s["out_weight"] = torch.zeros(s["out_rows"], device="cuda")
        s["out_index"] = torch.zeros(s["out_rows"], dtype=torch.int32, device="cuda")
        if case["prompt"]:
            s["cu"], s["weight"] = _ints(s["cu_host"]), torch.zeros(s["rows"], device="cuda")
        if case["rows"] == "q4":
            s["ko"], s["vo"] = bf16(s["out_rows"]), bf16(s["out_rows"])
    else:
        n = case["steps"]
        s["max_ctx"] = max(s["cap"])
        s["len0"], s["length"], s["cap_dev"] = _ints(s["lens"]), _ints(s["lens"]), _ints(s["cap"])
        s["dout"] = torch.empty((n, b, hq, d), device="cuda")
        size = sonic.decode_q4_workspace_bytes(b, hq, d, s["max_ctx"], case["weights"]) if kind == "decode_q4" else \
            sonic.decode_weighted_workspace_bytes(b, hq, d, s["max_ctx"])
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
        if case["weights"]:
            s["weight"] = torch.empty_like(s["weight0"])
        if kind == "decode_q4":
            s["new_off"], s["new_cap"] = _ints(_starts([n] * b), torch.int64), _ints([n] * b)
            s["ko"], s["vo"] = bf16(b * n), bf16(b * n)
        s["graph"] = _capture(lambda: _own_steps(s, sonic))
    return s


# ------------------------------------------------------------------ one pass, this library's calls
def _ok(code):
    if code != 0:
        raise RuntimeError("status %d" % code)


def _own_steps(s, sonic):
    case = s["case"]
    torch.add(s["len0"], 0, out=s["length"])   # each pass generates from the same contexts
    if case["weights"]:
        torch.add(s["weight0"], 0, out=s["weight"])
    for t in range(case["steps"]):
        if case["kind"] == "decode_q4":
            _ok(sonic.compressed_decode_q4(s["k"], s["ks"], s["v"], s["vs"], s["row_off"], s["cap_dev"], s["length"], s["dq"][t],
                                           s["dk"][t], s["dv"][t], s["dout"][t], s["ws"], s["status"], s["max_ctx"],
                                           row_weight=s.get("weight")))
        else:
            _ok(sonic.compressed_decode_weighted(s["k"], s["v"], s["row_off"], s["cap_dev"], s["length"], s["dq"][t], s["dk"][t],
                                                 s["dv"][t], s["dout"][t], s["weight"], s["ws"], s["status"], s["max_ctx"]))
    if case["kind"] == "decode_q4":            # the rows appended, as a program reads them back
        _ok(sonic.cache_expand_q4(s["k"], s["ks"], s["v"], s["vs"], s["row_off"], s["cap_dev"], s["len0"], s["length"], s["ko"], s["vo"],
                                  s["new_off"], s["new_cap"], s["status"], case["steps"]))


def _run_own(s):
    from paper_2601_21927_amd import sonic
    case, kind = s["case"], s["case"]["kind"]
    if kind == "compact_q4":
        k, ks, v, vs = s["planes"]
        _ok(sonic.kv_compact_q4(s["cu"], s["role"], s["k"], s["v"], k, ks, v, vs, s["row_off"], s["cap_dev"], s["length"],
                                s["keep_idx"], s["status"], max(s["lens"])))
        _ok(sonic.cache_expand_q4(k, ks, v, vs, s["row_off"], s["cap_dev"], s["zero"], s["length"], s["ko"], s["vo"], s["row_off"],
                                  s["cap_dev"], s["status"], max(s["kept"])))
        return {"k": s["ko"], "v": s["vo"], "length": s["length"], "index": s["keep_idx"]}
    if kind == "evict":
        if case["prompt"]:
            _ok(sonic.kv_compact_weights(s["cu"], s["key_weight"], s["row_off"], s["length"], s["index"], s["weight"], s["status"],
                                         s["max_rows"]))
        o = s["out"]
        _ok(sonic.cache_evict(s["k"], s["v"], s["row_off"], s["length"], s["weight"], s["head"], s["tail"], s["budget"], s["ws"],
                              s["status"], s["max_rows"], k_scale=s.get("ks"), v_scale=s.get("vs"), k_out=o["k"], v_out=o["v"],
                              k_scale_out=o.get("ks"), v_scale_out=o.get("vs"), out_row_off=s["out_row_off"],
                              out_row_cap=s["out_cap"], out_len=s["out_len"], out_weight=s["out_weight"], keep_idx=s["out_index"]))
        k, v = o["k"], o["v"]
        if case["rows"] == "q4":
            _ok(sonic.cache_expand_q4(k, o["ks"], v, o["vs"], s["out_row_off"], s["out_cap"], s["zero"], s["out_len"], s["ko"], s["vo"],
                                      s["out_row_off"], s["out_cap"], s["status"], max(s["kept"])))
            k, v = s["ko"], s["vo"]
        return {"k": k, "v": v, "weight": s["out_weight"], "length": s["out_len"], "index": s["out_index"]}
    s["graph"].replay()
    got = {"decoded": s["dout"], "length": s["length"]}
    got["k"], got["v"] = (s["ko"], s["vo"]) if kind == "decode_q4" else (s["k"], s["v"])
    if case["weights"]:
        got["weight"] = s["weight"]
    return got


# ------------------------------------------------------------------ one pass, plain form
def _attend(q, k, v):
    """q [Hq, d]; k, v [n, Hkv, d] -> (out [Hq, d], each row's weight averaged over the q-heads [n])."""
    (hq, d), hkv = q.shape, k.shape[1]
    qg = q.view(hkv, hq // hkv, d)
    p = torch.softmax(torch.matmul(qg, k.permute(1, 2, 0).contiguous()) * d ** -0.5, -1)
    return torch.matmul(p, v.permute(1, 0, 2).contiguous()).reshape(hq, d), p.sum((0, 1)) / hq


def _run_decode(s):
    case = s["case"]
    q4, n = case["kind"] == "decode_q4", case["steps"]
    out = torch.empty(s["dq"].shape, device="cuda")
    weight = s["weight0"].clone() if case["weights"] else None
    for t in range(n):
        new = [s["dk"][t], s["dv"][t]]
        if q4:
            new = [part for x in new for part in _codes(x)]
        for b, (o, length) in enumerate(zip(s["off"], s["lens"])):
            o, e = int(o), int(o) + length + t
            for name, x in zip(("k", "ks", "v", "vs") if q4 else ("k", "v"), new):
                s[name][e] = x[b]
            if q4:
                k, v = _values(s["k"][o:e + 1], s["ks"][o:e + 1]), _values(s["v"][o:e + 1], s["vs"][o:e + 1])
            else:
                k, v = s["k"][o:e + 1].float(), s["v"][o:e + 1].float()
            out[t, b], w = _attend(s["dq"][t, b].float(), k, v)
            if weight is not None:
                weight[o:e] += w[:-1]
                weight[e] = w[-1]
    got = {"decoded": out, "length": _ints([x + n for x in s["lens"]])}
    if q4:
        rows = torch.cat([torch.arange(int(o) + x, int(o) + x + n, device="cuda") for o, x in zip(s["off"], s["lens"])])
        got["k"], got["v"] = (_values(s[c][rows], s[c + "s"][rows]).to(torch.bfloat16) for c in ("k", "v"))
    else:
        got["k"], got["v"] = s["k"], s["v"]
    if weight is not None:
        got["weight"] = weight
    return got


def _run_evict(s):
    case = s["case"]
    budget = case["ctx_max"] * case["budget_pct"] // 100
    weight = s.get("weight")
    if case["prompt"]:
        first = torch.repeat_interleave(_ints(s["cu_host"][:-1]), _ints(s["lens"]))
        weight = s["key_weight"][s["index"] + first]
    rows, index = [], []
    for o, n in zip(s["off"], s["lens"]):
        o = int(o)
        h = min(case["head"], n)
        t = min(case["tail"], n - h)
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        if n > budget:
            order = torch.sort(weight[o + h:o + n - t], descending=True, stable=True).indices
            keep[h + order[max(budget - h - t, 0):]] = False
        kept = torch.nonzero(keep).flatten()
        rows.append(kept + o)
        index.append(kept.int())
    rows = torch.cat(rows)
    if case["rows"] == "q4":
        k, v = (_values(s[c][rows], s[c + "s"][rows]).to(torch.bfloat16) for c in ("k", "v"))
    else:
        k, v = s["k"][rows], s["v"][rows]
    return {"k": k, "v": v, "weight": weight[rows], "length": _ints(x.numel() for x in index), "index": torch.cat(index)}


def run(s):
    if own:
        return _run_own(s)
    if s["case"]["kind"] == "compact_q4":
        rows = torch.nonzero(s["role"] != TEXT).flatten()
        first = torch.repeat_interleave(_ints(s["cu_host"][:-1]), _ints(s["kept"]))
        k, v = (_values(*_codes(s[c][rows])).to(torch.bfloat16) for c in ("k", "v"))
        return {"k": k, "v": v, "length": _ints(s["kept"]), "index": rows.int() - first}
    return _run_evict(s) if s["case"]["kind"] == "evict" else _run_decode(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, b, hq, hkv, d = (case[n] for n in ("kind", "batch", "q_heads", "kv_heads", "head_dim"))
    lens = _lengths(case)
    wide, packed = hkv * d * 4, hkv * (d + d // 16)        # bytes of K and V of one row: bf16, 4 bits
    if kind == "compact_q4":
        period, keep = 100, case["keep_pct"]
        kept = sum(n // period * keep + min(n % period, keep) + int((n - 1) % period >= keep) for n in lens)
        return {"bytes": sum(lens) + kept * (2 * wide + packed + 4), "flops": 0}
    if kind == "evict":
        kept = sum(_kept(case))
        row = packed if case["rows"] == "q4" else wide
        moved = kept * (row + (wide if case["rows"] == "q4" else row) + 8)
        return {"bytes": moved + sum(lens) * (8 if case["prompt"] else 4), "flops": 0}
    row = packed if kind == "decode_q4" else wide
    total = {"bytes": 0, "flops": 0}
    for t in range(case["steps"]):
        seen = sum(n + t + 1 for n in lens)
        total["bytes"] += seen * row + b * (hq * d * 6 + wide) + (8 * seen if case["weights"] else 0)
        total["flops"] += 4 * hq * d * seen
    return total


# ------------------------------------------------------------------ the outputs in 64 bits
def _exact_rounded(x):
    """A 4-bit row's values of x [..., d], from the definition."""
    y = x.double().unflatten(-1, (-1, 32))
    fraction, exponent = torch.frexp(y.abs().amax(-1, keepdim=True))   # max|x| = fraction * 2^exponent, 7 = 0.875 * 2^3
    e = (exponent - torch.where(fraction <= 0.875, 3, 2)).clamp(-127, 125)
    step = torch.ldexp(torch.ones((), dtype=torch.float64, device=x.device), e)
    u = (y / step).abs()
    # borders halfway between neighbours; the one above an odd code's lower neighbour belongs to the even code
    level = torch.zeros_like(u)
    for i in range(7):
        border, gap = (GRID[i] + GRID[i + 1]) / 2, GRID[i + 1] - GRID[i]
        level += gap * ((u > border) | ((u == border) if i % 2 else torch.zeros_like(u, dtype=torch.bool)))
    return (torch.copysign(level, y) * step).flatten(-2)


def _exact_cache(codes, scales):
    """The values of given 4-bit rows: the code's sign, exponent and one fraction bit, read as numbers."""
    code = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    sign, expo, frac = 1.0 - 2.0 * (code // 8).double(), code // 2 % 4, (code % 2).double()
    size = torch.where(expo == 0, frac / 2, (1 + frac / 2) * torch.ldexp(torch.ones((), dtype=torch.float64, device=codes.device), expo - 1))
    two = torch.ldexp(torch.ones((), dtype=torch.float64, device=codes.device), scales.long() - 127)
    return (sign * size).unflatten(-1, (-1, 32)).mul(two[..., None]).flatten(-2)


def _exact_steps(s, case):
    q4, n, hkv, d = case["kind"] == "decode_q4", case["steps"], case["kv_heads"], case["head_dim"]
    group = case["q_heads"] // hkv
    out = torch.empty(s["dq"].shape, dtype=torch.float64, device="cuda")
    new = [_exact_rounded(x) if q4 else x.double() for x in (s["dk"], s["dv"])]
    weight = s["weight0"].double() if case["weights"] else None
    for b, (o, length) in enumerate(zip(s["off"], s["lens"])):
        o = int(o)
        k, v = (torch.cat([_exact_cache(s[c][o:o + length], s[c + "s"][o:o + length]) if q4 else s[c][o:o + length].double(), x[:, b]])
                for c, x in zip(("k", "v"), new))
        for t in range(n):
            m = length + t + 1
            total = torch.zeros(m, dtype=torch.float64, device="cuda")
            for h in range(case["q_heads"]):
                score = torch.mv(k[:m, h // group], s["dq"][t, b, h].double()) / d ** 0.5
                p = torch.exp(score - score.max())
                p /= p.sum()
                out[t, b, h] = torch.mv(v[:m, h // group].t(), p)
                total += p
            if weight is not None:
                total /= case["q_heads"]
                weight[o:o + m - 1] += total[:-1]
                weight[o + m - 1] = total[-1]
    got = {"decoded": out, "length": _ints([x + n for x in s["lens"]])}
    if q4:
        got["k"], got["v"] = (x.transpose(0, 1).flatten(0, 1) for x in new)
    else:
        got["k"], got["v"] = (s[c].double() for c in ("k", "v"))
        for name, x in zip(("k", "v"), new):
            for b, (o, length) in enumerate(zip(s["off"], s["lens"])):
                got[name][int(o) + length:int(o) + length + n] = x[:, b]
    if weight is not None:
        got["weight"] = weight
    return got


def _exact_evict(s, case):
    weight = s["weight"] if not case["prompt"] else torch.cat(
        [s["key_weight"][int(c):][s["index"][int(o):int(o) + n].long()] for c, o, n in zip(s["cu_host"], s["off"], s["lens"])])
    rows, index = [], []
    budget = case["ctx_max"] * case["budget_pct"] // 100
    host = weight.cpu().numpy()
    for o, n in zip(s["off"], s["lens"]):
        o = int(o)
        h = min(case["head"], n)
        t = min(case["tail"], n - h)
        kept = np.arange(n)
        if n > budget:
            middle = np.arange(h, n - t)
            best = middle[np.lexsort((middle, -host[o + h:o + n - t].astype(np.float64)))][:max(budget - h - t, 0)]
            kept = np.sort(np.concatenate([np.arange(h), best, np.arange(n - t, n)]))
        rows.append(kept + o)
        index.append(kept)
    length = [len(x) for x in index]
    rows = torch.from_numpy(np.concatenate(rows)).cuda()
    if case["rows"] == "q4":
        k, v = (_exact_cache(s[c][rows], s[c + "s"][rows]) for c in ("k", "v"))
    else:
        k, v = s["k"][rows].double(), s["v"][rows].double()
    return {"k": k, "v": v, "weight": weight[rows].double(), "length": _ints(length),
            "index": torch.from_numpy(np.concatenate(index)).cuda().int()}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "compact_q4":
        role = s["role"].cpu().numpy()
        index = [np.flatnonzero(role[a:a + n] != TEXT) for a, n in zip(s["cu_host"], s["lens"])]
        rows = torch.from_numpy(np.concatenate([i + int(a) for i, a in zip(index, s["cu_host"])])).cuda()
        k, v = (_exact_rounded(s[c][rows]) for c in ("k", "v"))
        return {"k": k, "v": v, "length": _ints(len(i) for i in index),
                "index": torch.from_numpy(np.concatenate(index)).cuda().int()}
    return _exact_evict(s, case) if case["kind"] == "evict" else _exact_steps(s, case)
