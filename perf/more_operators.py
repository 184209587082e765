"""Timed cases of what a long stream of tokens needs next to attention over packed sequences: a sliding window with a few
first tokens that stay visible (whole prompts, one new token over a cache, training steps), a cache whose keys and
values are quantised to 4 bits as they are written and read back, and attention over that cache; each in a plain
form and through the library.

``own`` False: the operators' plain form, elementary torch operations in 32 bits (64 where a value is rounded to its 4-bit
code), rounded once at the end.  ``own`` True: the calls a user makes of ``paper_2608_02504_b200.api``.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_SCORES = 1 << 26          # plain form: scores held at a time (fp32)
_GROUP = 32                # channels that share a step and a lowest value in the 4-bit cache


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # -- sliding window with first tokens that stay visible ------------------------------------------
        # prompts of different lengths in one pack, grouped heads: prefill of a layer with a window
        dict(name="window_prompts", op="attn", cache="", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True, window=1024,
             sinks=4, lens_q="16384,1,2045,977,128,8192,333,609", lens_k="", slots=0),
        # one new token for each of 32 sequences over caches of different lengths
        dict(name="window_one_token_batch", op="attn", cache="", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True,
             window=4096, sinks=16, lens_q="1*32", lens_k=",".join(str(32768 - 1013 * i) for i in range(32)), slots=32768),
        # training step over packed prompts
        dict(name="window_train_prompts", op="train", cache="", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True, window=512,
             sinks=4, lens_q="8192,1531,2048,7,510", lens_k="", slots=0),
        # training step over a clip of nine 480p frames (1,560 tokens each): the last two frames and the first one stay visible
        dict(name="window_train_frames", op="train", cache="", dtype="fp16", heads=12, kv_heads=12, d=64, causal=True, window=3120,
             sinks=1560, lens_q="14040", lens_k="", slots=0),
        # training step over two short prompts: latency
        dict(name="window_train_short", op="train", cache="", dtype="bf16", heads=2, kv_heads=2, d=64, causal=True, window=16,
             sinks=2, lens_q="64,37", lens_k="", slots=0),
        # -- a cache of 4 bits: written and read back -----------------------------------------------------
        # a packed prompt's keys and values into their slots, and back
        dict(name="cache4_prompt", op="cache", dtype="bf16", kv_heads=8, d=128, tokens=16381, slots=40000),
        # the new tokens of 64 sequences, one each: latency
        dict(name="cache4_tokens", op="cache", dtype="fp16", kv_heads=8, d=128, tokens=64, slots=65536),
        # keys and values of the 32.7K-token clip
        dict(name="cache4_clip", op="cache", dtype="fp16", kv_heads=12, d=64, tokens=32760, slots=32760),
        # -- attention over the cache of 4 bits -----------------------------------------------------------
        # one new token for each of 64 sequences over caches of different lengths
        dict(name="cache4_one_token_batch", op="attn", cache="4", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True, window=0,
             sinks=0, lens_q="1*64", lens_k=",".join(str(32768 - 509 * i) for i in range(64)), slots=32768),
        # one new token of one sequence over a short cache: latency
        dict(name="cache4_one_token_short", op="attn", cache="4", dtype="fp16", heads=12, kv_heads=12, d=64, causal=True, window=0,
             sinks=0, lens_q="1", lens_k="777", slots=1024),
        # a short chunk of a prompt behind a long cache
        dict(name="cache4_chunk_long", op="attn", cache="4", dtype="bf16", heads=12, kv_heads=2, d=128, causal=True, window=0,
             sinks=0, lens_q="97", lens_k="65500", slots=65536),
        # chunks of four prompts behind their caches, with a window
        dict(name="cache4_window_chunks", op="attn", cache="4", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True,
             window=4096, sinks=64, lens_q="1024,700,1024,333", lens_k="9000,16000,1024,12345", slots=16384),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["prompts", "train", "train", "one", "cache", "cache", "one4", "one4", "chunk4", "chunk4"])
    d, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp16"])
    kv = rng.choice([1, 2, 4, 8])
    if kind == "cache":
        tokens = _log_int(rng, 1, 30000)
        return dict(op="cache", dtype=dtype, kv_heads=kv, d=d, tokens=tokens, slots=tokens + _log_int(rng, 1, 20000))
    case = dict(op="train" if kind == "train" else "attn", cache="4" if kind.endswith("4") else "", dtype=dtype,
                heads=kv * rng.choice([1, 1, 2, 3, 5, 6, 8, 12]), kv_heads=kv, d=d, causal=True, window=_log_int(rng, 1, 5000),
                sinks=rng.choice([0, _log_int(rng, 1, 300), _log_int(rng, 1, 16)]))
    if case["cache"] and rng.random() < 0.6:
        case["window"] = case["sinks"] = 0
    if kind in ("one", "one4"):
        lens = [_log_int(rng, 1, 30000) for _ in range(_log_int(rng, 1, 60 if case["cache"] else 30))]
        return dict(case, lens_q=f"1*{len(lens)}", lens_k=",".join(map(str, lens)), slots=max(lens) + rng.choice([0, 1, 64]))
    if kind == "chunk4":
        lens_q = [_log_int(rng, 1, 900) for _ in range(_log_int(rng, 1, 5))]
        lens_k = [q + _log_int(rng, 1, 12000) for q in lens_q]
        return dict(case, lens_q=",".join(map(str, lens_q)), lens_k=",".join(map(str, lens_k)), slots=max(lens_k))
    lens = [_log_int(rng, 1, 5000) for _ in range(_log_int(rng, 1, 8))]
    if rng.random() < 0.25:
        lens[rng.randrange(len(lens))] = 0          # a sequence without tokens
    if sum(lens) == 0:
        lens[0] = 17
    return dict(case, lens_q=",".join(map(str, lens)), lens_k="", slots=0)


def _lens(text):
    out = []
    for part in text.split(","):
        n, _, times = part.partition("*")
        out += [int(n)] * (int(times) if times else 1)
    return out


def _case_lens(case):
    lq = _lens(case["lens_q"])
    return lq, (_lens(case["lens_k"]) if case["lens_k"] else lq)


# --------------------------------------------------------------------------------------------- inputs
def _randn(shape, g, dtype, mul=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(mul).to(dtype)


def _keys_values(n, case, g):
    """Keys whose channels differ in size and have offsets, as keys do behind a projection, and values."""
    hk, d, dt = case["kv_heads"], case["d"], _DTYPES[case["dtype"]]
    size = torch.exp(0.5 * torch.randn((hk, d), generator=g, device="cuda"))
    shift = 0.3 * torch.randn((hk, d), generator=g, device="cuda")
    k = torch.randn((n, hk, d), generator=g, device="cuda").mul_(size).add_(shift)
    return k.to(dt), _randn((n, hk, d), g, dt)


def _prepare_cache(case, g):
    k, v = _keys_values(case["tokens"], case, g)
    room = case["slots"] - case["tokens"]
    if case["tokens"] > 1000:                       # a prompt: one run of slots
        slots = torch.randint(0, room + 1, (1,), generator=g, device="cuda") + torch.arange(case["tokens"], device="cuda")
    else:                                           # new tokens of different sequences
        slots = torch.randperm(case["slots"], generator=g, device="cuda")[:case["tokens"]]
    st = {"case": case, "k": k, "v": v, "slots": slots.to(torch.int32).contiguous(), "cache": None}
    shape = (case["slots"], case["kv_heads"], case["d"])
    if own:
        from paper_2608_02504_b200 import api
        st["cache"] = api.Cache4(api.PackedAttn(case["kv_heads"], case["kv_heads"], case["d"], dtype=k.dtype), case["slots"])
    else:
        for name in "kv":
            st["codes_" + name] = torch.zeros(shape, dtype=torch.uint8, device="cuda")
            st["step_" + name], st["low_" + name] = (torch.zeros(shape[:2] + (shape[2] // _GROUP,), dtype=k.dtype, device="cuda")
                                                     for _ in range(2))
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "cache":
        return _prepare_cache(case, g)
    dt, d, hq, hk = _DTYPES[case["dtype"]], case["d"], case["heads"], case["kv_heads"]
    lq, lk = _case_lens(case)
    cq = [0]
    for n in lq:
        cq.append(cq[-1] + n)
    begin = [i * case["slots"] if case["slots"] else sum(lk[:i]) for i in range(len(lk))]
    tq, tk = sum(lq), case["slots"] * len(lk) if case["slots"] else sum(lk)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    st = {"case": case, "lq": lq, "lk": lk, "cq": cq, "begin": begin, "scale": 1.0 / math.sqrt(d), "q": _randn((tq, hq, d), g, dt),
          "cu_q": i32(cq), "k_begin": i32(begin), "k_end": i32([b + n for b, n in zip(begin, lk)]), "max_q": max(lq),
          "max_k": max(lk), "attn": None}
    if own:
        from paper_2608_02504_b200 import api
        st["attn"] = api.PackedAttn(hq, hk, d, dtype=dt, causal=case["causal"], window=case["window"], sinks=case["sinks"])
    if case["op"] == "train":
        st["do"] = _randn((tq, hq, d), g, dt)
    if not case["cache"]:
        st["k"], st["v"] = _keys_values(tk, case, g)
        return st
    # a cache of 4 bits, filled sequence by sequence
    if own:
        st["cache"] = api.Cache4(st["attn"], tk)
    else:
        for name in "kv":
            st["codes_" + name] = torch.zeros((tk, hk, d), dtype=torch.uint8, device="cuda")
            st["step_" + name], st["low_" + name] = (torch.zeros((tk, hk, d // _GROUP), dtype=dt, device="cuda") for _ in range(2))
    for b, n in zip(begin, lk):
        kv = _keys_values(n, case, g)
        if own:
            st["cache"].write(*kv, torch.arange(b, b + n, dtype=torch.int32, device="cuda"))
        else:
            for name, x in zip("kv", kv):
                codes, step, low = _quantise(x)
                st["codes_" + name][b:b + n], st["step_" + name][b:b + n], st["low_" + name][b:b + n] = codes, step, low
    return st


# ----------------------------------------------------------------------------------------- plain forms
def _quantise(x):
    """Groups of 32 channels: lowest value, step = a fifteenth of the range, rounded up to the tensors' type, and the
    number of steps above the lowest value, rounded to the nearest (halves up)."""
    n, h, d = x.shape
    f = x.float().view(n, h, d // _GROUP, _GROUP)
    lo, hi = f.amin(-1, keepdim=True), f.amax(-1, keepdim=True)
    s = ((0.5 * hi - 0.5 * lo) / 7.5).to(x.dtype)
    s = torch.where(15 * s.double() < hi.double() - lo.double(), (s.view(torch.int16) + 1).view(x.dtype), s)
    t = (f - lo).double() / s.double()
    codes = torch.where(s > 0, torch.floor(t + 0.5), 0.0).to(torch.uint8)
    return codes.view(n, h, d), s.squeeze(-1), lo.squeeze(-1).to(x.dtype)


def _values(codes, step, low):
    """What codes stand for, in 32 bits."""
    n, h, d = codes.shape
    return (codes.float().view(n, h, -1, _GROUP) * step.float()[..., None] + low.float()[..., None]).view(n, h, d)


def _plain_cache(st):
    slots, outs = st["slots"].long(), []
    for name in "kv":
        codes, step, low = _quantise(st[name])
        st["codes_" + name][slots], st["step_" + name][slots], st["low_" + name][slots] = codes, step, low
    for name in "kv":
        outs.append(_values(*(st[part + name][slots] for part in ("codes_", "step_", "low_"))).to(st[name].dtype))
    return outs


def _rows_of(st, name, rows, heads):
    """Keys or values of some rows and heads, in 32 bits."""
    if st["case"]["op"] == "train" or not st["case"]["cache"]:
        return st[name][rows][:, heads].float()
    return _values(*(st[part + name][rows][:, heads] for part in ("codes_", "step_", "low_")))


def _blocks(st):
    """Score blocks that fit in memory: (first row of q, rows, rows of the keys that any of them sees, mask, key/value heads)."""
    case = st["case"]
    group, window, sinks = case["heads"] // case["kv_heads"], case["window"], case["sinks"]
    for s, (lq, lk) in enumerate(zip(st["lq"], st["lk"])):
        most = min(lq, 512 if window else 4096)
        i = 0
        while i < lq:
            n = min(most, lq - i)
            first = i + lk - lq                                # position of the block's first query
            lo = max(first - window + 1, 0) if window else 0
            hi = min(max(first + n, 0), lk)
            lo = min(lo, hi)
            keys = torch.cat([torch.arange(min(sinks, lo), device="cuda"), torch.arange(lo, hi, device="cuda")])
            at = first + torch.arange(n, device="cuda")[:, None]
            seen = keys[None] <= at
            if window:
                seen &= (keys[None] > at - window) | (keys[None] < sinks)
            hk = max(1, min(case["kv_heads"], _SCORES // max(1, group * n * max(len(keys), 1))))
            for h in range(0, case["kv_heads"], hk):
                yield st["cq"][s] + i, n, st["begin"][s] + keys, seen, slice(h, min(h + hk, case["kv_heads"]))
            i += n


def _split(x, n, heads, g):
    """[n, heads * g, d] -> [heads, g * n, d] of some key/value heads"""
    x = x.view(n, -1, g, x.shape[-1])[:, heads]
    return x.permute(1, 2, 0, 3).reshape(x.shape[1], g * n, x.shape[-1]).float()


def _unsplit(x, n, g):
    return x.view(x.shape[0], g, n, -1).permute(2, 0, 1, 3).reshape(n, x.shape[0] * g, -1)


def _plain_attn(st):
    case = st["case"]
    g, train = case["heads"] // case["kv_heads"], case["op"] == "train"
    o = torch.zeros_like(st["q"])
    if train:
        dq = torch.zeros_like(o)
        dk, dv = (torch.zeros(st["k"].shape, device="cuda") for _ in range(2))
    for q0, n, rows, seen, heads in _blocks(st):
        q = _split(st["q"][q0:q0 + n], n, heads, g)
        k, v = (_rows_of(st, name, rows, heads).transpose(0, 1) for name in "kv")
        if not len(rows):
            continue
        p = torch.matmul(q, k.transpose(1, 2)).mul_(st["scale"])
        p.view(-1, g, n, len(rows)).masked_fill_(~seen, float("-inf"))
        top = p.amax(-1, keepdim=True)
        p = p.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp_()
        p.div_(p.sum(-1, keepdim=True).clamp_min_(1e-38))
        out = torch.matmul(p, v)
        q_heads = slice(heads.start * g, heads.stop * g)
        o[q0:q0 + n, q_heads] = _unsplit(out, n, g).to(o.dtype)
        if train:
            do = _split(st["do"][q0:q0 + n], n, heads, g)
            dv[:, heads].index_add_(0, rows, torch.matmul(p.transpose(1, 2), do).transpose(0, 1))
            ds = torch.matmul(do, v.transpose(1, 2)).sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(st["scale"])
            dk[:, heads].index_add_(0, rows, torch.matmul(ds.transpose(1, 2), q).transpose(0, 1))
            dq[q0:q0 + n, q_heads] = _unsplit(torch.matmul(ds, k), n, g).to(o.dtype)
    return [o, dq, dk.to(o.dtype), dv.to(o.dtype)] if train else [o]


# ------------------------------------------------------------------------------------- library's calls
def run(state):
    case = state["case"]
    if not own:
        return _plain_cache(state) if case["op"] == "cache" else _plain_attn(state)
    if case["op"] == "cache":
        state["cache"].write(state["k"], state["v"], state["slots"])
        return list(state["cache"].read(state["slots"]))
    attn, q, cu = state["attn"], state["q"], state["cu_q"]
    sizes = dict(max_q=state["max_q"], max_k=state["max_k"])
    if case["cache"]:
        return [attn.forward_cache4(q, state["cache"], cu, k_range=(state["k_begin"], state["k_end"]), **sizes)[0]]
    k, v = state["k"], state["v"]
    if case["op"] == "attn":
        return [attn.forward(q, k, v, cu, k_range=(state["k_begin"], state["k_end"]), **sizes)[0]]
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **sizes)
    return [o, *attn.backward(state["do"], q, k, v, o, lse, cu, **sizes)]


# --------------------------------------------------------------------------------------- work and exact
def work(case):
    d = case["d"]
    row4 = d // 2 + d // _GROUP * 4                          # bytes of a row in the cache of 4 bits
    if case["op"] == "cache":
        rows = 2 * case["tokens"] * case["kv_heads"]
        return {"bytes": 2 * rows * (2 * d + row4) + 8 * case["tokens"], "flops": 6 * rows * d}
    lq, lk = _case_lens(case)
    pairs = keys = 0
    for a, b in zip(lq, lk):
        if not a or not b:
            continue
        sees = np.clip(np.arange(a, dtype=np.int64) + b - a + 1, 0, b)         # causal
        if case["window"]:
            old = np.maximum(sees - case["window"], 0)                         # keys that have left the window
            sees = sees - old + np.minimum(old, case["sinks"])
            left = max(b - a + 1 - case["window"], 0)                          # keys in front of every query's window
            keys += b - left + min(left, case["sinks"])
        else:
            keys += b
        pairs += int(sees.sum())
    rows_q, rows_k = sum(lq) * case["heads"], keys * case["kv_heads"]
    if case["cache"]:
        return {"bytes": 4 * rows_q * d + 2 * rows_k * row4, "flops": 4 * d * case["heads"] * pairs}
    if case["op"] == "attn":
        return {"bytes": 4 * (rows_q + rows_k) * d, "flops": 4 * d * case["heads"] * pairs}
    return {"bytes": 8 * (rows_q + sum(lk) * case["kv_heads"]) * d, "flops": 14 * d * case["heads"] * pairs}


def _exact_codes(x):
    """(values that 4 bits hold, from the definition in 64 bits), [n, h, d]"""
    f = x.double().unflatten(-1, (-1, _GROUP))
    lo, hi = f.min(-1, keepdim=True).values, f.max(-1, keepdim=True).values
    near = ((hi - lo) / 15).to(x.dtype)                      # to be the smallest number of the type whose 15-fold covers the range
    step = torch.where(15 * near.double() < hi - lo, (near.view(torch.int16) + 1).view(x.dtype), near).double()
    return (lo + step * torch.floor(torch.where(step > 0, (f - lo) / step, 0.0) + 0.5)).flatten(-2)


def _exact_keys_values(case, seed):
    """The keys and values that prepare() made of this seed (its draws in the same order), as the attention reads them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lq, lk = _case_lens(case)
    _randn((sum(lq), case["heads"], case["d"]), g, torch.float32)
    return [tuple(_exact_codes(x) for x in _keys_values(n, case, g)) for n in lk]


def _exact_attn(case, seed):
    """From the definition, in 64 bits: a softmax over the keys that a query sees, one key/value head at a time, gradients by
    differentiation."""
    cached = _exact_keys_values(case, seed) if case["cache"] else None
    plain = prepare(dict(case, cache=""), seed) if not case["cache"] else None
    lq, lk = _case_lens(case)
    train, g = case["op"] == "train", case["heads"] // case["kv_heads"]
    if plain is None:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        q_all = _randn((sum(lq), case["heads"], case["d"]), gen, _DTYPES[case["dtype"]])
    else:
        q_all = plain["q"]
    zero = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    o = zero(q_all)
    if train:
        dq, dk, dv = zero(q_all), zero(plain["k"]), zero(plain["v"])
    row = 0
    for s, (a, b) in enumerate(zip(lq, lk)):
        for h in range(case["kv_heads"] if a and b else 0):
            if cached is not None:
                k_all, v_all = cached[s][0][:, h], cached[s][1][:, h]
            else:
                at = slice(plain["begin"][s], plain["begin"][s] + b)
                k_all, v_all = plain["k"][at, h].double(), plain["v"][at, h].double()
            heads = slice(h * g, (h + 1) * g)
            step = max(1, min(a, 1024, (1 << 25) // (g * min(b, (case["window"] or b) + 1024 + case["sinks"]))))
            for i in range(0, a, step):
                n = min(step, a - i)
                at = torch.arange(i, i + n, device="cuda") + (b - a)           # positions of these queries
                far = int(at[0]) + 1 - case["window"] if case["window"] else 0
                j = torch.arange(b, device="cuda")
                j = j[(j <= int(at[-1])) & ((j >= far) | (j < case["sinks"]))]
                if not len(j):
                    continue
                hidden = j[None] > at[:, None]
                if case["window"]:
                    hidden |= (at[:, None] - j[None] >= case["window"]) & (j[None] >= case["sinks"])
                rows = slice(row + i, row + i + n)
                q = q_all[rows, heads].double().requires_grad_(train)
                k, v = k_all[j].requires_grad_(train), v_all[j].requires_grad_(train)
                score = torch.einsum("nhd,md->hnm", q, k) / math.sqrt(case["d"])
                weight = torch.softmax(score.masked_fill(hidden, -1e300), -1).masked_fill(hidden, 0.0)
                out = torch.einsum("hnm,md->nhd", weight, v)
                o[rows, heads] = out.detach()
                if train:
                    x, y, z = torch.autograd.grad(out, [q, k, v], plain["do"][rows, heads].double())
                    dq[rows, heads] = x
                    dk[plain["begin"][s] + j, h] += y
                    dv[plain["begin"][s] + j, h] += z
        row += a
    return [o, dq, dk, dv] if train else [o]


def exact(case, seed):
    w = work(case)
    if case["op"] == "cache":
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        return [_exact_codes(x) for x in _keys_values(case["tokens"], case, g)]
    return None if w["flops"] > 1.2e12 or (case["cache"] and w["bytes"] > 3e9) else _exact_attn(case, seed)
