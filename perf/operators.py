"""Timed cases of the operators around the sparse layer: what a transformer layer runs before its attention
(head norm, rotary positions with several axes, token order) and attention over packed sequences (whole
prompts and clips, one new token over a cache, a training step), each in a plain form and through the library.

``own`` False: the operators' plain form, elementary torch operations in 32 bits (angles in 64), rounded once
at the end.  ``own`` True: the calls a user makes of ``paper_2608_02504_b200.api``.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EPS = 1e-6
_THETA = 10000.0
_SCORES = 1 << 27          # plain form: scores held at a time (fp32)


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # -- head norm + rotary positions + token order ------------------------------------------------
        # smallest grid of the package's configurations: launch latency
        dict(name="rotary_tiny_grid", op="rotary", dir="fwd", dtype="bf16", batch=1, T=4, H=8, W=8, n_text=0,
             tile_h=4, tile_w=4, block=64, tokens=0, pos_max=0, heads=2, kv_heads=2, d=64, norm="rms", halves=False),
        # one layer of the 75.6K-token shape, from a fused projection to tile-major Q, K, V
        dict(name="rotary_720p_layer", op="rotary", dir="fwd", dtype="bf16", batch=1, T=21, H=45, W=80, n_text=0,
             tile_h=8, tile_w=16, block=128, tokens=0, pos_max=0, heads=40, kv_heads=40, d=128, norm="rms",
             halves=False),
        # its gradient on the 32.7K-token shape with text behind the video, weights' gradients included
        dict(name="rotary_480p_text_backward", op="rotary", dir="bwd", dtype="bf16", batch=1, T=21, H=30, W=52,
             n_text=77, tile_h=8, tile_w=16, block=128, tokens=0, pos_max=0, heads=12, kv_heads=12, d=128, norm="rms",
             halves=False),
        # packed prompts with far positions, grouped heads, channels paired across the halves, layer norm
        dict(name="rotary_packed_positions", op="rotary", dir="fwd", dtype="fp16", batch=1, T=0, H=0, W=0, n_text=0,
             tile_h=0, tile_w=0, block=0, tokens=16381, pos_max=1000000, heads=40, kv_heads=8, d=128, norm="layer",
             halves=True),
        # -- attention over packed sequences -----------------------------------------------------------
        # whole prompts of different lengths in one pack, causal, grouped heads
        dict(name="attn_prompts_causal", op="attn", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True,
             lens_q="8192,1,2045,977,128,4096,333,609", lens_k="", slots=0),
        # two clips of the 32.7K-token grid and a shorter one in one pack, every token sees its clip
        dict(name="attn_clips_dense", op="attn", dtype="bf16", heads=12, kv_heads=12, d=128, causal=False,
             lens_q="32760,32760,10921", lens_k="", slots=0),
        # one new token for each of 64 sequences over caches of different lengths
        dict(name="attn_one_token_batch", op="attn", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True,
             lens_q="1*64", lens_k=",".join(str(32768 - 509 * i) for i in range(64)), slots=32768),
        # one new token of one sequence over a short cache: latency
        dict(name="attn_one_token_short", op="attn", dtype="fp16", heads=12, kv_heads=12, d=64, causal=True,
             lens_q="1", lens_k="777", slots=1024),
        # a short chunk of a prompt behind a long cache: few rows, long key axis
        dict(name="attn_chunk_long_cache", op="attn", dtype="bf16", heads=12, kv_heads=2, d=128, causal=True,
             lens_q="97", lens_k="65500", slots=65536),
        # training step (forward and backward) over packed prompts
        dict(name="train_prompts_causal", op="train", dtype="bf16", heads=40, kv_heads=8, d=128, causal=True,
             lens_q="4096,1531,2048,7,510", lens_k="", slots=0),
        # training step over the frames of a 480p clip, each frame a sequence of 1560 tokens
        dict(name="train_frames_dense", op="train", dtype="fp16", heads=12, kv_heads=12, d=64, causal=False,
             lens_q="1560*9", lens_k="", slots=0),
        # training step over a few short prompts: latency
        dict(name="train_short", op="train", dtype="bf16", heads=2, kv_heads=2, d=64, causal=True,
             lens_q="64,37", lens_k="", slots=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["grid", "positions", "attn", "attn", "one", "chunk", "train", "train"])
    d = rng.choice([64, 128])
    if kind == "grid":
        d = rng.choice([64, 128, 128])
        heads = rng.choice([2, 5, 12, 40])
        return dict(op="rotary", dir=rng.choice(["fwd", "bwd"]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    batch=rng.choice([1, 1, 2]), T=_log_int(rng, 1, 13), H=_log_int(rng, 3, 45), W=_log_int(rng, 4, 80),
                    n_text=rng.choice([0, 0, _log_int(rng, 1, 500)]), tile_h=8, tile_w=16, block=128, tokens=0,
                    pos_max=0, heads=heads, kv_heads=heads, d=d, norm=rng.choice(["", "rms", "layer"]),
                    halves=rng.random() < 0.3)
    if kind == "positions":
        kv = rng.choice([1, 2, 8])
        return dict(op="rotary", dir=rng.choice(["fwd", "bwd"]), dtype=rng.choice(["bf16", "fp16", "fp32"]), batch=1,
                    T=0, H=0, W=0, n_text=0, tile_h=0, tile_w=0, block=0, tokens=_log_int(rng, 1, 60000),
                    pos_max=_log_int(rng, 10, 4000000), heads=kv * rng.choice([1, 3, 5]), kv_heads=kv,
                    d=rng.choice([32, 64, 96, 128, 256]), norm=rng.choice(["", "rms", "layer"]),
                    halves=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 1, 2, 3, 5, 6, 8])
    if kind == "one":
        n = _log_int(rng, 1, 100)
        lens = [_log_int(rng, 1, 32000) for _ in range(n)]
        return dict(op="attn", dtype=dtype, heads=kv * group, kv_heads=kv, d=d, causal=True, lens_q=f"1*{n}",
                    lens_k=",".join(map(str, lens)), slots=max(lens) + rng.choice([0, 1, 64]))
    if kind == "chunk":
        n = _log_int(rng, 1, 6)
        lens_q = [_log_int(rng, 1, 300) for _ in range(n)]
        lens_k = [q + _log_int(rng, 1, 40000) for q in lens_q]
        return dict(op="attn", dtype=dtype, heads=kv * group, kv_heads=kv, d=d, causal=rng.random() < 0.8,
                    lens_q=",".join(map(str, lens_q)), lens_k=",".join(map(str, lens_k)), slots=max(lens_k))
    lens = [_log_int(rng, 1, 5000 if kind == "train" else 9000) for _ in range(_log_int(rng, 1, 12))]
    if rng.random() < 0.25:
        lens[rng.randrange(len(lens))] = 0          # a sequence without tokens
    if sum(lens) == 0:
        lens[0] = 17
    return dict(op="train" if kind == "train" else "attn", dtype=dtype, heads=kv * group, kv_heads=kv, d=d,
                causal=rng.random() < 0.6, lens_q=",".join(map(str, lens)), lens_k="", slots=0)


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
def _axis_dims(d):
    """Channels of the time, height and width axis (the split of the package's synthetic embeddings)."""
    side = 2 * (d // 6)
    return d - 2 * side, side, side


def _frequencies(d):
    axis, freq = [], []
    for a, c in enumerate(_axis_dims(d)):
        for k in range(c // 2):
            axis.append(a)
            freq.append(_THETA ** (-2.0 * k / c))
    return axis, freq


def _tile_order(T, H, W, tile_h, tile_w):
    """Raster index of every tile-major position: frame by frame, tile by tile, row-major inside a tile."""
    n = torch.arange(T * H * W, device="cuda")
    t, y, x = n // (H * W), (n // W) % H, n % W
    tiles_y, tiles_x = -(-H // tile_h), -(-W // tile_w)
    key = (((t * tiles_y + y // tile_h) * tiles_x + x // tile_w) * tile_h + y % tile_h) * tile_w + x % tile_w
    return torch.argsort(key)


def _randn(shape, g, dtype, mul=1.0, add=0.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return x.mul_(mul).add_(add).to(dtype)


def _prepare_rotary(case, g):
    dt, d, B = _DTYPES[case["dtype"]], case["d"], case["batch"]
    hq, hk = case["heads"], case["kv_heads"]
    grid = case["T"] > 0
    N = case["T"] * case["H"] * case["W"] + case["n_text"] if grid else case["tokens"]
    st = {"case": case, "order": None, "pos": None, "plan": None, "rot": None}
    qkv = torch.empty(B, N, hq + 2 * hk, d, dtype=dt, device="cuda")          # output of a fused projection
    for b in range(B):
        qkv[b] = _randn((N, hq + 2 * hk, d), g, dt)
    st["qkv"] = (qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:])
    axis, freq = _frequencies(d)
    if grid:
        n = torch.arange(N - case["n_text"], device="cuda")
        W, HW = case["W"], case["H"] * case["W"]
        st["grid_pos"] = torch.stack([n // HW, (n // W) % case["H"], n % W], 1).to(torch.int32)
        order = _tile_order(case["T"], case["H"], W, case["tile_h"], case["tile_w"])
        st["order"] = torch.cat([order, torch.arange(N - case["n_text"], N, device="cuda")])
    else:
        st["pos"] = torch.randint(0, case["pos_max"] + 1, (N, 3), generator=g, device="cuda", dtype=torch.int32)
    st["axis"] = torch.tensor(axis, device="cuda")
    st["freq"] = torch.tensor(freq, device="cuda", dtype=torch.float64)
    w = {}
    if case["norm"]:
        for name in ("q", "k"):
            w[name + "_weight"] = _randn((d,), g, dt, 0.1, 1.0)
            if case["norm"] == "layer":
                w[name + "_bias"] = _randn((d,), g, dt, 0.1)
    st["w"] = w
    if case["dir"] == "bwd":
        shape = (lambda h: (B, h, N, d)) if grid else (lambda h: (B, N, h, d))
        st["grads"] = tuple(_randn(shape(h), g, dt) for h in (hq, hk, hk))
    if own:
        from paper_2608_02504_b200 import api
        st["rot"] = api.Rotary(d, _axis_dims(d), theta=_THETA, halves=case["halves"], norm=case["norm"] or None,
                               eps=_EPS)
        if grid:
            st["plan"] = api.Plan(case["T"], case["H"], case["W"], d if d in (64, 128) else 128, case["block"],
                                  case["tile_h"], case["tile_w"], n_text=case["n_text"])
    return st


def _prepare_attn(case, g):
    dt, d, hq, hk = _DTYPES[case["dtype"]], case["d"], case["heads"], case["kv_heads"]
    lq, lk = _case_lens(case)
    tq = sum(lq)
    if case["slots"]:
        begin = [i * case["slots"] for i in range(len(lk))]
        tk = case["slots"] * len(lk)
    else:
        begin = [sum(lk[:i]) for i in range(len(lk))]
        tk = sum(lk)
    cq = [0]
    for n in lq:
        cq.append(cq[-1] + n)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    st = {"case": case, "lq": lq, "lk": lk, "cq": cq, "begin": begin, "scale": 1.0 / math.sqrt(d),
          "q": _randn((tq, hq, d), g, dt, 1.5), "k": _randn((tk, hk, d), g, dt), "v": _randn((tk, hk, d), g, dt),
          "cu_q": i32(cq), "k_begin": i32(begin), "k_end": i32([b + n for b, n in zip(begin, lk)]),
          "max_q": max(lq), "max_k": max(lk), "attn": None}
    if case["op"] == "train":
        st["do"] = _randn((tq, hq, d), g, dt)
    if own:
        from paper_2608_02504_b200 import api
        st["attn"] = api.PackedAttn(hq, hk, d, dtype=dt, causal=case["causal"])
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return _prepare_rotary(case, g) if case["op"] == "rotary" else _prepare_attn(case, g)


# ----------------------------------------------------------------------------------------- plain forms
def _cos_sin(st):
    pos = st["pos"] if st["pos"] is not None else st["grid_pos"]
    ang = pos.to(torch.float64)[:, st["axis"]] * st["freq"]
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    n_text = st["case"]["n_text"]
    if n_text:                                       # text tokens keep their channels as they are
        cos = torch.cat([cos, torch.ones(n_text, cos.shape[1], device="cuda")])
        sin = torch.cat([sin, torch.zeros(n_text, sin.shape[1], device="cuda")])
    return cos[None, :, None], sin[None, :, None]    # [1, N, 1, d/2]


def _pairs(x, halves):
    d = x.shape[-1]
    return (x[..., :d // 2], x[..., d // 2:]) if halves else (x[..., 0::2], x[..., 1::2])


def _join(a, b, halves):
    return torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2)


def _head_norm(x, norm):
    """(normalised x, 1 / deviation)"""
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
    return x * r, r


def _plain_rotary_forward(st):
    case, outs = st["case"], []
    cos, sin = _cos_sin(st)
    for x, name in zip(st["qkv"], "qkv"):
        dt = x.dtype
        if name != "v":
            x = x.float()
            if case["norm"]:
                x = _head_norm(x, case["norm"])[0] * st["w"][name + "_weight"].float()
                if case["norm"] == "layer":
                    x = x + st["w"][name + "_bias"].float()
            a, b = _pairs(x, case["halves"])
            x = _join(a * cos - b * sin, a * sin + b * cos, case["halves"])
        if st["order"] is not None:
            x = x[:, st["order"]].transpose(1, 2)
        outs.append(x.to(dt).contiguous())
    return outs


def _plain_rotary_backward(st):
    case, (hq, hk) = st["case"], (st["case"]["heads"], st["case"]["kv_heads"])
    cos, sin = _cos_sin(st)
    B, N, _, d = st["qkv"][0].shape
    dqkv = torch.empty(B, N, hq + 2 * hk, d, dtype=st["grads"][0].dtype, device="cuda")
    outs, at = [dqkv], 0
    for x, dy, name in zip(st["qkv"], st["grads"], "qkv"):
        h = x.shape[2]
        if st["order"] is not None:
            back = torch.empty_like(st["order"])
            back[st["order"]] = torch.arange(N, device="cuda")
            dy = dy.transpose(1, 2)[:, back]
        if name != "v":
            a, b = _pairs(dy.float(), case["halves"])
            dy = _join(a * cos + b * sin, b * cos - a * sin, case["halves"])
            if case["norm"]:
                xn, r = _head_norm(x.float(), case["norm"])
                outs.append((dy * xn).sum((0, 1, 2)))
                if case["norm"] == "layer":
                    outs.append(dy.sum((0, 1, 2)))
                g = dy * st["w"][name + "_weight"].float()
                dx = g - xn * (g * xn).mean(-1, keepdim=True)
                if case["norm"] == "layer":
                    dx = dx - g.mean(-1, keepdim=True)
                dy = dx * r
        dqkv[:, :, at:at + h] = dy.to(dqkv.dtype)
        at += h
    return outs


def _blocks(st):
    """(sequence rows of q, rows of k, first query row inside its sequence) of score blocks that fit in memory."""
    case = st["case"]
    group = case["heads"] // case["kv_heads"]
    for s, (lq, lk) in enumerate(zip(st["lq"], st["lk"])):
        if lq == 0:
            continue
        hk = max(1, min(case["kv_heads"], _SCORES // max(1, group * min(lq, 128) * max(lk, 1))))
        step = max(1, min(lq, _SCORES // max(1, group * hk * max(lk, 1))))
        for h in range(0, case["kv_heads"], hk):
            h1 = min(h + hk, case["kv_heads"])
            for i in range(0, lq, step):
                n = min(step, lq - i)
                yield st["cq"][s] + i, n, st["begin"][s], lk, h, h1, lk - lq + i


def _plain_attn_block(st, q0, n, k0, lk, h, h1, first):
    """Scores' softmax of one block: q [h, group * n, d], k, v [h, lk, d], probabilities."""
    case, d = st["case"], st["case"]["d"]
    g = case["heads"] // case["kv_heads"]
    q = st["q"][q0:q0 + n].float().view(n, case["kv_heads"], g, d)[:, h:h1].permute(1, 2, 0, 3).reshape(h1 - h, g * n, d)
    k = st["k"][k0:k0 + lk, h:h1].float().transpose(0, 1)
    v = st["v"][k0:k0 + lk, h:h1].float().transpose(0, 1)
    s = torch.matmul(q, k.transpose(1, 2)).mul_(st["scale"])
    if case["causal"]:
        seen = torch.arange(lk, device="cuda")[None, :] <= (first + torch.arange(n, device="cuda"))[:, None]
        s.view(h1 - h, g, n, lk).masked_fill_(~seen, float("-inf"))
    if lk:
        top = s.amax(-1, keepdim=True)
        p = s.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp_()
        p.div_(p.sum(-1, keepdim=True).clamp_min_(1e-38))
    else:
        p = s
    return q, k, v, p


def _unpack(x, n, h, h1, g):
    return x.view(h1 - h, g, n, -1).permute(2, 0, 1, 3).reshape(n, (h1 - h) * g, -1)


def _plain_attn(st):
    case = st["case"]
    g = case["heads"] // case["kv_heads"]
    o = torch.zeros_like(st["q"])
    for q0, n, k0, lk, h, h1, first in _blocks(st):
        _, _, v, p = _plain_attn_block(st, q0, n, k0, lk, h, h1, first)
        o[q0:q0 + n, h * g:h1 * g] = _unpack(torch.matmul(p, v), n, h, h1, g).to(o.dtype)
    return [o]


def _plain_train(st):
    case = st["case"]
    g = case["heads"] // case["kv_heads"]
    o, dq = torch.zeros_like(st["q"]), torch.zeros_like(st["q"])
    dk, dv = (torch.zeros(st["k"].shape, device="cuda") for _ in range(2))
    for q0, n, k0, lk, h, h1, first in _blocks(st):
        q, k, v, p = _plain_attn_block(st, q0, n, k0, lk, h, h1, first)
        out = torch.matmul(p, v)
        do = st["do"][q0:q0 + n].float().view(n, case["kv_heads"], g, case["d"])[:, h:h1]
        do = do.permute(1, 2, 0, 3).reshape(h1 - h, g * n, case["d"])
        dv[k0:k0 + lk, h:h1] += torch.matmul(p.transpose(1, 2), do).transpose(0, 1)
        ds = torch.matmul(do, v.transpose(1, 2)).sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(st["scale"])
        dk[k0:k0 + lk, h:h1] += torch.matmul(ds.transpose(1, 2), q).transpose(0, 1)
        dq[q0:q0 + n, h * g:h1 * g] = _unpack(torch.matmul(ds, k), n, h, h1, g).to(dq.dtype)
        o[q0:q0 + n, h * g:h1 * g] = _unpack(out, n, h, h1, g).to(o.dtype)
    return [o, dq, dk.to(o.dtype), dv.to(o.dtype)]


# ------------------------------------------------------------------------------------- library's calls
def _own_rotary_backward(st):
    q, k, v = st["qkv"]
    B, N, hq, d = q.shape
    hk = k.shape[2]
    dqkv = torch.empty(B, N, hq + 2 * hk, d, dtype=q.dtype, device="cuda")
    views = (dqkv[:, :, :hq], dqkv[:, :, hq:hq + hk], dqkv[:, :, hq + hk:])
    normed = bool(st["case"]["norm"])
    w = {n: st["w"][n] for n in ("q_weight", "k_weight") if n in st["w"]}
    _, wg = st["rot"].backward(*st["grads"], q=q if normed else None, k=k if normed else None, plan=st["plan"],
                               pos=st["pos"], out=views, **w)
    outs = [dqkv]
    for name in ("q", "k"):
        if st["case"]["norm"]:
            outs.append(wg[name + "_weight"])
        if st["case"]["norm"] == "layer":
            outs.append(wg[name + "_bias"])
    return outs


def run(state):
    case = state["case"]
    if case["op"] == "rotary":
        if not own:
            return _plain_rotary_forward(state) if case["dir"] == "fwd" else _plain_rotary_backward(state)
        if case["dir"] == "bwd":
            return _own_rotary_backward(state)
        return list(state["rot"].forward(*state["qkv"], plan=state["plan"], pos=state["pos"], **state["w"]))
    if not own:
        return _plain_attn(state) if case["op"] == "attn" else _plain_train(state)
    attn, a = state["attn"], (state["q"], state["k"], state["v"])
    if case["op"] == "attn":
        o, _ = attn.forward(*a, state["cu_q"], k_range=(state["k_begin"], state["k_end"]), max_q=state["max_q"],
                            max_k=state["max_k"])
        return [o]
    o, lse = attn.forward(*a, state["cu_q"], max_q=state["max_q"], max_k=state["max_k"], want_lse=True)
    return [o, *attn.backward(state["do"], *a, o, lse, state["cu_q"], max_q=state["max_q"], max_k=state["max_k"])]


# --------------------------------------------------------------------------------------- work and exact
def work(case):
    if case["op"] == "rotary":
        N = case["batch"] * ((case["T"] * case["H"] * case["W"] + case["n_text"]) if case["T"] else case["tokens"])
        size = 4 if case["dtype"] == "fp32" else 2
        rot, all_rows = N * (case["heads"] + case["kv_heads"]), N * (case["heads"] + 2 * case["kv_heads"])
        moved = 2 * all_rows
        if case["dir"] == "bwd" and case["norm"]:
            moved += rot                                       # x again, for the norm's gradient
        flops = rot * case["d"] * (3 + (0 if not case["norm"] else 4 if case["dir"] == "fwd" else 12))
        return {"bytes": moved * case["d"] * size + (0 if case["T"] else 12 * N), "flops": flops}
    lq, lk = _case_lens(case)
    pairs = 0
    for a, b in zip(lq, lk):
        if not case["causal"]:
            pairs += a * b
        else:                                                  # query i sees keys 0 .. i + b - a
            lo, hi = max(0, b - a + 1), b
            n = hi - lo + 1 if a and b else 0
            pairs += n * (lo + hi) // 2
    d, size = case["d"], 2
    rows_q, rows_k = sum(lq) * case["heads"], sum(lk) * case["kv_heads"]
    if case["op"] == "attn":
        return {"bytes": (2 * rows_q + 2 * rows_k) * d * size, "flops": 4 * d * case["heads"] * pairs}
    return {"bytes": (4 * rows_q + 4 * rows_k) * d * size, "flops": 14 * d * case["heads"] * pairs}


def _exact_rotary(st):
    """From the definition: channel pairs as complex numbers, gradients by differentiation."""
    case, d = st["case"], st["case"]["d"]
    pos = (st["pos"] if st["pos"] is not None else st["grid_pos"]).to(torch.float64)
    angle = torch.zeros(st["qkv"][0].shape[1], d // 2, dtype=torch.float64, device="cuda")
    angle[:pos.shape[0]] = pos[:, st["axis"]] * st["freq"]
    turn = torch.polar(torch.ones_like(angle), angle)

    def one(x, weight, bias, rotate):                          # x [n, d] of one head of one batch entry
        if not rotate:
            return x
        if case["norm"] == "rms":
            x = weight * x / torch.sqrt((x ** 2).sum(1, keepdim=True) / d + _EPS)
        elif case["norm"] == "layer":
            mean = x.sum(1, keepdim=True) / d
            x = weight * (x - mean) / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / d + _EPS) + bias
        z = torch.view_as_complex((x.view(-1, 2, d // 2).transpose(1, 2) if case["halves"]
                                   else x.view(-1, d // 2, 2)).contiguous()) * turn
        z = torch.view_as_real(z)
        return (z.transpose(1, 2) if case["halves"] else z).reshape(-1, d)

    outs, grads = [], []
    for i, (x, name) in enumerate(zip(st["qkv"], "qkv")):
        rotate = name != "v"
        w, b = ((st["w"][name + end].double().requires_grad_() if name + end in st["w"] else None)
                for end in ("_weight", "_bias"))
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        wb = [t for t in (w, b) if t is not None]
        total = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in wb]
        for n in range(x.shape[0]):
            for h in range(x.shape[2]):
                xd = x[n, :, h].double()
                if case["dir"] == "fwd":
                    with torch.no_grad():
                        out[n, :, h] = one(xd, w, b, rotate)
                    continue
                xd.requires_grad_()
                dy = st["grads"][i][n, h].double() if st["order"] is not None else st["grads"][i][n, :, h].double()
                y = one(xd, w, b, rotate)
                if st["order"] is not None:
                    y = y[st["order"]]
                got = torch.autograd.grad(y, [xd] + (wb if rotate else []), dy)
                out[n, :, h] = got[0]
                for t, gr in zip(total, got[1:]):
                    t += gr
        outs.append(out)
        if rotate:
            grads += total
    if case["dir"] == "bwd":
        return [torch.cat(outs, 2)] + grads
    return [o if st["order"] is None else o.permute(0, 2, 1, 3)[:, :, st["order"]] for o in outs]


def _exact_attn(st):
    """From the definition, in 64 bits: one head at a time, softmax over the keys a query sees, gradients by
    differentiation."""
    case, train = st["case"], st["case"]["op"] == "train"
    g = case["heads"] // case["kv_heads"]
    f64 = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    o, dq, dk, dv = f64(st["q"]), f64(st["q"]), f64(st["k"]), f64(st["v"])
    for s, (lq, lk) in enumerate(zip(st["lq"], st["lk"])):
        if lq == 0 or lk == 0:
            continue
        keys = slice(st["begin"][s], st["begin"][s] + lk)
        # rows and key heads of one block of scores: about 2^26 of them
        step = max(1, min(lq, (1 << 26) // (g * lk)))
        many = max(1, (1 << 26) // (g * lk * step))
        for h in range(0, case["kv_heads"], many):
            kh = slice(h, min(h + many, case["kv_heads"]))
            qh = slice(kh.start * g, kh.stop * g)
            k, v = (st[n][keys, kh].double().permute(1, 2, 0).requires_grad_(train) for n in "kv")     # [h, d, lk]
            for i in range(0, lq, step):
                n = min(step, lq - i)
                rows = slice(st["cq"][s] + i, st["cq"][s] + i + n)
                q = st["q"][rows, qh].double().requires_grad_(train)
                score = st["scale"] * (q.view(n, -1, g, case["d"]).transpose(0, 1).reshape(-1, n * g, case["d"]) @ k)
                if case["causal"]:
                    row = torch.arange(i, i + n, device="cuda").repeat_interleave(g)
                    hidden = torch.arange(lk, device="cuda")[None] > row[:, None] + (lk - lq)
                    weight = torch.softmax(score.masked_fill(hidden, -1e300), -1).masked_fill(hidden, 0.0)
                else:
                    weight = torch.softmax(score, -1)
                out = (weight @ v.transpose(1, 2)).view(-1, n, g, case["d"]).transpose(0, 1).reshape(n, -1, case["d"])
                o[rows, qh] = out.detach()
                if train:
                    a, b, c = torch.autograd.grad(out, [q, k, v], st["do"][rows, qh].double())
                    dq[rows, qh] = a
                    dk[keys, kh] += b.permute(2, 0, 1)
                    dv[keys, kh] += c.permute(2, 0, 1)
    return [o, dq, dk, dv] if train else [o]


def exact(case, seed):
    w = work(case)
    if case["op"] == "rotary":
        return None if w["bytes"] > 2.5e9 else _exact_rotary(prepare(case, seed))
    return None if w["flops"] > 3e12 else _exact_attn(prepare(case, seed))
