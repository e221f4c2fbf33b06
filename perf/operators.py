"""The 8-bit layer path, operator by operator: what each computes and real sizes of it.

  norm     residual addition, root-mean-square norm and 8-bit rows with a scale per 128 columns
  linear   product of 8-bit rows and 8-bit weights with a scale per block of 128
  append   rotary embedding of queries and keys, keys and values into an 8-bit paged cache with one
           power-of-two scale per (block of 16 tokens, KV head)
  prefill  causal attention of each request's suffix rows over that cache
  decode   attention of one query row per request over that cache

8 bits are e4m3 (largest value 448), rounded to nearest even. Where `own` is true, `run` calls the
framework's operators; else it computes them from elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BS = 16            # tokens per cache block
GROUP = 128        # columns per scale of 8-bit rows, rows and columns per scale of 8-bit weights
FP8_MAX = 448.0
MIN_EXP, MAX_EXP = -100, 120   # exponents of a cache block's scale
EPS = 1e-5
ROPE_BASE = 500000.0
F8 = torch.float8_e4m3fn
HEADS = {  # query heads, KV heads, head_dim, hidden
    "tiny": (4, 1, 64, 256),
    "d64": (16, 4, 64, 1024),
    "qwen7b": (28, 4, 128, 3584),
    "llama8b": (32, 8, 128, 4096),
    "llama70b": (64, 8, 128, 8192),
}


def listed():
    return [
        # One generated token of 16 requests of an 8B server: latency.
        dict(name="norm-decode", op="norm", rows=16, hidden=4096),
        # The 16,128 suffix tokens of the benchmark's trace batch.
        dict(name="norm-trace", op="norm", rows=16128, hidden=4096),
        # The layer's query / key / value projection: 16 generated tokens (the weights' read), one
        # request of a 7B server with a bias, three of five chunks cached, and the trace batch.
        dict(name="linear-decode", op="linear", rows=16, hidden=4096, feats=6144, bias=False),
        dict(name="linear-single-qwen7b", op="linear", rows=576, hidden=3584, feats=4608, bias=True),
        dict(name="linear-trace", op="linear", rows=16128, hidden=4096, feats=6144, bias=False),
        # One new token of 64 requests, most of them in a block that holds others already.
        dict(name="append-decode", op="append", heads="llama8b", batch=64, prefix=1375, suffix=1, spread=True, shape_seed=1),
        # A batch with as many suffix tokens as the trace batch, at ragged lengths.
        dict(name="append-trace", op="append", heads="llama8b", batch=16, prefix=400, suffix=1008, spread=True, shape_seed=2),
        # The smallest batch the framework runs (its smoke test).
        dict(name="prefill-tiny", op="prefill", heads="tiny", batch=1, prefix=64, suffix=32),
        # A ragged batch of a 7B model with seven query heads per KV head, prefixes of any length
        # (a conversation's next turn).
        dict(name="prefill-qwen7b-ragged", op="prefill", heads="qwen7b", batch=6, prefix=700, suffix=411, spread=True,
             shape_seed=3),
        # Ten chunks of 512 tokens with 60 % of the blocks cached.
        dict(name="prefill-topk10", op="prefill", heads="llama8b", batch=8, prefix=3136, suffix=2112),
        # The next token of 16 requests after five chunks of 256, and of 64 requests of a 70B-shaped
        # model after 20 chunks of 512.
        dict(name="decode-16", op="decode", heads="llama8b", batch=16, prefix=1407, suffix=1, spread=True, shape_seed=4),
        dict(name="decode-long", op="decode", heads="llama70b", batch=64, prefix=10367, suffix=1, spread=True, shape_seed=5),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["norm", "linear", "append", "prefill", "decode"])
        if op in ("norm", "linear"):
            case = dict(op=op, rows=log_int(1, 16384), hidden=16 * log_int(4, 512))
            if op == "linear":
                case.update(feats=16 * log_int(4, 512), bias=rng.random() < 0.5)
        else:
            case = dict(op=op, heads=rng.choice(sorted(HEADS)), batch=log_int(1, 64), suffix=1, spread=True,
                        prefix=0 if rng.random() < 0.1 else log_int(1, 10000), shape_seed=rng.randrange(1000))
            if op == "prefill" or (op == "append" and rng.random() < 0.7):
                case["suffix"] = log_int(1, 2500)
        w = work(case)
        if w["flops"] > 8e11 or w["bytes"] > 1.2e9:
            continue
        if op == "prefill":
            s = _Shape(case)   # the plain form's scores of a padded batch
            if s.batch * s.hq * max(s.S) * max(s.L) > 2.5e9:
                continue
        return case


class _Shape:
    """Lengths and heads of a case with a cache; they depend on the case alone."""

    def __init__(self, case):
        self.hq, self.hkv, self.D, self.hidden = HEADS[case["heads"]]
        self.scale = self.D ** -0.5
        self.batch = n = case["batch"]
        r = random.Random(case.get("shape_seed", 0))

        def lengths(mean, least):
            return [max(least, round(mean * r.uniform(0.5, 1.5))) if case.get("spread") and mean > 1 else mean
                    for _ in range(n)]

        self.S, self.P = lengths(case["suffix"], 1), lengths(case["prefix"], 0)
        self.L = [p + s for p, s in zip(self.P, self.S)]
        self.nblk = [-(-length // BS) for length in self.L]
        self.stride = max(self.nblk)
        self.num_blocks = sum(self.nblk) + 5
        self.rows = sum(self.S)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6364136223846793005 % (1 << 62) + 11)
    return g


def _block_table(s, g):
    order = torch.randperm(s.num_blocks, generator=g, device="cuda").to(torch.int32)
    n = torch.tensor(s.nblk, device="cuda")
    first = torch.cumsum(n, 0) - n
    j = torch.arange(s.stride, device="cuda")
    ids = order[(first[:, None] + j).clamp(max=s.num_blocks - 1)]
    return torch.where(j < n[:, None], ids, -1).to(torch.int32).contiguous()


def _cache(s, bt, lengths, g):
    """An 8-bit cache whose used blocks hold keys (or values) of `lengths` tokens; NaN behind them."""
    amp = torch.exp(0.4 * torch.randn(s.num_blocks, s.hkv, 1, 1, generator=g, device="cuda"))
    x = torch.randn(s.num_blocks, s.hkv, BS, s.D, generator=g, device="cuda") * amp
    scale = torch.exp2(_exponent(x.abs().amax((2, 3))))
    code = (x / scale[..., None, None]).to(F8).view(torch.uint8)
    tokens = torch.arange(s.stride * BS, device="cuda").view(s.stride, BS)
    stale = tokens[None] >= torch.tensor(lengths, device="cuda")[:, None, None]   # [batch, block, slot]
    used = bt >= 0
    code[bt[used].long()] = torch.where(stale[used][:, None, :, None], 0x7F, code[bt[used].long()])
    return code.view(F8), scale


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    if case["op"] == "norm":
        T, H = case["rows"], case["hidden"]
        # a residual stream whose rows differ in size, with a few large channels
        channel = torch.exp(torch.randn(H, generator=g, device="cuda") * 0.5)
        size = torch.exp(torch.randn(T, 1, generator=g, device="cuda"))
        st["residual"] = (torch.randn(T, H, generator=g, device="cuda") * channel * size).to(torch.bfloat16)
        st["x"] = normal(T, H)
        st["weight"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(torch.bfloat16)
        st["residual_out"] = torch.empty_like(st["x"])
        st["out8"] = torch.empty(T, H, dtype=F8, device="cuda")
        st["scales"] = torch.empty(T, -(-H // GROUP), device="cuda")
        return st
    if case["op"] == "linear":
        T, K, N = case["rows"], case["hidden"], case["feats"]
        kb, nb = -(-K // GROUP), -(-N // GROUP)
        x = torch.randn(T, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
        w = torch.randn(N, K, generator=g, device="cuda") * K ** -0.5
        w *= torch.exp(0.3 * torch.randn(N, 1, generator=g, device="cuda"))
        st["x_scale"] = _amax(x, 1, GROUP) / FP8_MAX
        st["w_scale"] = _amax(w, GROUP, GROUP) / FP8_MAX
        st["x8"] = (x / _spread(st["x_scale"], 1, GROUP, T, K)).clamp(-FP8_MAX, FP8_MAX).to(F8)
        st["w8"] = (w / _spread(st["w_scale"], GROUP, GROUP, N, K)).clamp(-FP8_MAX, FP8_MAX).to(F8)
        st["bias_row"] = normal(N, std=0.5) if case["bias"] else None
        st["out"] = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
        assert st["x_scale"].shape == (T, kb) and st["w_scale"].shape == (nb, kb)
        return st
    s = _Shape(case)
    st["shape"] = s
    st["bt"] = bt = _block_table(s, g)
    st["prefix_len"] = torch.tensor(s.P, dtype=torch.int32, device="cuda")
    st["seq_len"] = torch.tensor(s.L, dtype=torch.int32, device="cuda")
    st["cu"] = torch.tensor([sum(s.S[:i]) for i in range(s.batch + 1)], dtype=torch.int32, device="cuda")
    held = s.P if case["op"] == "append" else s.L
    st["k8"], st["k_scale"] = _cache(s, bt, held, g)
    st["v8"], st["v_scale"] = _cache(s, bt, held, g)
    if case["op"] == "append":
        st["qkv"] = normal(s.rows, (s.hq + 2 * s.hkv) * s.D)   # what the projection wrote
        half = s.D // 2
        theta = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(max(s.L), dtype=torch.float64, device="cuda")[:, None] * theta
        st["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        st["q_out"] = torch.empty(s.rows, s.hq, s.D, dtype=torch.bfloat16, device="cuda")
    else:
        st["q"] = normal(s.rows, s.hq, s.D)
        st["out"] = torch.empty_like(st["q"])
    if own:
        # what a serving program keeps for the layers of a model: the batch's plan, a workspace
        from paper_2606_19667_amd import cw
        st["cw"] = cw
        st["cache"] = cw.Fp8KvCache.of(st["k8"], st["v8"], st["k_scale"], st["v_scale"])
        if case["op"] == "decode":
            splits = cw.decode_split_count(s.batch, s.hq, s.hkv, s.stride * BS)
            need = cw.decode_workspace_bytes(s.batch, s.hq, s.D, splits)
            st["splits"], st["workspace"] = splits, torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
        else:
            st["meta"] = cw.BatchMeta(bt.cpu().numpy(), st["cu"].cpu().numpy(), s.P, s.hq, s.hkv, s.D)
    return st


# ---------------------------------------------------------------- the plain forms
def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, within the range of a cache block's scale."""
    m, e = torch.frexp(amax)   # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(amax > 0, e, MIN_EXP).clamp(MIN_EXP, MAX_EXP).to(amax.dtype)


def _amax(x, rows, cols):
    """Largest magnitude of each block of rows x cols, ragged at the end."""
    n, k = x.shape
    pad = torch.nn.functional.pad(x.abs(), (0, -k % cols, 0, -n % rows))
    return pad.view(-(-n // rows), rows, -(-k // cols), cols).amax((1, 3))


def _spread(s, rows, cols, n, k):
    """The blocks' scales for each element of an [n, k] matrix."""
    return s.repeat_interleave(rows, 0)[:n].repeat_interleave(cols, 1)[:, :k]


def run(st):
    if own:
        return _run_own(st)
    return {"norm": _plain_norm, "linear": _plain_linear, "append": _plain_append,
            "prefill": _plain_attention, "decode": _plain_attention}[st["op"]](st)


def _plain_norm(st):
    h16 = (st["x"].float() + st["residual"].float()).to(torch.bfloat16)
    h = h16.float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * st["weight"].float()
    scale = _amax(y, 1, GROUP) / FP8_MAX
    scale = torch.where(scale > 0, scale, 1.0)
    q = (y / _spread(scale, 1, GROUP, *y.shape)).clamp(-FP8_MAX, FP8_MAX).to(F8)
    return {"out8": q, "scales": scale, "residual_out": h16}


def _plain_linear(st):
    T, K, N = st["rows"], st["hidden"], st["feats"]
    x = st["x8"].float() * _spread(st["x_scale"], 1, GROUP, T, K)
    w = st["w8"].float() * _spread(st["w_scale"], GROUP, GROUP, N, K)
    y = x @ w.t()
    if st["bias_row"] is not None:
        y = y + st["bias_row"].float()
    return y.to(torch.bfloat16)


def _positions(st):
    """Request and position of each suffix row."""
    s = st["shape"]
    S = (st["cu"][1:] - st["cu"][:-1]).long()
    req = torch.repeat_interleave(torch.arange(s.batch, device="cuda"), S, output_size=s.rows)
    pos = torch.arange(s.rows, device="cuda") - st["cu"][req] + st["prefix_len"][req]
    return req, pos


def _plain_append(st):
    s = st["shape"]
    req, pos = _positions(st)
    y = st["qkv"].float().view(s.rows, s.hq + 2 * s.hkv, s.D)
    c, sn = st["rope"][pos][:, None, :, 0], st["rope"][pos][:, None, :, 1]
    u, half = y[:, :s.hq + s.hkv], s.D // 2
    rot = torch.cat([u[..., :half] * c - u[..., half:] * sn, u[..., half:] * c + u[..., :half] * sn], -1)
    _plain_store(st, "k", req, pos, rot[:, s.hq:])
    _plain_store(st, "v", req, pos, y[:, s.hq + s.hkv:])
    return {"q": rot[:, :s.hq].to(torch.bfloat16), "k8": st["k8"], "v8": st["v8"], "k_scale": st["k_scale"],
            "v_scale": st["v_scale"]}


def _plain_store(st, name, req, pos, rows):
    s = st["shape"]
    code, scale = st[name + "8"].view(torch.uint8), st[name + "_scale"]
    blk = st["bt"][req, pos // BS].long()
    # the distinct blocks that get rows, and the first slot that gets one in each
    new = torch.zeros(s.num_blocks, BS, dtype=torch.bool, device="cuda")
    new[blk, pos % BS] = True
    ids = new.any(1).nonzero()[:, 0]
    new = new[ids]
    at = torch.zeros(s.num_blocks, dtype=torch.long, device="cuda")
    at[ids] = torch.arange(len(ids), device="cuda")
    x = torch.zeros(len(ids), BS, s.hkv, s.D, device="cuda")
    x[at[blk], pos % BS] = rows
    x = x.transpose(1, 2)
    first = new.int().argmax(1)
    need = torch.exp2(_exponent(x.abs().amax((2, 3))))
    had = scale[ids]
    now = torch.where(first[:, None] > 0, torch.maximum(had, need), need)
    old = code[ids]
    ratio = (had / now)[..., None, None]
    kept = torch.where(ratio < 1, (old.view(F8).float() * ratio).to(F8).view(torch.uint8), old)
    slot = torch.arange(BS, device="cuda")
    kept = torch.where((slot < first[:, None])[:, None, :, None], kept, old)
    coded = (x / now[..., None, None]).to(F8).view(torch.uint8)
    code[ids] = torch.where(new[:, None, :, None], coded, kept)
    scale[ids] = now


def _plain_rows(st, name):
    """Every request's keys (or values) in 32 bits, padded: [batch, hkv, stride * 16, D]."""
    s = st["shape"]
    ids = st["bt"].clamp(min=0).long()
    x = st[name + "8"].view(torch.uint8)[ids].view(F8).float() * st[name + "_scale"][ids][..., None, None]
    return x.transpose(1, 2).reshape(s.batch, s.hkv, s.stride * BS, s.D)


def _plain_attention(st):
    s = st["shape"]
    req, pos = _positions(st)
    G, most = s.hq // s.hkv, max(s.S)
    at = pos - st["prefix_len"][req]
    q = torch.zeros(s.batch, most, s.hq, s.D, device="cuda")
    q[req, at] = st["q"].float()
    q = q.view(s.batch, most, s.hkv, G, s.D).permute(0, 2, 3, 1, 4).reshape(s.batch, s.hkv, G * most, s.D)
    keys = torch.arange(s.stride * BS, device="cuda")
    inside = keys < st["seq_len"][:, None]
    k = torch.where(inside[:, None, :, None], _plain_rows(st, "k"), 0.0)
    v = torch.where(inside[:, None, :, None], _plain_rows(st, "v"), 0.0)
    p = (q @ k.transpose(2, 3).contiguous()).mul_(s.scale)
    hidden = keys > st["prefix_len"][:, None, None] + torch.arange(most, device="cuda")[:, None]
    hidden = hidden | ~inside[:, None]
    p.view(s.batch, s.hkv, G, most, -1).masked_fill_(hidden[:, None, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    o = (p @ v) / p.sum(-1, keepdim=True)
    o = o.view(s.batch, s.hkv, G, most, s.D).permute(0, 3, 1, 2, 4).reshape(s.batch, most, s.hq, s.D)
    return o[req, at].to(torch.bfloat16)


# ---------------------------------------------------------------- the framework's operators
def _run_own(st):
    op = st["op"]
    if op in ("norm", "linear"):
        from paper_2606_19667_amd import cw
        if op == "norm":
            cw.add_rms_norm_fp8(st["x"], st["weight"], EPS, residual=st["residual"], residual_out=st["residual_out"],
                                out8=st["out8"], scales=st["scales"])
            return {n: st[n] for n in ("out8", "scales", "residual_out")}
        return cw.fp8_linear(st["x8"], st["x_scale"], st["w8"], st["w_scale"], bias=st["bias_row"], out=st["out"])
    cw, s, cache = st["cw"], st["shape"], st["cache"]
    if op == "append":
        q, k, v = (x.view(s.rows, -1, s.D) for x in st["qkv"].split([s.hq * s.D, s.hkv * s.D, s.hkv * s.D], 1))
        cw.rope_append_fp8(st["meta"], k, v, cache, q=q, rope=st["rope"], q_out=st["q_out"])
        return {"q": st["q_out"], "k8": st["k8"], "v8": st["v8"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    if op == "prefill":
        return cw.suffix_prefill_attn_fp8(st["meta"], st["q"], cache, s.scale, out=st["out"])
    return cw.decode_attn_fp8(st["q"], cache, st["bt"], st["seq_len"], s.scale, num_splits=st["splits"],
                              workspace=st["workspace"], out=st["out"])


# ---------------------------------------------------------------- what they cannot do without
def work(case):
    if case["op"] == "norm":
        T, H = case["rows"], case["hidden"]
        return {"bytes": T * H * 7 + T * -(-H // GROUP) * 4 + 2 * H, "flops": 8 * T * H}
    if case["op"] == "linear":
        T, K, N = case["rows"], case["hidden"], case["feats"]
        kb = -(-K // GROUP)
        return {"bytes": T * K + N * K + 2 * T * N + 4 * kb * (T + -(-N // GROUP)) + 2 * N * bool(case["bias"]),
                "flops": 2 * T * K * N}
    s = _Shape(case)
    if case["op"] == "append":
        return {"bytes": s.rows * s.D * (2 * (s.hq + 2 * s.hkv) + 2 * s.hq + 2 * s.hkv) + max(s.L) * s.D * 4,
                "flops": s.rows * s.D * (3 * (s.hq + s.hkv) + 2 * s.hkv)}
    kv = sum(s.L) * s.hkv * s.D * 2 + sum(s.nblk) * s.hkv * 8
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(s.S, s.P))
    return {"bytes": 4 * s.rows * s.hq * s.D + kv, "flops": 4 * s.D * s.hq * pairs}


# ---------------------------------------------------------------- the definitions in 64 bits
def _e4m3(x):
    """x rounded to an e4m3 value (nearest, ties to even), in 64 bits."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6.0)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-FP8_MAX, FP8_MAX)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h16 = (st["x"].double() + st["residual"].double())
        h = h16.float().to(torch.bfloat16).double()
        y = h / (h.pow(2).mean(1) + EPS).sqrt()[:, None] * st["weight"].double()
        q, scales = torch.empty_like(y), []
        for a in range(0, case["hidden"], GROUP):
            part = y[:, a:a + GROUP]
            top = part.abs().max(1).values / FP8_MAX
            top = torch.where(top == 0, 1.0, top)
            q[:, a:a + GROUP] = _e4m3(part / top[:, None])
            scales.append(top)
        return {"out8": q, "scales": torch.stack(scales, 1), "residual_out": h16}
    if op == "linear":
        y = torch.zeros(case["rows"], case["feats"], dtype=torch.float64, device="cuda")
        for b, a in enumerate(range(0, case["hidden"], GROUP)):
            w = st["w8"][:, a:a + GROUP].double()
            w = w * st["w_scale"][torch.arange(len(w), device="cuda") // GROUP, b].double()[:, None]
            y += (st["x8"][:, a:a + GROUP].double() @ w.t()) * st["x_scale"][:, b].double()[:, None]
        return y + st["bias_row"].double() if case["bias"] else y
    s = st["shape"]
    cu = [sum(s.S[:i]) for i in range(s.batch + 1)]
    bt = st["bt"].tolist()
    if op == "append":
        return _exact_append(st, s, cu, bt)
    out = torch.empty(s.rows, s.hq, s.D, dtype=torch.float64, device="cuda")
    G = s.hq // s.hkv
    for r in range(s.batch):
        L, P = s.L[r], s.P[r]
        ids = torch.tensor(bt[r][:s.nblk[r]], device="cuda")
        keys = torch.arange(L, device="cuda")
        k, v = ((st[n + "8"].view(torch.uint8)[ids].view(F8).double() * st[n + "_scale"][ids].double()[..., None, None])
                .transpose(0, 1).reshape(s.hkv, -1, s.D)[:, :L] for n in "kv")
        step = max(1, (1 << 27) // (s.hq * L))
        for a in range(0, s.S[r], step):
            b = min(s.S[r], a + step)
            for g in range(s.hkv):
                q = st["q"][cu[r] + a:cu[r] + b, g * G:(g + 1) * G].double()
                sc = (q.reshape(-1, s.D) @ k[g].t()).view(b - a, G, L) * s.scale
                sc[(keys > P + torch.arange(a, b, device="cuda")[:, None])[:, None].expand(-1, G, -1)] = -math.inf
                out[cu[r] + a:cu[r] + b, g * G:(g + 1) * G] = (torch.softmax(sc, -1).view(-1, L) @ v[g]).view(-1, G, s.D)
    return out


def _exact_append(st, s, cu, bt):
    half = s.D // 2
    y = st["qkv"].double().view(s.rows, -1, s.D)
    pos = torch.cat([torch.arange(p, p + n) for p, n in zip(s.P, s.S)]).cuda()
    turn = torch.complex(st["rope"][pos, :, 0].double(), st["rope"][pos, :, 1].double())[:, None]
    z = torch.complex(y[:, :s.hq + s.hkv, :half], y[:, :s.hq + s.hkv, half:]) * turn
    y = torch.cat([torch.cat([z.real, z.imag], -1), y[:, s.hq + s.hkv:]], 1)
    res = {"q": y[:, :s.hq]}
    for name, h0 in (("k", s.hq), ("v", s.hq + s.hkv)):
        code, scale = st[name + "8"].double(), st[name + "_scale"].double()
        for r in range(s.batch):
            p = s.P[r]
            while p < s.L[r]:
                end = min(s.L[r], (p // BS + 1) * BS)
                b, a = bt[r][p // BS], p % BS
                rows = y[cu[r] + p - s.P[r]:cu[r] + end - s.P[r], h0:h0 + s.hkv].transpose(0, 1)
                top = rows.abs().amax((1, 2))
                now = torch.exp2(torch.ceil(torch.log2(top / FP8_MAX)).clamp(MIN_EXP, MAX_EXP))
                if a > 0:
                    now = torch.maximum(now, scale[b])
                    code[b, :, :a] = _e4m3(code[b, :, :a] * (scale[b] / now)[:, None, None])
                code[b, :, a:a + end - p] = _e4m3(rows / now[:, None, None])
                scale[b] = now
                p = end
        res[name + "8"], res[name + "_scale"] = code, scale
    return res
