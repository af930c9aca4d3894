"""The operators between the query, key and value projections and the output projection of
a transformer block, as cases that can be timed and compared.

``listed()`` names twelve cases, ``draw(rng)`` makes one more of the same ranges. A case has a
``kind`` (what is called), its sizes, storage type and options:

* ``rope``: rotary positions of queries and keys, one or several position axes; with ``train``
  the rotation back of their gradients;
* ``norm_rope``: MS-RMSNorm of each head of queries and keys and the rotation in one pass, with
  or without a gain per column; with ``train`` its backward;
* ``attention``: softmax(scale q k^T) v, causal or not, grouped heads, sequences that are dense
  (one length), packed one behind the other, or at the front of a padded cache; with ``train``
  its backward;
* ``block``: the three on the fused output of a block's projections, as one module, forward and
  backward.

``heads`` / ``kv_heads`` count query and key heads, ``dim`` is a head's width. ``lengths`` (and
``key_lengths``) are the sequences' lengths, as a text. Causal: the last query sees the last key.
"""

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
EPS = 1e-5
BASE = 10000.0


def listed():
    return [
        # One token of LLaMA-7B while it is generated: queries and keys rotated, all latency.
        {"name": "rope_decode_1", "kind": "rope", "dtype": "bf16", "tokens": 1, "heads": 32, "kv_heads": 32, "dim": 128,
         "rotated": 128, "axes": 1, "interleaved": False, "far": 4000, "train": False},
        # LLaMA-7B fine-tuning, 4 sequences of 2048, queries and keys inside the fused projection's output.
        {"name": "rope_llama7b_train", "kind": "rope", "dtype": "bf16", "tokens": 4 * 2048, "heads": 32, "kv_heads": 32,
         "dim": 128, "rotated": 128, "axes": 1, "interleaved": False, "far": 0, "train": True},
        # Video patches (time, height, width) of a ViT-B-wide model, 32 bits, interleaved pairs, part of each head.
        {"name": "rope_video_fp32", "kind": "rope", "dtype": "fp32", "tokens": 8 * 197, "heads": 12, "kv_heads": 12,
         "dim": 64, "rotated": 60, "axes": 3, "interleaved": True, "far": 0, "train": True},
        # LLaMA-7B's sizes with a norm of each head and no gain: its backward from the rotated output.
        {"name": "norm_rope_llama7b_train", "kind": "norm_rope", "dtype": "bf16", "tokens": 4 * 2048, "heads": 32,
         "kv_heads": 32, "dim": 128, "rotated": 128, "axes": 1, "interleaved": False, "far": 0, "train": True,
         "gain": False},
        # Grouped heads of an odd width with gains, far positions, a ragged number of tokens.
        {"name": "norm_rope_odd_gain_train", "kind": "norm_rope", "dtype": "fp32", "tokens": 1531, "heads": 10,
         "kv_heads": 2, "dim": 72, "rotated": 36, "axes": 2, "interleaved": False, "far": 1000000, "train": True,
         "gain": True},
        # One image of ViT-B, evaluation.
        {"name": "attention_vit_b_image", "kind": "attention", "dtype": "bf16", "form": "dense", "lengths": "197",
         "key_lengths": "197", "heads": 12, "kv_heads": 12, "dim": 64, "causal": False, "train": False},
        # ViT-B fine-tuning, 64 images.
        {"name": "attention_vit_b_bs64_train", "kind": "attention", "dtype": "bf16", "form": "dense",
         "lengths": ",".join(["197"] * 64), "key_lengths": ",".join(["197"] * 64), "heads": 12, "kv_heads": 12,
         "dim": 64, "causal": False, "train": True},
        # One new token of 16 sequences, each at the front of its part of a padded cache.
        {"name": "attention_decode_16", "kind": "attention", "dtype": "bf16", "form": "cache",
         "lengths": ",".join(["1"] * 16),
         "key_lengths": "4096,17,2048,1000,3333,1,511,4095,129,2500,64,1777,900,3000,4000,250",
         "heads": 32, "kv_heads": 32, "dim": 128, "causal": True, "train": False},
        # One new token behind one long sequence, grouped heads: work only along the keys.
        {"name": "attention_decode_long", "kind": "attention", "dtype": "bf16", "form": "cache", "lengths": "1",
         "key_lengths": "65537", "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "train": False},
        # Fine-tuning on packed sequences of different lengths, grouped heads.
        {"name": "attention_packed_train", "kind": "attention", "dtype": "bf16", "form": "packed",
         "lengths": "1500,333,1,2048,700,95,1285,64,2001,165", "key_lengths": "1500,333,1,2048,700,95,1285,64,2001,165",
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "train": True},
        # A LLaMA-7B block's attention in fine-tuning: rotation and attention on 4 sequences of 2048.
        {"name": "block_llama7b_train", "kind": "block", "dtype": "bf16", "form": "dense",
         "lengths": "2048,2048,2048,2048", "key_lengths": "2048,2048,2048,2048", "heads": 32, "kv_heads": 32, "dim": 128,
         "rotated": 128, "axes": 1, "interleaved": False, "far": 0, "norm": False, "causal": True, "train": True},
        # One long document, grouped heads.
        {"name": "attention_long_train", "kind": "attention", "dtype": "bf16", "form": "dense", "lengths": "16384",
         "key_lengths": "16384", "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "train": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = ((32, 32), (32, 8), (40, 40), (12, 12), (16, 2), (6, 3), (8, 1), (5, 5))


def _rotation_of(rng, dim):
    axes = rng.choice((1, 1, 2, 3))
    rotated = dim if rng.random() < 0.6 else max(2, 2 * rng.randint(1, dim // 2))
    return {"rotated": rotated, "axes": axes, "interleaved": rng.random() < 0.4,
            "far": rng.choice((0, 0, 5000, 1000000))}


def _lengths(rng, count, longest, total):
    """Lengths spread over their logarithm, their sum at most ``total``."""
    out = []
    for _ in range(count):
        out.append(_log_int(rng, 1, max(1, min(longest, total - (count - len(out))))))
        total -= out[-1]
        if total <= count - len(out):
            break
    return out


def _text(lengths):
    return ",".join(str(n) for n in lengths)


def draw(rng):
    kind = rng.choice(("rope", "norm_rope", "norm_rope", "attention", "attention", "attention", "attention", "block"))
    heads, kv_heads = rng.choice(_HEADS)
    if kind in ("rope", "norm_rope"):
        dim = rng.choice((64, 80, 96, 128, 128, 72, 2 * rng.randint(2, 120)))
        case = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "fp32")), "heads": heads, "kv_heads": kv_heads,
                "dim": dim, **_rotation_of(rng, dim), "train": rng.random() < 0.7}
        case["tokens"] = _log_int(rng, 1, max(2, min(16384, 60_000_000 // ((heads + kv_heads) * dim))))
        if kind == "norm_rope":
            case["gain"] = rng.random() < 0.5
        return case
    dim = rng.choice((64, 128, 128, 80, 96, 8 * rng.randint(2, 16)))
    case = {"kind": kind, "dtype": "bf16", "heads": heads, "kv_heads": kv_heads, "dim": dim}
    if kind == "block":
        form = rng.choice(("dense", "packed"))
        lengths = [_log_int(rng, 16, 2048)] * rng.randint(1, 4) if form == "dense" else _lengths(rng, rng.randint(1, 10), 2048, 6000)
        return dict(case, form=form, lengths=_text(lengths), key_lengths=_text(lengths), **_rotation_of(rng, dim),
                    norm=rng.random() < 0.5, causal=rng.random() < 0.7, train=True)
    form = rng.choice(("dense", "packed", "packed", "cache"))
    if form == "dense":
        n = _log_int(rng, 1, 4096)
        lengths = [n] * _log_int(rng, 1, max(1, min(64, 12288 // n)))
        keys = lengths if rng.random() < 0.7 else [n + _log_int(rng, 1, 4096)] * len(lengths)
        train = rng.random() < 0.6
    elif form == "packed":
        lengths = _lengths(rng, _log_int(rng, 1, 64), 4096, 12288)
        keys = lengths if rng.random() < 0.7 else [n + rng.randint(0, 500) for n in lengths]
        train = rng.random() < 0.6
    else:
        n = rng.choice((1, 1, 1, rng.randint(2, 16)))
        lengths = [n] * _log_int(rng, 1, 64)
        longest = min(65536, 400_000 // len(lengths))
        keys = [n + _log_int(rng, 1, longest) for _ in lengths]
        train = False
    return dict(case, form=form, lengths=_text(lengths), key_lengths=_text(keys),
                causal=form == "cache" or rng.random() < 0.7, train=train)


def _numbers(text):
    return [int(n) for n in text.split(",")]


# ------------------------------------------------------------------------- inputs

def _normal(gen, shape, std, dtype):
    return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * std).to(DTYPES[dtype])


def _frequencies(case):
    """The angle per position of every pair, and the axis whose position it takes (equal shares, in turn)."""
    pairs = case["rotated"] // 2
    return [BASE ** (-i / pairs) for i in range(pairs)], [i * case["axes"] // pairs for i in range(pairs)]


def _positions(gen, case, lengths):
    """[tokens], or [axes, tokens] of several axes: counted from the sequence's start, or a grid's."""
    count = sum(lengths)
    step = torch.cat([torch.arange(n, device=DEVICE) for n in lengths])
    far = int(torch.randint(case["far"] // 2, case["far"], (1,), generator=gen, device=DEVICE)) if case["far"] > 1 else 0
    if case["axes"] == 1:
        return step + far
    side = max(1, int(math.sqrt(count)))
    grid = (step // side, step % side) if case["axes"] == 2 else (step // (side * 4), step // 4 % side, step % side)
    return torch.stack(grid) + far


def _starts(lengths):
    out = torch.zeros(len(lengths) + 1, dtype=torch.int32)
    out[1:] = torch.tensor(lengths, dtype=torch.int64).cumsum(0)
    return out.to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, dtype, dim = case["kind"], case["dtype"], case["dim"]
    heads, kv_heads = case["heads"], case["kv_heads"]
    state = {"case": case}
    if kind in ("rope", "norm_rope"):
        n = case["tokens"]
        # what the fused projection of queries, keys and values gives; the values are not touched
        qkv = _normal(gen, (n, heads + 2 * kv_heads, dim), 1.0, dtype)
        state["q"], state["k"] = qkv[:, :heads], qkv[:, heads:heads + kv_heads]
        state["positions"] = _positions(gen, case, [n])
        state["frequencies"], state["pair_axes"] = _frequencies(case)
        if kind == "norm_rope" and case["gain"]:
            state["q_gain"] = _normal(gen, (dim,), 0.3, dtype) + 1.0
            state["k_gain"] = _normal(gen, (dim,), 0.3, dtype) + 1.0
        if case["train"]:
            state["dq"] = _normal(gen, (n, heads, dim), 1e-3, dtype)
            state["dk"] = _normal(gen, (n, kv_heads, dim), 1e-3, dtype)
        return state
    lengths, keys = _numbers(case["lengths"]), _numbers(case["key_lengths"])
    state["lengths"], state["keys"] = lengths, keys
    total, total_k = sum(lengths), sum(keys)
    if kind == "block":
        qkv = _normal(gen, (total, heads + 2 * kv_heads, dim), 1.0, dtype)
        state["qkv"] = qkv.requires_grad_()
        state["positions"] = _positions(gen, case, lengths)
        state["frequencies"], state["pair_axes"] = _frequencies(case)
        state["do"] = _normal(gen, (total, heads, dim), 1e-3, dtype)
        state["starts"] = _starts(lengths) if case["form"] == "packed" else None
        return state
    if case["form"] == "cache":
        # a cache with room for the longest sequence; what lies behind a sequence is left from earlier ones
        room = max(keys) + 7
        state["q"] = _normal(gen, (len(lengths), lengths[0], heads, dim), 1.0, dtype)
        state["k"] = _normal(gen, (len(lengths), room, kv_heads, dim), 1.0, dtype)
        state["v"] = _normal(gen, (len(lengths), room, kv_heads, dim), 1.0, dtype)
        state["key_lens"] = torch.tensor(keys, dtype=torch.int32, device=DEVICE)
        return state
    shape = (total,) if case["form"] == "packed" else (len(lengths), lengths[0])
    shape_k = (total_k,) if case["form"] == "packed" else (len(keys), keys[0])
    state["q"] = _normal(gen, (*shape, heads, dim), 1.0, dtype)
    state["k"] = _normal(gen, (*shape_k, kv_heads, dim), 1.0, dtype)
    state["v"] = _normal(gen, (*shape_k, kv_heads, dim), 1.0, dtype)
    if case["form"] == "packed":
        state["starts"], state["key_starts"] = _starts(lengths), _starts(keys)
    if case["train"]:
        state["do"] = _normal(gen, (*shape, heads, dim), 1e-3, dtype)
    return state


# ---------------------------------------------------------------- the plain form

def _plain_angles(state):
    """cos and sin of every token's pairs, [tokens, 1, pairs]: the angles in 64 bits."""
    positions = state["positions"]
    positions = positions if positions.dim() == 2 else positions[None]
    axes = torch.tensor(state["pair_axes"], device=DEVICE, dtype=torch.int64)
    freqs = torch.tensor(state["frequencies"], device=DEVICE, dtype=torch.float64)
    angle = positions[axes].t().double() * freqs
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _plain_turn(x, cos, sin, interleaved):
    pairs = cos.shape[-1]
    r = x[..., :2 * pairs]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :pairs], r[..., pairs:])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((c, d), -1).flatten(-2) if interleaved else torch.cat((c, d), -1)
    return torch.cat((turned, x[..., 2 * pairs:]), -1)


def _plain_rope(case, state, out):
    t, side = DTYPES[case["dtype"]], case["interleaved"]
    cos, sin = _plain_angles(state)
    for name in ("q", "k"):
        out[name] = _plain_turn(state[name].float(), cos, sin, side).to(t)
        if case["train"]:
            out["d" + name] = _plain_turn(state["d" + name].float(), cos, -sin, side).to(t)
    return out


def _plain_norm_rope(case, state, out):
    t, side = DTYPES[case["dtype"]], case["interleaved"]
    cos, sin = _plain_angles(state)
    for name in ("q", "k"):
        x = state[name].float()
        rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        z = x * rstd
        gain = state[name + "_gain"].float() if case["gain"] else None
        out[name] = _plain_turn(z if gain is None else z * gain, cos, sin, side).to(t)
        out["rstd_" + name] = rstd[..., 0]
        if case["train"]:
            g = _plain_turn(state["d" + name].float(), cos, -sin, side)
            if gain is None:
                dz, z = g, _plain_turn(out[name].float(), cos, -sin, side)   # from the output that was kept
            else:
                dz = g * gain
                out[name + "_gain"] = (g * z).sum((0, 1)).to(t)
            out["d" + name] = (rstd * (dz - z * (z * dz).mean(-1, keepdim=True))).to(t)
    return out


def _plain_attend(q, k, v, do, causal):
    """One or more sequences of one length, [n, heads, rows, dim] in 32 bits: o, lse, and with do
    dq, dk, dv."""
    n, heads, rows, dim = q.shape
    kv_heads, cols = k.shape[1], k.shape[2]
    group = heads // kv_heads
    q = q.reshape(n, kv_heads, group * rows, dim)
    scale = dim ** -0.5
    s = (q @ k.transpose(-1, -2)) * scale
    if causal:
        at = torch.arange(rows, device=q.device) + (cols - rows)
        hidden = torch.arange(cols, device=q.device)[None] > at[:, None]
        s = s.view(n, kv_heads, group, rows, cols).masked_fill_(hidden, -math.inf).view(n, kv_heads, group * rows, cols)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    p = s.div_(total)
    o = p @ v
    lse = (top + torch.log(total)).view(n, heads, rows)
    if do is None:
        return o.view(n, heads, rows, dim), lse
    do = do.reshape(n, kv_heads, group * rows, dim)
    dv = p.transpose(-1, -2) @ do
    ds = do @ v.transpose(-1, -2)
    # the row's share, from the output as it is kept
    ds.sub_((do * o.to(torch.bfloat16).float()).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = ds @ k, ds.transpose(-1, -2) @ q
    return o.view(n, heads, rows, dim), lse, dq.view(n, heads, rows, dim), dk, dv


def _groups(state, heads):
    """(first sequence, first row, first key row, sequences, rows, keys): runs of sequences of the same
    lengths, each so small that its scores fit."""
    lengths, keys = state["lengths"], state["keys"]
    out, at, row, key = [], 0, 0, 0
    while at < len(lengths):
        n, m = lengths[at], keys[at]
        most = max(1, (1 << 28) // (heads * n * m))
        count = 1
        while at + count < len(lengths) and count < most and (lengths[at + count], keys[at + count]) == (n, m):
            count += 1
        out.append((at, row, key, count, n, m))
        at, row, key = at + count, row + count * n, key + count * m
    return out


def _plain_attention(case, state, q, k, v, do):
    """q, k, v (and do) in their storage type, rows of all sequences one behind the other."""
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    o = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device)
    grads = [torch.empty(t.shape, dtype=torch.float32, device=q.device) for t in (q, k, v)] if do is not None else []
    for _, row, key, count, n, m in _groups(state, heads):
        rows, cols = slice(row, row + count * n), slice(key, key + count * m)
        share = max(1, min(kv_heads, (1 << 28) // (count * group * n * m)))   # key heads at a time
        for h in range(0, kv_heads, share):
            hk = slice(h, min(kv_heads, h + share))
            hq = slice(hk.start * group, hk.stop * group)

            def part(t, at, size, which):
                return t[at, which].float().reshape(count, size, -1, dim).transpose(1, 2).contiguous()

            got = _plain_attend(part(q, rows, n, hq), part(k, cols, m, hk), part(v, cols, m, hk),
                                None if do is None else part(do, rows, n, hq), case["causal"])
            o[rows, hq] = got[0].transpose(1, 2).reshape(count * n, -1, dim)
            lse[rows, hq] = got[1].transpose(1, 2).reshape(count * n, -1)
            if do is not None:
                grads[0][rows, hq] = got[2].transpose(1, 2).reshape(count * n, -1, dim)
                grads[1][cols, hk] = got[3].transpose(1, 2).reshape(count * m, -1, dim)
                grads[2][cols, hk] = got[4].transpose(1, 2).reshape(count * m, -1, dim)
    return o, lse, grads


def _used(state, name):
    """The rows of the sequences in a padded cache, one behind the other."""
    return torch.cat([state[name][i, :n] for i, n in enumerate(state["keys"])])


def _plain_block(case, state):
    heads, kv_heads, t = case["heads"], case["kv_heads"], DTYPES[case["dtype"]]
    qkv = state["qkv"].detach()
    inner = dict(state, q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads])
    inner_case = dict(case, gain=False, train=False)
    turned = (_plain_norm_rope if case["norm"] else _plain_rope)(inner_case, inner, {})
    o, _, (dq, dk, dv) = _plain_attention(case, state, turned["q"], turned["k"], qkv[:, heads + kv_heads:], state["do"])
    cos, sin = _plain_angles(state)
    parts = []
    for name, d in (("q", dq), ("k", dk)):
        g = _plain_turn(d, cos, -sin, case["interleaved"])
        if case["norm"]:
            z = _plain_turn(turned[name].float(), cos, -sin, case["interleaved"])
            g = turned["rstd_" + name][..., None] * (g - z * (z * g).mean(-1, keepdim=True))
        parts.append(g)
    return {"o": o.to(t), "dqkv": torch.cat((*parts, dv), 1).to(t)}


def _plain(state):
    case = state["case"]
    kind, t = case["kind"], DTYPES[case["dtype"]]
    if kind == "rope":
        return _plain_rope(case, state, {})
    if kind == "norm_rope":
        return _plain_norm_rope(case, state, {})
    if kind == "block":
        return _plain_block(case, state)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["form"] == "cache":
        k, v = _used(state, "k"), _used(state, "v")
    else:
        k, v = state["k"].view(-1, kv_heads, dim), state["v"].view(-1, kv_heads, dim)
    do = state["do"].view(-1, heads, dim) if case["train"] else None
    o, lse, grads = _plain_attention(case, state, state["q"].view(-1, heads, dim), k, v, do)
    out = {"o": o.to(t).view(state["q"].shape), "lse": lse.view(state["q"].shape[:-1])}
    for name, g in zip(("q", "k", "v"), grads):
        out["d" + name] = g.to(t).view(state[name].shape)
    return out


# ------------------------------------------------------------- the framework's calls

def _calls(state):
    import paper_2406_16282_amd as lmbp
    case = state["case"]
    kind = case["kind"]
    if "frequencies" in state and "rotation" not in state:   # a user's program builds it once, with the model
        state["rotation"] = lmbp.Rotation(state["frequencies"], state["pair_axes"], case["interleaved"])
    if kind == "rope":
        out = {}
        out["q"], out["k"] = lmbp.rope_fwd(state["q"], state["k"], state["positions"], state["rotation"])
        if case["train"]:
            out["dq"], out["dk"] = lmbp.rope_bwd(state["dq"], state["dk"], state["positions"], state["rotation"])
        return out
    if kind == "norm_rope":
        gains = (state["q_gain"], state["k_gain"]) if case["gain"] else (None, None)
        q, k, rstd_q, rstd_k = lmbp.msrms_rope_fwd(state["q"], state["k"], EPS, state["positions"], state["rotation"], *gains)
        out = {"q": q, "k": k, "rstd_q": rstd_q, "rstd_k": rstd_k}
        if case["train"]:
            kept = (state["q"], state["k"]) if case["gain"] else (q, k)
            got = lmbp.msrms_rope_bwd(state["dq"], state["dk"], *kept, rstd_q, rstd_k, state["positions"], state["rotation"],
                                      *gains)
            out["dq"], out["dk"] = got[:2]
            if case["gain"]:
                out["q_gain"], out["k_gain"] = got[2:]
        return out
    if kind == "block":
        from paper_2406_16282_amd import nn as lnn
        if "module" not in state:   # as well
            state["module"] = lnn.QKVAttention(case["heads"], case["kv_heads"], case["dim"], state["rotation"],
                                               causal=case["causal"], eps=EPS if case["norm"] else None)
        qkv = state["qkv"] if case["form"] == "packed" else state["qkv"].view(len(state["lengths"]), -1, *state["qkv"].shape[1:])
        positions = state["positions"]
        if case["form"] != "packed":
            positions = positions.view(*positions.shape[:-1], *qkv.shape[:2])
        o = state["module"](qkv, positions, state["starts"])
        (dqkv,) = torch.autograd.grad(o, state["qkv"], state["do"].view(o.shape))
        return {"o": o.detach().view(state["do"].shape), "dqkv": dqkv}
    if case["form"] == "cache":
        where = {"k_lens": state["key_lens"]}
    else:
        where = {"q_starts": state["starts"], "k_starts": state["key_starts"]} if case["form"] == "packed" else {}
    o, lse = lmbp.attention_fwd(state["q"], state["k"], state["v"], causal=case["causal"], **where)
    out = {"o": o, "lse": lse}
    if case["train"]:
        out["dq"], out["dk"], out["dv"] = lmbp.attention_bwd(state["do"], state["q"], state["k"], state["v"], o, lse,
                                                             causal=case["causal"], **where)
    return out


def run(state):
    if own:
        return _calls(state)
    with torch.no_grad():
        return _plain(state)


def _pairs(case):
    """Queries times the keys that each sees, over all sequences."""
    total = 0
    for n, m in zip(_numbers(case["lengths"]), _numbers(case["key_lengths"])):
        total += n * m - (n * (n - 1) // 2 if case["causal"] else 0)
    return total


def work(case):
    kind, e, dim = case["kind"], BYTES[case["dtype"]], case["dim"]
    heads, kv_heads = case["heads"], case["kv_heads"]
    if kind in ("rope", "norm_rope"):
        rows = case["tokens"] * (heads + kv_heads)
        size, at = rows * dim, case["tokens"] * case["axes"] * 8
        total, ops = 2 * size * e + at, 3 * size
        if case["train"]:
            total, ops = total + 2 * size * e + at, ops + 3 * size
        if kind == "norm_rope":
            total, ops = total + 4 * rows, ops + 3 * size
            if case["train"]:
                total, ops = total + size * e + 4 * rows, ops + 6 * size
            if case["gain"]:
                total += 2 * dim * e * (3 if case["train"] else 1)
        return {"bytes": total, "flops": ops}
    rows, cols = sum(_numbers(case["lengths"])), sum(_numbers(case["key_lengths"]))
    q, kv, product = rows * heads * dim * e, cols * kv_heads * dim * e, 2 * dim * heads * _pairs(case)
    total, ops = 2 * q + 2 * kv + 4 * rows * heads, 2 * product
    if case["train"]:
        total, ops = total + 4 * q + 4 * kv + 4 * rows * heads, ops + 5 * product
    if kind == "block":
        total += 2 * 2 * (q + kv) + 2 * 8 * rows * case["axes"]   # the rotation there and back
    return {"bytes": total, "flops": ops}


# ---------------------------------------------------------------------- in 64 bits

def _exact_rotate(x, positions, frequencies, pair_axes, interleaved, back):
    """Every pair as a complex number, times e^(i angle)."""
    pairs = len(frequencies)
    pos = positions if positions.dim() == 2 else positions.unsqueeze(0)
    unit = torch.tensor(frequencies, dtype=torch.float64, device=x.device)
    which = torch.tensor(pair_axes, dtype=torch.int64, device=x.device)
    angle = torch.index_select(pos, 0, which).to(torch.float64).transpose(0, 1) * unit
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle).unsqueeze(1)
    index = torch.arange(pairs, device=x.device)
    first, second = (2 * index, 2 * index + 1) if interleaved else (index, index + pairs)
    value = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    y = x.clone()
    y[..., first] = value.real
    y[..., second] = value.imag
    return y


def _exact_heads(case, state, name, d, kept):
    """(y, rstd, dx, dgain) of queries or keys in 64 bits; d: the gradient of y or None; kept: the output as
    it is held, which the backward without gain starts from, or None for y itself."""
    def turn(t, back):
        return _exact_rotate(t, state["positions"], state["frequencies"], state["pair_axes"], case["interleaved"], back)

    x = state[name].to(torch.float64)
    if case["kind"] == "rope" or not case.get("norm", True):
        return turn(x, False), None, None if d is None else turn(d, True), None
    rstd = torch.pow((x * x).sum(dim=-1) / x.shape[-1] + EPS, -0.5)
    z = x * rstd.unsqueeze(-1)
    gain = state[name + "_gain"].to(torch.float64) if case.get("gain") else None
    y = turn(z if gain is None else z * gain, False)
    if d is None:
        return y, rstd, None, None
    g = turn(d, True)
    dgain = None
    if gain is not None:
        dgain = (g * z).sum(dim=1).sum(dim=0)
        g = g * gain
    elif kept is not None:
        z = turn(kept.to(torch.float64), True)
    along = (z * g).sum(dim=-1, keepdim=True) / z.shape[-1]
    return y, rstd, (g - along * z) * rstd.unsqueeze(-1), dgain


def _exact_head(q, k, v, do, causal):
    """One query head of one sequence, [rows, dim] in 64 bits."""
    rows, cols = q.shape[0], k.shape[0]
    scores = torch.mm(q, k.t().contiguous()) / math.sqrt(q.shape[1])
    if causal:
        keep = torch.ones((rows, cols), dtype=torch.bool, device=q.device).tril(cols - rows)
        scores = torch.where(keep, scores, torch.full((), -math.inf, dtype=torch.float64, device=q.device))
    lse = torch.logsumexp(scores, dim=1)
    p = torch.exp(scores - lse.unsqueeze(1))
    o = torch.mm(p, v)
    if do is None:
        return o, lse, None, None, None
    kept = o.to(torch.bfloat16).to(torch.float64)       # the output as the backward finds it
    ds = p * (torch.mm(do, v.t().contiguous()) - (do * kept).sum(dim=1, keepdim=True)) / math.sqrt(q.shape[1])
    return o, lse, torch.mm(ds, k), torch.mm(ds.t().contiguous(), q), torch.mm(p.t().contiguous(), do)


def _exact_attention(case, lengths, keys, q, k, v, do):
    heads, group = case["heads"], case["heads"] // case["kv_heads"]
    q, k, v = (t.to(torch.float64) for t in (q, k, v))
    do = do.to(torch.float64) if do is not None else None
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    row = key = 0
    for n, m in zip(lengths, keys):
        a, b = slice(row, row + n), slice(key, key + m)
        for h in range(heads):
            got = _exact_head(q[a, h], k[b, h // group], v[b, h // group], None if do is None else do[a, h], case["causal"])
            o[a, h], lse[a, h] = got[:2]
            if do is not None:
                dq[a, h] = got[2]
                dk[b, h // group] += got[3]
                dv[b, h // group] += got[4]
        row, key = row + n, key + m
    return o, lse, dq, dk, dv


def exact(case, seed):
    state = prepare(case, seed)
    kind, t = case["kind"], DTYPES[case["dtype"]]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    with torch.no_grad():
        if kind in ("rope", "norm_rope"):
            out = {}
            for name in ("q", "k"):
                d = state["d" + name].to(torch.float64) if case["train"] else None
                kept = _exact_heads(case, state, name, None, None)[0].to(t) if case["train"] else None
                y, rstd, dx, dgain = _exact_heads(case, state, name, d, kept)
                out[name] = y
                if rstd is not None:
                    out["rstd_" + name] = rstd
                if dgain is not None:
                    out[name + "_gain"] = dgain
                if dx is not None:
                    out["d" + name] = dx
            return out
        lengths, keys = state["lengths"], state["keys"]
        if kind == "block":
            qkv = state["qkv"].detach()
            inner = dict(state, q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads])
            v = qkv[:, heads + kv_heads:]
            held = [_exact_heads(case, inner, name, None, None)[0].to(t) for name in ("q", "k")]   # as attention finds them
            o, _, dq, dk, dv = _exact_attention(case, lengths, keys, *held, v, state["do"])
            parts = [_exact_heads(case, inner, name, d, y)[2] for name, d, y in (("q", dq, held[0]), ("k", dk, held[1]))]
            return {"o": o, "dqkv": torch.cat((*parts, dv), dim=1)}
        if case["form"] == "cache":
            k, v = (torch.cat([state[name][i, :n] for i, n in enumerate(keys)]) for name in ("k", "v"))
        else:
            k, v = (state[name].reshape(-1, kv_heads, dim) for name in ("k", "v"))
        do = state["do"].reshape(-1, heads, dim) if case["train"] else None
        o, lse, dq, dk, dv = _exact_attention(case, lengths, keys, state["q"].reshape(-1, heads, dim), k, v, do)
        shape = state["q"].shape
        out = {"o": o.reshape(shape), "lse": lse.reshape(shape[:-1])}
        if case["train"]:
            out.update(dq=dq.reshape(shape), dk=dk.reshape(state["k"].shape), dv=dv.reshape(state["v"].shape))
        return out
