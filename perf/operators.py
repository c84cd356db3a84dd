"""The operators of encoders that pack sequences of different lengths, as measurable cases: attention over packed
sequences (causal or not, grouped heads, kept history), norms of queries and keys for each head with the rotation by position in the same
pass, and that rotation alone.

Where `own` is false, `run` computes them from elementary torch operations in 32 bits (angles in 64); where it is true it
makes the calls of the binding.  `exact` states each operator once more in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
GOLDEN = 0.6180339887498949


def listed():
    return [
        # ---- attention over packed sequences
        # one camera on the small embedded model: a frame of 197 tokens, 3 heads; latency and launches count
        {"name": "att_frame_1", "op": "attention", "kind": "frames", "seqs": 1, "shortest": 197, "longest": 197, "heads": 3,
         "kv_heads": 3, "dim": 64, "causal": False, "kept": 0, "pad": 0, "type": "bf16"},
        # cameras of different sizes in one batch, ViT-base heads; the batch is padded to a bucket behind the last frame
        {"name": "att_frames_mixed", "op": "attention", "kind": "frames", "seqs": 64, "shortest": 65, "longest": 577, "heads": 12,
         "kv_heads": 12, "dim": 64, "causal": False, "kept": 0, "pad": 100, "type": "bf16"},
        # whole clips in causal order, grouped heads of 128, ragged: the largest
        {"name": "att_clips_grouped", "op": "attention", "kind": "clips", "seqs": 3, "shortest": 1501, "longest": 8192, "heads": 32,
         "kv_heads": 8, "dim": 128, "causal": True, "kept": 0, "pad": 0, "type": "bf16"},
        # a second of video appended to what four streams have kept
        {"name": "att_clips_appended", "op": "attention", "kind": "clips", "seqs": 4, "shortest": 250, "longest": 985, "heads": 12,
         "kv_heads": 4, "dim": 64, "causal": True, "kept": 4000, "pad": 0, "type": "bf16"},
        # one new token for each of 48 streams with up to 8192 kept ones, in slots of a cache
        {"name": "att_step_streams", "op": "attention", "kind": "step", "seqs": 48, "shortest": 1, "longest": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "causal": True, "kept": 8192, "pad": 0, "type": "bf16"},
        # one new token of one stream with a long history: few rows, a long axis
        {"name": "att_step_one", "op": "attention", "kind": "step", "seqs": 1, "shortest": 1, "longest": 1, "heads": 16,
         "kv_heads": 4, "dim": 128, "causal": True, "kept": 32000, "pad": 0, "type": "bf16"},
        # the debug type
        {"name": "att_frames_fp32", "op": "attention", "kind": "frames", "seqs": 8, "shortest": 50, "longest": 577, "heads": 6,
         "kv_heads": 6, "dim": 64, "causal": False, "kept": 0, "pad": 0, "type": "fp32"},
        # ---- norms of queries and keys with the rotation
        # one frame of the small model
        {"name": "norm_frame_1", "op": "norm", "rows": 196, "heads": 3, "kv_heads": 3, "dim": 64, "norm": "rms", "beta": False,
         "per_head": False, "axes": 2, "interleaved": False, "rot": 64, "base": 100.0, "scaling": "none", "far": 14, "type": "bf16"},
        # the batch of 256 frames on ViT-base, LayerNorm with shift, rotation by row and column of the patch
        {"name": "norm_frames_256", "op": "norm", "rows": 50176, "heads": 12, "kv_heads": 12, "dim": 64, "norm": "layer", "beta": True,
         "per_head": False, "axes": 2, "interleaved": False, "rot": 64, "base": 100.0, "scaling": "none", "far": 14, "type": "bf16"},
        # grouped heads of 128, each with its own weights, in 32 bits
        {"name": "norm_clips_fp32", "op": "norm", "rows": 6011, "heads": 32, "kv_heads": 8, "dim": 128, "norm": "rms", "beta": False,
         "per_head": True, "axes": 1, "interleaved": True, "rot": 128, "base": 10000.0, "scaling": "none", "far": 8192, "type": "fp32"},
        # ---- the rotation alone
        # one token for each of 48 streams, half of the head rotated
        {"name": "rope_step_48", "op": "rope", "rows": 48, "heads": 32, "dim": 128, "axes": 1, "interleaved": False, "rot": 64,
         "base": 10000.0, "scaling": "linear", "far": 30000, "type": "bf16"},
        # far positions of long clips, frequencies scaled by bands
        {"name": "rope_clips_far", "op": "rope", "rows": 32771, "heads": 16, "dim": 128, "axes": 1, "interleaved": True, "rot": 128,
         "base": 500000.0, "scaling": "bands", "far": 1000000, "type": "bf16"},
    ]


def _spread(rng, low, high):
    """An integer of [low, high], spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


LARGEST_FLOPS = 8.5e11              # of the largest listed attention, rounded down; in 32 bits what takes as long
LARGEST_FLOPS_FP32 = 2.5e10
LARGEST_BYTES = 7e8                 # of the listed case that moves most


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "norm", "rope"])
    kind = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "attention":
        what = rng.choice(["frames", "clips", "step"])
        if what == "frames":
            heads = rng.choice([3, 6, 12])
            case = {"seqs": _spread(rng, 1, 256), "shortest": rng.randint(1, 197), "longest": _spread(rng, 197, 785), "heads": heads,
                    "kv_heads": heads, "dim": 64, "causal": False, "kept": 0, "pad": rng.choice([0, 0, 77])}
        elif what == "clips":
            heads, kv_heads = rng.choice([(12, 12), (12, 4), (16, 4), (32, 8), (14, 2), (8, 1), (5, 5)])
            case = {"seqs": _spread(rng, 1, 8), "shortest": _spread(rng, 1, 500), "longest": _spread(rng, 500, 8192), "heads": heads,
                    "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "causal": rng.random() < 0.8, "kept": rng.choice([0, 0, _spread(rng, 1, 8192)]),
                    "pad": 0}
        else:
            heads, kv_heads = rng.choice([(12, 12), (12, 4), (16, 4), (32, 8), (14, 2), (8, 1), (64, 8)])
            case = {"seqs": _spread(rng, 1, 64), "shortest": 1, "longest": rng.choice([1, 1, 2, 5]), "heads": heads,
                    "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "causal": True, "kept": _spread(rng, 100, 32000), "pad": rng.choice([0, 3])}
            case["kept"] = min(case["kept"], 400000 // case["seqs"])
        case = {"op": op, "kind": what, **case, "type": kind}
        top = LARGEST_FLOPS if kind == "bf16" else LARGEST_FLOPS_FP32
        while work(case)["flops"] > top or work(case)["bytes"] > LARGEST_BYTES:
            if case["seqs"] > 1:
                case["seqs"] = (case["seqs"] + 1) // 2
            elif case["kept"] > case["longest"]:
                case["kept"] //= 2
            else:
                case["longest"] = max(case["longest"] * 2 // 3, case["shortest"])
        return case
    dim = rng.choice([64, 128, 128, 80, 256])
    case = {"op": op, "rows": _spread(rng, 1, 40000), "dim": dim, "axes": rng.choice([1, 2]), "interleaved": rng.random() < 0.5,
            "rot": rng.choice([dim, dim, dim // 32 * 16]), "base": rng.choice([100.0, 10000.0, 500000.0]),
            "scaling": rng.choice(["none", "linear", "ntk", "bands"]), "far": _spread(rng, 14, 1000000), "type": kind}
    heads, kv_heads = rng.choice([(3, 3), (6, 6), (12, 12), (16, 4), (32, 8), (14, 2), (5, 1)])
    if op == "norm":
        case.update(heads=heads, kv_heads=kv_heads, norm=rng.choice(["rms", "layer"]), per_head=rng.random() < 0.3)
        case["beta"] = case["norm"] == "layer" and rng.random() < 0.7
        per_row = (heads + kv_heads) * dim
    else:
        case["heads"] = heads
        per_row = heads * dim
    size = 2 if kind == "bf16" else 4
    case["rows"] = max(1, min(case["rows"], int(1.5e8) // (per_row * size)))
    return case


# ---- sizes and plans that follow from the case alone -----------------------------------------------
def _lengths(case):
    """Queries and keys of each sequence.  A step's idle stream (every seventh) has neither."""
    span = case["longest"] - case["shortest"]
    n_q = [case["longest"]] + [case["shortest"] + int(((i * GOLDEN) % 1.0) * (span + 1)) for i in range(1, case["seqs"])]
    kept = [case["kept"]] + [int(((i * GOLDEN * GOLDEN) % 1.0) * (case["kept"] + 1)) for i in range(1, case["seqs"])]
    if case["kind"] == "step":
        n_q = [0 if i % 7 == 3 else n for i, n in enumerate(n_q)]
        kept = [0 if i % 7 == 3 else k for i, k in enumerate(kept)]
    return n_q, [a + b for a, b in zip(n_q, kept)]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _visible(n_q, n_k, causal):
    """(query, key) pairs of a sequence."""
    if not causal:
        return n_q * n_k
    hidden = n_q - 1                                     # the first query does not see the last n_q - 1 keys
    return n_q * n_k - hidden * (hidden + 1) // 2


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "attention":
        n_q, n_k = _lengths(case)
        pairs = sum(_visible(a, b, case["causal"]) for a, b in zip(n_q, n_k))
        rows = 2 * sum(n_q) * case["heads"] + 2 * sum(n_k) * case["kv_heads"]
        return {"bytes": size * case["dim"] * rows, "flops": 4 * case["dim"] * case["heads"] * pairs}
    heads = case["heads"] + case.get("kv_heads", 0)
    elements = case["rows"] * heads * case["dim"]
    rotated = case["rows"] * heads * case["rot"]
    return {"bytes": 2 * size * elements + 4 * case["rows"] * case["axes"],
            "flops": 3 * rotated + (4 * elements if case["op"] == "norm" else 0)}


# ---- what a program holds before the call -----------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table_arguments(case):
    d = {"rot_dim": case["rot"], "base": case["base"], "interleaved": case["interleaved"], "axes": case["axes"], "scaling": case["scaling"]}
    if case["scaling"] != "none":
        d["factor"] = 8.0
    if case["scaling"] == "bands":
        d.update(original=8192, low_turns=1.0, high_turns=4.0, amplitude=1.2)
    return d


def prepare(case, seed):
    g, t = _generator(seed), TYPES[case["type"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    state = {"case": case}
    if case["op"] == "attention":
        n_q, n_k = _lengths(case)
        heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
        q_at = _starts(n_q)
        rows = q_at[-1] + case["pad"]
        state.update(n_q=n_q, n_k=n_k, q_at=q_at, max_q=max(n_q), max_kv=max(n_k), q_offsets=_ints(q_at))
        if case["kind"] == "step":
            # slots of equal size in a cache; what lies behind a stream's length is left from before
            slot = max(n_k)
            state["k_at"] = [slot * i for i in range(len(n_k) + 1)]
            state["kv_lengths"] = _ints(n_k)
        else:
            state["k_at"] = _starts(n_k)
        if case["kept"] == 0 and case["kind"] == "frames":
            # queries, keys and values as one projection leaves them
            qkv = normal(rows, heads + 2 * kv_heads, dim).to(t)
            q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        else:
            state["kv_offsets"] = _ints(state["k_at"])
            q = (2 * normal(rows, heads, dim)).to(t)
            k, v = (normal(state["k_at"][-1], kv_heads, dim).to(t) for _ in range(2))
        state.update(q=q, k=k, v=v, out=torch.zeros((rows, heads, dim), dtype=t, device="cuda"))
        return state
    rows, heads, dim = case["rows"], case["heads"], case["dim"]
    if case["axes"] == 2:
        # row and column of the patch
        at = torch.randint(case["far"], (rows, 2), generator=g, device="cuda")
    else:
        at = torch.randint(case["far"], (rows,), generator=g, device="cuda")
    state["positions"] = at.int()
    if own:
        from paper_2507_14959_b200 import binding
        state["table"] = binding.RopeTable(dim, **_table_arguments(case))
    if case["op"] == "rope":
        state["x"] = normal(rows, heads, dim).to(t)
        state["y"] = torch.empty_like(state["x"])
        return state
    kv_heads = case["kv_heads"]
    qkv = (normal(rows, heads + 2 * kv_heads, dim) * 2 + 0.3).to(t)          # one projection, the values behind
    state.update(qkv=qkv, q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads], q_out=torch.empty((rows, heads, dim), dtype=t, device="cuda"),
                 k_out=torch.empty((rows, kv_heads, dim), dtype=t, device="cuda"))
    for name, n in (("q", heads), ("k", kv_heads)):
        shape = (n, dim) if case["per_head"] else (dim,)
        state[name + "_gamma"] = 1.0 + 0.2 * normal(*shape)
        state[name + "_beta"] = 0.2 * normal(*shape) if case["beta"] else None
    return state


# ---- one pass ---------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    return _run_own(state, case) if own else _run_plain(state, case)


def _run_own(state, case):
    from paper_2507_14959_b200 import binding
    dtype = 0 if case["type"] == "bf16" else 1
    if case["op"] == "attention":
        binding.attention_packed(state["q"], state["k"], state["v"], state["out"], state["q_offsets"], state["max_q"], state["max_kv"], dtype,
                                 kv_offsets=state.get("kv_offsets"), kv_lengths=state.get("kv_lengths"), causal=case["causal"])
        return state["out"]
    if case["op"] == "rope":
        binding.rope(state["x"], state["y"], state["positions"], state["table"], dtype)
        return state["y"]
    binding.qk_norm_rope(state["q"], state["k"], state["q_out"], state["k_out"], state["q_gamma"], state["k_gamma"], norm=case["norm"], eps=1e-6,
                         dtype=dtype, q_beta=state["q_beta"], k_beta=state["k_beta"], positions=state["positions"], table=state["table"])
    return {"q": state["q_out"], "k": state["k_out"]}


def _run_plain(state, case):
    if case["op"] == "attention":
        return _attention_plain(state, case)
    cos, sin = _angles_plain(state["positions"], case)
    if case["op"] == "rope":
        return _rotate_plain(state["x"].float(), cos, sin, case).to(state["x"].dtype)
    out = {}
    for name in ("q", "k"):
        x = state[name].float()
        if case["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * state[name + "_gamma"]
        if case["beta"]:
            x = x + state[name + "_beta"]
        out[name] = _rotate_plain(x, cos, sin, case).to(state[name].dtype)
    return out


def _attention_plain(state, case):
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    out = torch.zeros_like(state["out"])
    for s, (n_q, n_k) in enumerate(zip(state["n_q"], state["n_k"])):
        if n_q == 0 or n_k == 0:
            continue
        a, b = state["q_at"][s], state["k_at"][s]
        step = max(1, 2 ** 29 // (group * n_q * n_k))    # K/V heads at once
        hidden = None
        if case["causal"]:
            hidden = torch.arange(n_k, device="cuda") > torch.arange(n_q, device="cuda")[:, None] + (n_k - n_q)
        for h in range(0, kv_heads, step):
            e = min(h + step, kv_heads)
            q = state["q"][a:a + n_q, h * group:e * group].float().transpose(0, 1).reshape(e - h, group, n_q, dim)
            k = state["k"][b:b + n_k, h:e].float().transpose(0, 1)
            v = state["v"][b:b + n_k, h:e].float().transpose(0, 1)
            scores = (q.reshape(e - h, group * n_q, dim) @ k.transpose(1, 2)).view(e - h, group, n_q, n_k) * dim ** -0.5
            if hidden is not None:
                scores.masked_fill_(hidden, -math.inf)
            p = torch.exp(scores - scores.amax(-1, keepdim=True))
            o = (p.view(e - h, group * n_q, n_k) @ v).view(e - h, group, n_q, dim) / p.sum(-1, keepdim=True)
            out[a:a + n_q, h * group:e * group] = o.reshape((e - h) * group, n_q, dim).transpose(0, 1).to(out.dtype)
    return out


def _angles_plain(positions, case):
    """cos and sin of every row's pairs, [rows, 1, rot / 2] in 32 bits from angles in 64."""
    pairs = case["rot"] // 2
    each = pairs // case["axes"]
    j = torch.arange(each, device="cuda", dtype=torch.float64)
    base = torch.tensor(case["base"], device="cuda", dtype=torch.float64)
    if case["scaling"] == "ntk" and each > 1:
        base = base * 8.0 ** (each / (each - 1))
    freq = base ** (-j / each)
    amplitude = 1.0
    if case["scaling"] == "linear":
        freq = freq / 8.0
    if case["scaling"] == "bands":
        turns = 8192 * freq / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / 8.0)
        amplitude = 1.2
    p = positions.double().view(-1, case["axes"], 1)
    angle = (p * freq).reshape(len(p), 1, pairs)
    return (amplitude * angle.cos()).float(), (amplitude * angle.sin()).float()


def _rotate_plain(x, cos, sin, case):
    rot = case["rot"]
    y = x.clone()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    return y


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "attention":
        return _attention_exact(state, case)
    if case["op"] == "rope":
        return _rotate_exact(state["x"].double(), state["positions"], case)
    out = {}
    for name in ("q", "k"):
        x = state[name].double()
        if case["norm"] == "layer":
            variance, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            x = x - mean
        else:
            variance = x.square().mean(-1, keepdim=True)
        x = x * torch.rsqrt(variance + 1e-6) * state[name + "_gamma"].double()
        if state[name + "_beta"] is not None:
            x = x + state[name + "_beta"].double()
        out[name] = _rotate_exact(x, state["positions"], case)
    return out


def _rotate_exact(x, positions, case):
    """Each pair as a complex number times amplitude e^(i angle)."""
    rot, axes = case["rot"], case["axes"]
    each = rot // 2 // axes
    frequencies = []
    for j in range(each):
        base = case["base"] * (8.0 ** (each / (each - 1)) if case["scaling"] == "ntk" and each > 1 else 1.0)
        f = math.exp(-j / each * math.log(base))
        if case["scaling"] == "linear":
            f /= 8.0
        elif case["scaling"] == "bands":
            turns = 8192 * f / (2.0 * math.pi)
            if turns <= 1.0:
                f /= 8.0
            elif turns < 4.0:
                r = (turns - 1.0) / 3.0
                f = r * f + (1.0 - r) * f / 8.0
        frequencies.append(f)
    f = torch.tensor(frequencies, dtype=torch.float64, device="cuda")
    at = positions.double().reshape(len(positions), axes)
    angle = torch.cat([at[:, i:i + 1] * f for i in range(axes)], -1)[:, None]
    turn = torch.polar(torch.full_like(angle, 1.2 if case["scaling"] == "bands" else 1.0), angle)
    head, rest = x[..., :rot], x[..., rot:]
    if case["interleaved"]:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, rest], -1)


def _attention_exact(state, case):
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(state["out"].shape, dtype=torch.float64, device="cuda")
    for s, (n_q, n_k) in enumerate(zip(state["n_q"], state["n_k"])):
        if n_k == 0:
            continue
        a, b = state["q_at"][s], state["k_at"][s]
        block = max(1, 2 ** 27 // (n_k * heads))         # queries at once, all heads
        k = state["k"][b:b + n_k].double().repeat_interleave(heads // kv_heads, 1)
        v = state["v"][b:b + n_k].double().repeat_interleave(heads // kv_heads, 1)
        for i in range(0, n_q, block):
            j = min(i + block, n_q)
            q = state["q"][a + i:a + j].double()
            seen = n_k if not case["causal"] else j + n_k - n_q
            scores = torch.einsum("qhd,khd->hqk", q, k[:seen]) / math.sqrt(dim)
            if case["causal"]:
                last = torch.arange(i, j, device="cuda")[:, None] + (n_k - n_q)
                scores = torch.where(torch.arange(seen, device="cuda") <= last, scores, -math.inf)
            out[a + i:a + j] = torch.einsum("hqk,khd->qhd", torch.softmax(scores, -1), v[:seen])
    return out
