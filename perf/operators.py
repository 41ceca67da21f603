"""The sequence operators of a pipeline stage, as cases to be timed: rotary positions with several axes, and attention
with a sliding window, first tokens that stay visible and shared key / value heads, each by itself and one behind the other.

A pass is what a training program has a stage do with one micro-batch: the forward pass of the operators and, where their
input wants its gradient, the backward pass, from tensors on the GPU to tensors on the GPU.  A branch whose parameters are
frozen runs forward only (`grad` false).

  rotary     x [b * S, F] rows as Q | K | V blocks of head_dim columns, positions [b * S, axes]: Q and K are rotated
  attention  the same rows, each query against the keys that its window and the first `sinks` tokens leave it
  block      rotary, then attention on its result
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a single token per sample: the shortest sequence a stage meets, all launch latency
        dict(name="attention_token_3x1", op="attention", b=3, seq=1, heads=8, kv_heads=2, head_dim=64, window=16, sinks=1, causal=True,
             ragged=False, dtype="bf16", grad=True),
        # a transformer branch as the benchmark has it (4 samples of 512 rows, 16 heads of 64), each patch sees its neighbourhood
        dict(name="attention_branch_4x512", op="attention", b=4, seq=512, heads=16, kv_heads=4, head_dim=64, window=128, sinks=0,
             causal=False, ragged=False, dtype="bf16", grad=True),
        # text of unequal lengths (one sample empty, one full), odd sizes, a head dimension between the powers of two
        dict(name="attention_ragged_8x1013", op="attention", b=8, seq=1013, heads=12, kv_heads=4, head_dim=96, window=256, sinks=1,
             causal=True, ragged=True, dtype="bf16", grad=True),
        # one long document with first tokens that stay visible: the largest step
        dict(name="attention_long_1x16384", op="attention", b=1, seq=16384, heads=16, kv_heads=2, head_dim=128, window=4096, sinks=4,
             causal=True, ragged=False, dtype="bf16", grad=True),
        # a stage kept in fp32, odd length
        dict(name="attention_f32_2x391", op="attention", b=2, seq=391, heads=8, kv_heads=8, head_dim=64, window=100, sinks=3, causal=True,
             ragged=False, dtype="f32", grad=True),
        # a frozen branch: forward only, every earlier token visible
        dict(name="attention_frozen_2x2048", op="attention", b=2, seq=2048, heads=32, kv_heads=8, head_dim=128, window=0, sinks=0,
             causal=True, ragged=False, dtype="bf16", grad=False),
        # the single token's positions
        dict(name="rotary_token_3x1", op="rotary", b=3, seq=1, heads=8, kv_heads=2, head_dim=64, pairs="8,12,12", base=10000.0,
             neighbours=False, per_axis=False, dtype="bf16", grad=True),
        # the benchmark's transformer branch with positions in time, height and width
        dict(name="rotary_branch_4x512", op="rotary", b=4, seq=512, heads=16, kv_heads=4, head_dim=64, pairs="8,12,12", base=10000.0,
             neighbours=False, per_axis=False, dtype="bf16", grad=True),
        # a long video: 32768 patches, the largest tensors
        dict(name="rotary_video_1x32768", op="rotary", b=1, seq=32768, heads=32, kv_heads=8, head_dim=128, pairs="16,24,24", base=1000000.0,
             neighbours=False, per_axis=False, dtype="bf16", grad=True),
        # images in fp32: a ladder of frequencies per axis, neighbouring columns paired, part of each head left as it is
        dict(name="rotary_f32_2x777", op="rotary", b=2, seq=777, heads=6, kv_heads=6, head_dim=80, pairs="16,16", base=100.0,
             neighbours=True, per_axis=True, dtype="f32", grad=True),
        # the two together on the benchmark's branch
        dict(name="block_branch_4x512", op="block", b=4, seq=512, heads=16, kv_heads=4, head_dim=64, window=128, sinks=0, causal=False,
             ragged=False, pairs="8,12,12", base=10000.0, neighbours=False, per_axis=False, dtype="bf16", grad=True),
        # and on clips of 4096 patches
        dict(name="block_clips_2x4096", op="block", b=2, seq=4096, heads=20, kv_heads=4, head_dim=128, window=1024, sinks=8, causal=False,
             ragged=False, pairs="16,24,24", base=1000000.0, neighbours=False, per_axis=False, dtype="bf16", grad=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def one():
        op = rng.choice(["attention", "attention", "rotary", "block"])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        kv = rng.choice([1, 2, 4, 8])
        c = dict(op=op, b=log(1, 16), seq=log(1, 32768 if op == "rotary" else 16384), heads=kv * rng.choice([1, 2, 4, 8]), kv_heads=kv,
                 head_dim=rng.choice([32, 64, 64, 80, 96, 128, 128]))
        if op != "rotary":
            c.update(window=0 if rng.random() < 0.2 else log(1, 4096), sinks=0 if rng.random() < 0.5 else log(1, 64),
                     causal=rng.random() < 0.6, ragged=rng.random() < 0.4)
        if op != "attention":
            axes, whole = rng.randint(1, 4), c["head_dim"] // 2
            p = whole if rng.random() < 0.7 else whole // 2
            cuts = sorted(rng.sample(range(1, p), axes - 1))
            c.update(pairs=",".join(str(y - x) for x, y in zip([0] + cuts, cuts + [p])), base=rng.choice([100.0, 10000.0, 1000000.0]),
                     neighbours=rng.random() < 0.3, per_axis=rng.random() < 0.4)
        c.update(dtype=dtype, grad=rng.random() < 0.85)
        return c

    most = {o: max(_cost(c) for c in listed() if c["op"] == o) for o in ("rotary", "attention", "block")}
    while True:
        c = one()
        room = c["b"] * c["heads"] * c["seq"] ** 2 <= 16 * 16384 ** 2 if c["op"] != "rotary" else True   # the scores of the plain form
        slow = 16.0 if c["dtype"] == "f32" else 1.0        # 32-bit matrix products run at a sixteenth of the rate
        if room and _cost(c) * (slow if c["op"] != "rotary" else 1.0) <= most[c["op"]]:
            return c


# ---- sizes ---------------------------------------------------------------------------------------------------
def _widths(c):
    return (c["heads"] + 2 * c["kv_heads"]) * c["head_dim"], c["heads"] * c["head_dim"]


def _lengths(c):
    """Lengths of a micro-batch's samples: evenly from 0 to the longest, so that one is empty and one is full."""
    b, s = c["b"], c["seq"]
    if not c.get("ragged"):
        return [s] * b
    return [s] if b == 1 else [int(round(s * i / (b - 1))) for i in range(b)]


def _visible(c, n):
    """Keys that each of n queries sees, summed."""
    i = np.arange(n, dtype=np.int64)
    last = i if c["causal"] else np.full(n, n - 1)
    if not c["window"]:
        return int((last + 1).sum())
    hi = np.minimum(last, i + c["window"] - 1)
    lo = np.maximum(0, i - c["window"] + 1)
    sinks = np.minimum(lo, min(c["sinks"], n))
    beyond = np.maximum(0, np.minimum(last + 1, min(c["sinks"], n)) - np.maximum(hi + 1, lo))     # first tokens behind the window
    return int((hi - lo + 1 + sinks + beyond).sum())


def work(c):
    rows, size = c["b"] * c["seq"], 2 if c["dtype"] == "bf16" else 4
    f, o = _widths(c)
    passes = 2 if c["grad"] else 1
    axes = len(c["pairs"].split(",")) if "pairs" in c else 0
    if c["op"] == "rotary":
        rotated = rows * (c["heads"] + c["kv_heads"]) * sum(int(p) for p in c["pairs"].split(","))
        return {"bytes": float(passes * 2 * rows * f * size + rows * axes * 4), "flops": float(passes * 6 * rotated)}
    pairs = c["heads"] * sum(_visible(c, n) for n in _lengths(c))
    return {"bytes": float(passes * rows * (f + o) * size + rows * axes * 4),
            "flops": float((14 if c["grad"] else 4) * pairs * c["head_dim"])}


def _cost(c):
    w = work(c)
    return w["bytes"] + w["flops"] / 200.0


# ---- what a program has in hand ------------------------------------------------------------------------------
def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    rows, kind = c["b"] * c["seq"], TYPE[c["dtype"]]
    f, o = _widths(c)
    s = dict(case=c, x=torch.randn(rows, f, generator=g, device=DEV).to(kind))
    if c["grad"]:
        s["dy"] = torch.randn(rows, f if c["op"] == "rotary" else o, generator=g, device=DEV).to(kind)
    if "pairs" in c:
        # a clip: time runs slowly, height and width through a grid; clips start somewhere in a longer recording
        axes = len(c["pairs"].split(","))
        at = torch.arange(c["seq"], device=DEV)
        start = torch.randint(0, 1 << 17, (c["b"], 1), generator=g, device=DEV)
        side = max(1, int(round(c["seq"] ** (1.0 / 3.0))))
        grid = [at // (side * side), (at // side) % side, at % side, at]
        chosen = [at] if axes == 1 else grid[1:3] if axes == 2 else grid[:axes]
        s["pos"] = torch.stack([(start + p if k == 0 else p.expand(c["b"], -1)).reshape(-1) for k, p in enumerate(chosen)], 1).to(torch.int32).contiguous()
    if c.get("ragged"):
        order = np.random.RandomState(int(seed) % (1 << 31)).permutation(c["b"])
        s["lengths"] = torch.tensor(np.array(_lengths(c))[order], dtype=torch.int32, device=DEV).reshape(-1, 1)
    if own:
        s.update(_stage(c, s))
    return s


def _ops(c):
    """The operator graph of the stage that a case is."""
    f, o = _widths(c)
    ops = [dict(kind="input", inputs=[], out_features=f, seq_len=c["seq"], dtype=c["dtype"], role="data" if c["grad"] else "frozen")]
    last = 0
    if "pairs" in c:
        pairs = [int(p) for p in c["pairs"].split(",")]
        ops.append(dict(kind="input", inputs=[], out_features=len(pairs), seq_len=c["seq"], dtype="i32"))
        ops.append(dict(kind="rotary", inputs=[0, 1], out_features=f, heads=c["heads"] + c["kv_heads"], head_dim=c["head_dim"],
                        axis_pairs=pairs, base=c["base"], pairing="neighbours" if c["neighbours"] else "halves",
                        ladder="per_axis" if c["per_axis"] else "shared", seq_len=c["seq"], dtype=c["dtype"]))
        last = 2
    if c["op"] != "rotary":
        ins = [last]
        if c["ragged"]:
            ops.append(dict(kind="input", inputs=[], out_features=1, dtype="i32"))
            ins.append(len(ops) - 1)
        ops.append(dict(kind="attention_window", inputs=ins, out_features=o, heads=c["heads"], kv_heads=c["kv_heads"],
                        head_dim=c["head_dim"], window=c["window"], sinks=c["sinks"], causal=c["causal"], seq_len=c["seq"],
                        dtype=c["dtype"]))
    return ops


def _stage(c, s):
    from paper_2406_17145_amd import binding as B
    stage = B.Stage(_ops(c), c["b"], {}, device=DEV)
    given = [s[k] for k in ("x", "pos", "lengths") if k in s]
    out, dx = stage.alloc_outputs(), stage.alloc_grad_inputs()
    return dict(B=B, stage=stage, given=given, out=out, dx=dx, loss=stage.loss,
                ptr_in=[t.data_ptr() for t in given], ptr_out=[t.data_ptr() for t in out],
                ptr_dy=[s["dy"].data_ptr()] if c["grad"] else [None],
                ptr_dx=[t.data_ptr() if t is not None else None for t in dx])


# ---- one pass ------------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        B, stage = s["B"], s["stage"]
        stream = torch.cuda.current_stream().cuda_stream
        B.gpp_stage_forward(stage.handle, 0, s["ptr_in"], s["ptr_out"], None, stream)
        B.gpp_stage_backward(stage.handle, 0, s["ptr_dy"], s["ptr_dx"], stream)      # (frozen: frees the micro-batch's slot)
        return [s["out"][0], s["dx"][0]] if c["grad"] else [s["out"][0]]
    x, dy = s["x"].float(), s["dy"].float() if c["grad"] else None
    if c["op"] != "attention":
        cos, sin = _angles(c, s["pos"])
    if c["op"] == "rotary":
        y = [_rotate(c, x, cos, sin), _rotate(c, dy, cos, -sin) if c["grad"] else None]
    elif c["op"] == "attention":
        y = _attend(c, x, dy, s.get("lengths"))
    else:
        # (a stage's operators keep their results in its storage type)
        y = _attend(c, _rotate(c, x, cos, sin).to(TYPE[c["dtype"]]).float(), dy, s.get("lengths"))
        if c["grad"]:
            y = [y[0], _rotate(c, y[1].to(TYPE[c["dtype"]]).float(), cos, -sin)]
    return [t.to(TYPE[c["dtype"]]) for t in y if t is not None]


def _angles(c, pos):
    """cos and sin of every row's pairs; the angles of far positions in 64 bits."""
    pairs = torch.tensor([int(p) for p in c["pairs"].split(",")], device=pos.device)
    total = int(sum(int(p) for p in c["pairs"].split(",")))
    axis = torch.repeat_interleave(torch.arange(len(pairs), device=pos.device), pairs, output_size=total)
    i = torch.arange(total, device=pos.device, dtype=torch.float64)
    inside = i - (torch.cumsum(pairs, 0) - pairs)[axis]
    exponent = inside / pairs[axis] if c["per_axis"] else i / total
    angle = pos[:, axis].double() * torch.exp(-math.log(c["base"]) * exponent)
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rotate(c, x, cos, sin):
    n, dh, p = c["heads"] + c["kv_heads"], c["head_dim"], cos.shape[1]
    h = x[:, :n * dh].reshape(-1, n, dh)
    cos, sin = cos[:, None], sin[:, None]
    if c["neighbours"]:
        x0, x1 = h[..., 0:2 * p:2], h[..., 1:2 * p:2]
        r = torch.stack([x0 * cos - x1 * sin, x0 * sin + x1 * cos], -1).flatten(-2)
    else:
        x0, x1 = h[..., :p], h[..., p:2 * p]
        r = torch.cat([x0 * cos - x1 * sin, x0 * sin + x1 * cos], -1)
    return torch.cat([torch.cat([r, h[..., 2 * p:]], -1).reshape(x.shape[0], n * dh), x[:, n * dh:]], 1)


def _attend(c, x, dy, lengths):
    """Output and gradient of the packed rows; scores of a whole micro-batch at once."""
    b, n, hq, hk, dh = c["b"], c["seq"], c["heads"], c["kv_heads"], c["head_dim"]
    i = torch.arange(n, device=x.device)
    back = i[:, None] - i[None, :]
    seen = torch.ones(n, n, dtype=torch.bool, device=x.device)
    if c["window"]:
        seen = (back.abs() < c["window"]) | (i[None, :] < c["sinks"])
    if c["causal"]:
        seen = seen & (back >= 0)
    seen = seen.expand(b, n, n)
    if lengths is not None:
        there = i[None] < lengths
        seen = seen & there[:, None, :] & there[:, :, None]
        x = torch.where(there.reshape(-1, 1), x, 0.0)
    seen = seen[:, None, None]

    def split(t, heads):
        return t.reshape(b, n, heads, dh).transpose(1, 2).reshape(b, hk, heads // hk, n, dh).contiguous()

    q, k, v = split(x[:, :hq * dh], hq), split(x[:, hq * dh:(hq + hk) * dh], hk), split(x[:, (hq + hk) * dh:], hk)
    scale = 1.0 / math.sqrt(dh)
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_min(1e-38))
    merge = lambda t, heads: t.reshape(b, heads, n, dh).transpose(1, 2).reshape(b * n, heads * dh)  # noqa: E731
    out = torch.matmul(p, v)
    if dy is None:
        return [merge(out, hq)]
    if lengths is not None:
        dy = torch.where(there.reshape(-1, 1), dy, 0.0)
    do = split(dy, hq)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2)
    return [merge(out, hq), torch.cat([merge(dq, hq), merge(dk, hk), merge(dv, hk)], 1)]


# ---- the same from the definitions in 64 bits -----------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    x = s["x"].double()
    dy = s["dy"].double() if c["grad"] else None
    turn = None
    if "pairs" in c:
        turn, stop = [], 0
        pairs = [int(p) for p in c["pairs"].split(",")]
        for a, p in enumerate(pairs):
            for j in range(p):
                w = c["base"] ** (-(j / p) if c["per_axis"] else -((stop + j) / sum(pairs)))
                turn.append(torch.polar(torch.ones_like(s["pos"][:, a], dtype=torch.float64), s["pos"][:, a].double() * w))
            stop += p
        turn = torch.stack(turn, 1)
    if c["op"] == "rotary":
        return [_turn(c, x, turn), _turn(c, dy, turn.conj())] if c["grad"] else [_turn(c, x, turn)]
    if c["op"] == "block":
        # (between the operators values are held in the storage type: the attention's inputs are those)
        x = _turn(c, x, turn).to(TYPE[c["dtype"]]).double()
    y = _attention_exact(c, x, dy, s["lengths"].flatten().tolist() if "lengths" in s else [c["seq"]] * c["b"])
    if c["op"] == "block" and c["grad"]:
        y[1] = _turn(c, y[1], turn.conj())
    return y


def _turn(c, x, turn):
    """Pairs of columns as complex numbers, times exp(i angle)."""
    y, p, dh = x.clone(), turn.shape[1], c["head_dim"]
    for h in range(c["heads"] + c["kv_heads"]):
        first = torch.arange(p, device=x.device) * (2 if c["neighbours"] else 1) + h * dh
        second = first + (1 if c["neighbours"] else p)
        z = torch.complex(x[:, first], x[:, second]) * turn
        y[:, first], y[:, second] = z.real, z.imag
    return y


def _attention_exact(c, x, dy, lengths):
    """Sample by sample, head by head; gradients by differentiating the definition."""
    hq, hk, dh, n = c["heads"], c["kv_heads"], c["head_dim"], c["seq"]
    out = torch.zeros(x.shape[0], hq * dh, dtype=torch.float64, device=x.device)
    grad = torch.zeros_like(x)
    for k, length in enumerate(lengths):
        if not length:
            continue
        rows = slice(k * n, k * n + length)
        i = torch.arange(length, device=x.device)
        hidden = torch.zeros(length, length, dtype=torch.bool, device=x.device)
        if c["causal"]:
            hidden |= i[:, None] < i[None, :]
        if c["window"]:
            hidden |= ((i[:, None] - i[None, :]).abs() >= c["window"]) & (i[None, :] >= c["sinks"])
        for h in range(hq):
            at = [h * dh, (hq + h // (hq // hk)) * dh, (hq + hk + h // (hq // hk)) * dh]
            q, key, v = (x[rows, a:a + dh].clone().requires_grad_(dy is not None) for a in at)
            logits = torch.matmul(q, key.T.contiguous()) / math.sqrt(dh)
            y = torch.matmul(torch.softmax(logits.masked_fill(hidden, -math.inf), -1), v)
            out[rows, h * dh:(h + 1) * dh] = y.detach()
            if dy is not None:
                for a, g in zip(at, torch.autograd.grad(y, (q, key, v), dy[rows, h * dh:(h + 1) * dh])):
                    grad[rows, a:a + dh] += g
    return [out, grad] if dy is not None else [out]
