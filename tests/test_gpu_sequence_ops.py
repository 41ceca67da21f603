"""Rotary positions and windowed attention on the GPU against the fp64 oracle.

Tolerances, l2-relative per tensor.  A rounding is off by at most half a step h of its type (bf16 2^-8, fp32 2^-24), relative
to the value.  bf16: a rotary rounds its result once, h; the attention output rounds the probabilities and the result, 2 h; dV the
same, 2 h; dQ and dK the forward output (in rowsum(dO * O)), the score gradients and the result, 3 h -- the whole gradient is held to
3 h.  fp32: sums of n terms in another order grow with sqrt(n) half steps and the exponent's argument, up to 16 in base 2,
carries its own roundings into the probabilities: (16 + sqrt(n)) h, several times over for the chain of products; 64 + 4 sqrt(n)
of them are allowed.  The max-norm guard is five times the bar, as everywhere."""
import numpy as np
import pytest

from tests import sequence_util as S

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2406_17145_amd.binding")
import torch  # noqa: E402


def bars(dtype, n):
    h = S.HALF_STEP[dtype]
    return (2 * h, 3 * h) if dtype == "bf16" else ((64 + 4 * n ** 0.5) * h,) * 2


def check(label, got, ref, bar):
    e2, em = S.rel(got, ref)
    assert e2 <= bar and em <= 5 * bar, f"{label}: l2 {e2:.3e} max {em:.3e} bar {bar:.3e}"


def lengths(values):
    return {1: lambda r, s: np.resize(np.array(values), s)}


def run_attention(flags=0, seed=0, values=None, fill=None, **case):
    ops = S.attention_ops(lengths=values is not None, **case)
    batch, gout = S.draw(ops, case["b"], seed, lengths(values) if values is not None else None)
    ref = S.oracle(ops, case["b"], batch, gout)
    if fill is not None:            # what lies behind a sample's length is not looked at
        for k in range(case["b"]):
            pad = slice(k * case["seq"] + int(batch[1].reshape(-1)[k]), (k + 1) * case["seq"])
            batch[0][pad] = fill
            gout[len(ops) - 1][pad] = fill
    got = S.gpu(ops, case["b"], batch, gout, flags=flags)
    b_out, b_grad = bars(case.get("dtype", "bf16"), case["seq"])
    check("out", got[0], ref[0], b_out)
    check("grad", got[1], ref[1], b_grad)
    return got, ref


# sequence lengths around the tiles of 32, 64 and 128 rows
@pytest.mark.parametrize("seq", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257])
@pytest.mark.parametrize("window,sinks,causal", [(0, 0, True), (0, 0, False), (1, 0, True), (5, 3, True), (40, 33, False), (70, 0, True), (64, 1, False)])
def test_window_lengths(seq, window, sinks, causal):
    run_attention(b=2, seq=seq, heads=4, kv=2, dh=64, window=window, sinks=sinks, causal=causal)


@pytest.mark.parametrize("dh", [8, 16, 20, 32, 40, 64, 72, 80, 96, 104, 128, 136, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, 1])
def test_window_head_dims(dh, dtype, flags):
    run_attention(b=1, seq=150, heads=2, kv=1, dh=dh, window=50, sinks=2, causal=True, dtype=dtype, flags=flags)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (8, 1), (5, 5)])
def test_window_head_layouts(heads, kv):
    run_attention(b=3, seq=100, heads=heads, kv=kv, dh=32, window=33, sinks=4, causal=False, dtype="f32")
    run_attention(b=3, seq=100, heads=heads, kv=kv, dh=64, window=33, sinks=4, causal=True)


@pytest.mark.parametrize("window,sinks,causal", [(0, 0, True), (0, 0, False), (17, 5, True), (17, 150, False), (300, 9, True), (1, 1, False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [None, float("nan"), float("inf")])
def test_window_ragged(window, sinks, causal, dtype, fill):
    run_attention(b=5, seq=140, heads=4, kv=2, dh=64, window=window, sinks=sinks, causal=causal, dtype=dtype,
                  values=[0, 140, 1, 77, 128], fill=fill)


@pytest.mark.parametrize("dh", [80, 128])
@pytest.mark.parametrize("b,seq,window,sinks,causal", [(1, 700, 0, 0, True), (2, 420, 90, 3, False), (3, 70, 33, 2, True), (13, 520, 40, 0, True)])
def test_window_wide_rows_of_fp32(dh, b, seq, window, sinks, causal):
    """Heads of more than 64 columns in fp32: few blocks of queries, whose waves share them, and (13 samples) many."""
    run_attention(b=b, seq=seq, heads=4, kv=2, dh=dh, window=window, sinks=sinks, causal=causal, dtype="f32")
    run_attention(b=b, seq=seq, heads=4, kv=2, dh=dh, window=window, sinks=sinks, causal=causal, dtype="f32",
                  values=[seq, 1, 0, seq // 2, 65][:b] + [seq - 33] * max(0, b - 5))


def test_window_all_samples_empty():
    ops = S.attention_ops(2, 40, 2, 1, 64, lengths=True)
    batch, gout = S.draw(ops, 2, 1, lengths([0, 0]))
    got = S.gpu(ops, 2, batch, gout)
    assert not got[0].any() and not got[1].any()


def test_window_one_visible_key_has_no_gradient_of_its_score():
    for dtype in ("bf16", "f32"):
        for flags in (0, 1):
            ops = S.attention_ops(3, 1, 4, 2, 64, causal=True, dtype=dtype)
            batch, gout = S.draw(ops, 3, 2)
            out, grad = S.gpu(ops, 3, batch, gout, flags=flags)
            assert np.array_equal(out.reshape(3, 2, 2, 64), np.repeat(batch[0][:, 384:].reshape(3, 2, 1, 64), 2, 2))
            assert not grad[:, :384].any()


@pytest.mark.parametrize("scale", [0.01, 0.5, 3.0])
def test_window_scale_and_large_scores(scale):
    # (scores up to 3 * 40: probabilities of 0 and 1; the running maximum moves)
    run_attention(b=1, seq=130, heads=2, kv=2, dh=64, window=0, causal=True, dtype="f32", scale=scale)


def test_window_mixed_storage():
    ops = S.attention_ops(2, 70, 4, 2, 64, window=20, causal=True, dtype="bf16", out_dtype="f32")
    batch, gout = S.draw(ops, 2, 3)
    got, ref = S.gpu(ops, 2, batch, gout), S.oracle(ops, 2, batch, gout)
    check("out", got[0], ref[0], bars("bf16", 70)[0])
    check("grad", got[1], ref[1], bars("bf16", 70)[1])


@pytest.mark.parametrize("window,sinks", [(512, 4), (0, 0)])
def test_window_long(window, sinks):
    """Long enough for work to be split along the sequence."""
    run_attention(b=1, seq=2500, heads=2, kv=1, dh=128, window=window, sinks=sinks, causal=True)
    run_attention(b=1, seq=2500, heads=2, kv=1, dh=64, window=window, sinks=sinks, causal=False)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("values", [None, [128, 0, 77, 1, 100, 128, 33, 64]])
def test_window_short_samples(dh, values):
    """Few blocks of keys that many query heads share, beside the blocks of queries."""
    run_attention(b=8, seq=128, heads=24, kv=3, dh=dh, window=70, sinks=2, causal=True, values=values)


@pytest.mark.parametrize("b,heads,kv,causal", [(1, 2, 1, True), (3, 4, 4, False)])
def test_window_many_first_tokens(b, heads, kv, causal):
    """First tokens over several blocks of keys, whose work is cut into parts, with samples that end inside them."""
    run_attention(b=b, seq=1900, heads=heads, kv=kv, dh=64, window=100, sinks=300, causal=causal, values=[1900, 200, 700][:b])


@pytest.mark.parametrize("flags", [0, 1])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 24), ("bf16", 20)])
def test_window_keeps_its_rows(dtype, dh, flags):
    """The caller's tensor may change between the passes: the backward pass reads the stage's own copy."""
    ops = S.attention_ops(2, 140, 6, 2, dh, window=30, sinks=2, causal=True, dtype=dtype, lengths=True)
    batch, gout = S.draw(ops, 2, 4, lengths([140, 99]))
    st = B.Stage(ops, 2, {}, flags=flags)
    ins = st.stage_inputs(batch)
    st.forward(0, ins)
    ins[0].fill_(float("nan")), ins[1].zero_()
    gin = st.backward(0, gout)
    check("grad", gin[0].float().cpu().numpy(), S.oracle(ops, 2, batch, gout)[1], bars(dtype, 140)[1])
    st.close()


def test_window_forward_only():
    ops = S.attention_ops(2, 100, 4, 2, 64, window=30, sinks=2, causal=True, lengths=True, grad=False)
    batch, gout = S.draw(ops, 2, 4, lengths([55, 100]))
    st = B.Stage(ops, 2, {})
    for _ in range(2):
        outs, _ = st.forward(0, batch)
        assert st.backward(0, gout) == [None, None]
        check("out", outs[0].float().cpu().numpy(), S.oracle(ops, 2, batch, gout)[0], bars("bf16", 100)[0])
    st.close()


def test_window_bad_lengths_are_reported_and_taken_as_the_nearer_end():
    ops = S.attention_ops(3, 50, 2, 1, 64, window=9, causal=True, lengths=True)
    batch, gout = S.draw(ops, 3, 5, lengths([-3, 60, 20]))
    fixed = {**batch, 1: np.array([[0], [50], [20]], np.int32)}
    st = B.Stage(ops, 3, {})
    outs, _ = st.forward(0, batch)
    gin = st.backward(0, gout)
    with pytest.raises(B.GppError) as e:
        st.sync_status()
    assert e.value.status == B.GPP_ERR_INDEX
    ref = S.oracle(ops, 3, fixed, gout)
    check("out", outs[0].float().cpu().numpy(), ref[0], bars("bf16", 50)[0])
    check("grad", gin[0].float().cpu().numpy(), ref[1], bars("bf16", 50)[1])
    st.forward(0, fixed)
    st.backward(0, gout)
    st.sync_status()
    st.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("heads,dh,pairs,rest", [(3, 64, (32,), 64), (4, 64, (8, 12, 12), 0), (2, 128, (16, 24, 24), 256), (2, 96, (24,), 8),
                                                 (3, 80, (10, 10), 80), (2, 20, (3, 1, 2), 7), (1, 5, (1, 1), 0), (2, 1000, (300, 100, 50, 50), 0)])
@pytest.mark.parametrize("rows", [1, 37])
def test_rotary(dtype, pairing, heads, dh, pairs, rest, rows):
    for ladder in ("shared", "per_axis"):
        ops = S.rotary_ops(2, rows, heads, dh, pairs, rest=rest, pairing=pairing, ladder=ladder, dtype=dtype)
        batch, gout = S.draw(ops, 2, rows, {1: lambda r, s: r.integers(-1000, 1 << 20, s)})
        got, ref = S.gpu(ops, 2, batch, gout), S.oracle(ops, 2, batch, gout)
        # fp32: the rounded fraction of a turn and the two functions' results, 8 half steps, beside the products' own
        bar = S.HALF_STEP[dtype] * (1 if dtype == "bf16" else 8)
        check("out", got[0], ref[0], bar)
        check("grad", got[1], ref[1], bar)


def test_rotary_ends_of_the_position_range():
    ops = S.rotary_ops(1, 6, 2, 32, (8, 8), base=10000.0, dtype="f32")
    far = [-2 ** 31, 2 ** 31 - 1, 0, 1, -1, 1 << 24]
    batch, gout = S.draw(ops, 1, 7, {1: lambda r, s: np.array(far * 2).reshape(2, 6).T})
    got, ref = S.gpu(ops, 1, batch, gout), S.oracle(ops, 1, batch, gout)
    # (an angle of 2^31 has 22 bits left behind the point in 64-bit radians: the oracle's own cos of it is 2^-22 off)
    check("out", got[0], ref[0], 8 * 2.0 ** -24 + 2.0 ** -21)
    check("grad", got[1], ref[1], 8 * 2.0 ** -24 + 2.0 ** -21)


def test_rotary_many_rows():
    """Several rows per workgroup."""
    ops = S.rotary_ops(1, 9001, 2, 16, (4, 4), rest=16)
    batch, gout = S.draw(ops, 1, 8, {1: lambda r, s: r.integers(0, 10000, s)})
    got, ref = S.gpu(ops, 1, batch, gout), S.oracle(ops, 1, batch, gout)
    check("out", got[0], ref[0], S.HALF_STEP["bf16"])
    check("grad", got[1], ref[1], S.HALF_STEP["bf16"])


# ---- as they are used: transformer branches, several micro-batches, streams, captured graphs -------------------------------
def _branches(**kw):
    from paper_2406_17145_amd import workloads as W
    base = dict(micro_batch=2, n_branches=3, n_layers=2, d_model=128, heads=4, d_ff=192, seq_len=40, d_head_out=64, n_classes=20,
                kv_heads=2, axis_pairs=[(16,), (8, 8), (4, 6, 6)], window=12, sinks=2, causal=True, ragged=True)
    base.update(kw)
    return W.mmt(**base)


@pytest.mark.parametrize("kw", [dict(), dict(dtype="f32"), dict(n_micro=3), dict(kv_heads=4, ragged=False, causal=False, sinks=0), dict(d_model=256, seq_len=130, window=0)])
@pytest.mark.parametrize("flags", [0, 1, 4])
def test_transformer_branches_with_positions(kw, flags):
    from tests import parity_util as P
    wl = _branches(**kw)
    if flags & 4:
        st_res = _grouped(wl)
    else:
        st_res = P.run_gpu(wl, flags=flags)
    P.compare(wl, *st_res, *P.run_oracle(wl), label=f"positions and windows {kw} flags {flags}")


def _grouped(wl):
    """All micro-batches in flight, weight gradients of all of them in one launch."""
    from tests import parity_util as P
    st = B.Stage(wl.ops, wl.micro_batch, wl.params, slots=wl.n_micro, flags=B.FLAG_GROUPED_DW)
    st.grad_reset()
    losses, gins = [], []
    for j in range(wl.n_micro):
        loss = torch.zeros(1, device=st.dev)
        st.forward(j, wl.batches[j], loss=loss)
        losses.append(loss)
    for j in range(wl.n_micro):
        gins.append(st.backward(j))
    st.backward_weights()
    st.sync_status()
    res = [dict(loss=float(a), outs={}, gin={i: P.t2n(t) for i, t in zip(st.input_ids, g) if t is not None}) for a, g in zip(losses, gins)]
    grads = st.grads_numpy()
    st.close()
    return res, grads


def _graph_of_sequence_ops():
    """Three readers of one tensor and of one list of lengths, positions shared by two rotaries, a rotary that is added to and merged,
    one that is an output beside an attention that is one."""
    f = 6 * 32
    ops = [dict(kind="input", inputs=[], out_features=f, seq_len=24, dtype="bf16", rows_extra=0),
           dict(kind="input", inputs=[], out_features=2, seq_len=24, dtype="i32", rows_extra=0, role="positions"),
           dict(kind="input", inputs=[], out_features=1, seq_len=1, dtype="i32", rows_extra=0, role="lengths")]
    rot = dict(kind="rotary", heads=4, head_dim=32, axis_pairs=[10, 6], base=100.0, seq_len=24, dtype="bf16", out_features=f)
    att = dict(kind="attention_window", heads=2, kv_heads=2, head_dim=32, seq_len=24, dtype="bf16", out_features=64)
    add = lambda kind, ins, **kw: ops.append(dict(kind=kind, inputs=ins, dtype="bf16", **kw)) or len(ops) - 1  # noqa: E731
    a = ops.append({**rot, "inputs": [0, 1]}) or len(ops) - 1
    b = ops.append({**rot, "inputs": [0, 1], "pairing": "neighbours"}) or len(ops) - 1
    lin = add("linear", [0], in_features=f, out_features=f, act="none", bias=True)
    c = ops.append({**rot, "inputs": [lin, 1], "base": 30.0}) or len(ops) - 1        # turns the layer's rows in place
    s = add("add", [b, c], out_features=f)
    ops.append({**att, "inputs": [a, 2], "window": 5, "causal": True})               # an output
    w = ops.append({**att, "inputs": [s, 2], "window": 9, "sinks": 3}) or len(ops) - 1
    v = ops.append({**att, "inputs": [c], "window": 0}) or len(ops) - 1
    add("concat", [w, v], out_features=128)                                          # an output
    ops.append({**rot, "inputs": [a, 1], "base": 7.0})                               # an output: reads what another one wrote
    return ops


def test_shared_inputs_merges_and_outputs():
    from paper_2406_17145_amd import workloads as W
    from oracle import gpp_oracle as O
    ops = _graph_of_sequence_ops()
    rng = np.random.default_rng(11)
    lin = next(i for i, o in enumerate(ops) if o["kind"] == "linear")
    params = {lin: {"W": W.round_to_bf16(rng.standard_normal((192, 192)) / 14), "b": rng.standard_normal(192).astype(np.float32)}}
    batch = {0: W.round_to_bf16(rng.standard_normal((72, 192))), 1: rng.integers(0, 500, (72, 2)).astype(np.int32),
             2: np.array([[24], [0], [13]], np.int32)}
    ora = O.OracleStage(ops, 3, params, model_storage=True)
    stash = ora.forward(batch)
    gout = {i: W.round_to_bf16(rng.standard_normal(stash.values[i].shape)) for i in ora.output_ids}
    ref = ora.backward(stash, gout)
    st = B.Stage(ops, 3, params, slots=2)
    st.grad_reset()
    other = {**batch, 0: -batch[0], 2: np.array([[1], [2], [3]], np.int32)}
    outs, _ = st.forward(0, batch)
    st.forward(1, other)                         # another micro-batch in flight: its positions and lengths are its own
    gin = st.backward(0, gout)
    st.sync_status()
    for i, t in zip(st.output_ids, outs):
        check(f"out {i}", t.float().cpu().numpy(), stash.values[i], 2e-2)
    check("grad", gin[0].float().cpu().numpy(), ref[0], 2e-2)
    grads = st.grads_numpy()
    check("dW", grads[lin]["W"], ora.grads[lin]["W"], 2e-2)
    check("db", grads[lin]["b"], ora.grads[lin]["b"], 2e-2)
    st.backward(1, gout)
    # unwanted results are not written, the others are as before
    outs2, _ = st.forward(0, batch, outputs=[torch.zeros_like(t) for t in outs])
    ptrs = [t.data_ptr() if k else None for k, t in enumerate(outs2)]
    st.backward(0, gout)
    B.gpp_stage_forward(st.handle, 0, [t.data_ptr() for t in st.stage_inputs(batch)], ptrs, None, st.stream())
    g2 = [st.to_device(i, gout[i]) for i in st.output_ids]
    B.gpp_stage_backward(st.handle, 0, [t.data_ptr() for t in g2], [None] * len(st.input_ids), st.stream())
    torch.cuda.synchronize()
    for a, c in zip(outs, outs2):
        assert torch.equal(a, c)
    st.close()


@pytest.mark.parametrize("op", ["attention", "rotary"])
def test_streams_and_captured_graphs(op):
    """A pass on a stream of its own, and the same pass captured and replayed among other work."""
    if op == "rotary":
        ops = S.rotary_ops(2, 300, 6, 64, (8, 12, 12), rest=64)
        batch, gout = S.draw(ops, 2, 12, {1: lambda r, s: r.integers(0, 9999, s)})
    else:
        ops = S.attention_ops(2, 300, 4, 1, 64, window=90, sinks=4, causal=True, lengths=True)
        batch, gout = S.draw(ops, 2, 12, lengths([300, 211]))
    st = B.Stage(ops, 2, {})
    ins, g = st.stage_inputs(batch), [st.to_device(len(ops) - 1, gout[len(ops) - 1])]
    outs, gin = st.alloc_outputs(), st.alloc_grad_inputs()

    def one():
        st.forward(0, ins, outs)
        st.backward(0, g, gin)
    one()
    torch.cuda.synchronize()
    want = [outs[0].clone(), gin[0].clone()]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        outs[0].zero_(), gin[0].zero_()
        one()
    side.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(gin[0], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for k in range(4):
        ins[0].copy_(st.to_device(0, (1 + k % 2) * batch[0]))
        outs[0].zero_(), gin[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [outs[0].clone(), gin[0].clone()]
        one()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], got[0]) and torch.equal(gin[0], got[1])
        if k % 2 == 0:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    st.close()


def test_same_inputs_same_bits():
    ops = S.attention_ops(2, 700, 8, 2, 64, window=100, sinks=3, causal=True)
    batch, gout = S.draw(ops, 2, 13)
    a, b = S.gpu(ops, 2, batch, gout), S.gpu(ops, 2, batch, gout, slots=2)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_a_pipeline_of_two_stages():
    """Rotary in one stage, attention in the next: the edge's tensors are the caller's tensors of both."""
    from oracle import gpp_oracle as O
    first = S.rotary_ops(2, 30, 3, 64, (16, 16), rest=64)
    second = S.attention_ops(2, 30, 2, 1, 64, window=7, causal=True)
    batch, _ = S.draw(first, 2, 14, {1: lambda r, s: r.integers(0, 99, s)})
    _, gout = S.draw(second, 2, 15)
    a = O.OracleStage(first, 2, {}, model_storage=True)
    sa = a.forward(batch)
    b = O.OracleStage(second, 2, {}, model_storage=True)
    sb = b.forward({0: sa.values[2]})
    ref = a.backward(sa, {2: O.store_as(b.backward(sb, gout)[0], "bf16")})
    st = [B.Stage(first, 2, {}, slots=2), B.Stage(second, 2, {}, slots=1)]
    handles, edges = [s.handle for s in st], [(0, 0, 1, 0)]
    i, k = B.gpp_assign_schedules(2, [(0, 1)], [2, 2], [[1], [1]])
    size = B.gpp_pipeline_workspace_bytes(handles, edges, i, k)
    ws = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    pipe = B.gpp_pipeline_create(handles, edges, i, k, (ws.data_ptr() + 255) // 256 * 256, size)
    ins = st[0].stage_inputs(batch)
    out, gin, g = st[1].alloc_outputs()[0], st[0].alloc_grad_inputs()[0], st[1].to_device(1, gout[1])
    io = [[([t.data_ptr() for t in ins], [None], None, [None], [gin.data_ptr(), None])] * 3,
          [([None], [out.data_ptr()], None, [g.data_ptr()], [None])] * 3]
    s = torch.cuda.current_stream().cuda_stream
    keep = B.gpp_pipeline_run(pipe, io, [s, s], [s, s])
    torch.cuda.synchronize()
    check("out", out.float().cpu().numpy(), sb.values[1], 2e-2)
    check("grad", gin.float().cpu().numpy(), ref[0], 2e-2)
    B.gpp_pipeline_destroy(pipe)
    assert keep is not None
    for x in st:
        x.close()


@pytest.mark.parametrize("op", ["attention", "rotary"])
def test_misaligned_tensors_are_refused(op):
    """On the host, before anything is enqueued; the stage can be used afterwards."""
    ops = S.attention_ops(1, 9, 2, 1, 16) if op == "attention" else S.rotary_ops(1, 9, 2, 16, (8,), rest=32)
    batch, gout = S.draw(ops, 1, 16, {1: lambda r, s: r.integers(0, 99, s)})
    st = B.Stage(ops, 1, {})
    ins, g = st.stage_inputs(batch), st.to_device(len(ops) - 1, gout[len(ops) - 1])
    outs, gin = st.alloc_outputs(), st.alloc_grad_inputs()
    fw = [t.data_ptr() for t in ins], [outs[0].data_ptr()]
    bw = [g.data_ptr()], [None if t is None else t.data_ptr() for t in gin]

    def moved(ptrs):
        return [ptrs[0] + 8] + ptrs[1:]

    def refused(call, a, b):
        with pytest.raises(B.GppError) as e:
            call(a, b)
        assert e.value.status == B.GPP_ERR_INVALID_ARG and "16-byte" in str(e.value)

    def forward(a, b):
        B.gpp_stage_forward(st.handle, 0, a, b, None, st.stream())

    def backward(a, b):
        B.gpp_stage_backward(st.handle, 0, a, b, st.stream())
    refused(forward, moved(fw[0]), fw[1])
    refused(forward, fw[0], moved(fw[1]))
    forward(*fw)
    refused(backward, moved(bw[0]), bw[1])
    refused(backward, bw[0], moved(bw[1]))
    backward(*bw)
    torch.cuda.synchronize()
    ref = S.oracle(ops, 1, batch, gout)
    check("out", outs[0].float().cpu().numpy(), ref[0], bars("bf16", 9)[0])
    check("grad", gin[0].float().cpu().numpy(), ref[1], bars("bf16", 9)[1])
    st.close()


def test_rows_beyond_32_bits():
    """[2 x 2^18, 6144]: offsets of the second sample pass 2^31 elements and 2^32 bytes.  The last queries and keys against a dense
    calculation in fp64 over the rows that they can see."""
    s, heads, kv, dh, window, sinks, tail = 1 << 18, 32, 8, 128, 100, 3, 200
    ops = S.attention_ops(2, s, heads, kv, dh, window=window, sinks=sinks, causal=True)
    st = B.Stage(ops, 2, {})
    gen = torch.Generator(device="cuda").manual_seed(17)
    x = torch.empty(2 * s, (heads + 2 * kv) * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    g = torch.empty(2 * s, heads * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    out, gx = torch.empty_like(g), torch.empty_like(x)
    B.gpp_stage_forward(st.handle, 0, [x.data_ptr()], [out.data_ptr()], None, st.stream())
    B.gpp_stage_backward(st.handle, 0, [g.data_ptr()], [gx.data_ptr()], st.stream())
    torch.cuda.synchronize()
    rows = torch.cat([torch.arange(sinks), torch.arange(s - tail - window, s)])
    part = x[(s + rows).cuda()].cpu().double().requires_grad_()
    r = part.reshape(len(rows), heads + 2 * kv, dh).transpose(0, 1)
    back = rows[-tail:, None] - rows[None, :]
    seen = (back >= 0) & ((back < window) | (rows[None, :] < sinks))
    k, v = (r[a:a + kv].repeat_interleave(heads // kv, 0) for a in (heads, heads + kv))
    p = ((r[:heads, -tail:] @ k.transpose(1, 2)) * dh ** -0.5).masked_fill(~seen, -float("inf")).softmax(-1)
    ref = (p @ v).transpose(0, 1).reshape(tail, heads * dh)
    (ref * g[-tail:].cpu().double()).sum().backward()
    check("out", out[-tail:].float().cpu().numpy(), ref.detach().numpy(), bars("bf16", window)[0])
    check("grad", gx[-tail:].float().cpu().numpy(), part.grad[-tail:].numpy(), bars("bf16", window)[1])
    st.close()
    del st, out, gx, g
    ops = S.rotary_ops(2, s, heads + kv, dh, (64,), rest=kv * dh)
    st = B.Stage(ops, 2, {})
    pos = torch.arange(2 * s, dtype=torch.int32, device="cuda").reshape(-1, 1)
    y = torch.empty_like(x)
    B.gpp_stage_forward(st.handle, 0, [x.data_ptr(), pos.data_ptr()], [y.data_ptr()], None, st.stream())
    torch.cuda.synchronize()
    a = x[-tail:].cpu().double()
    t = pos[-tail:].cpu().double() * 10000.0 ** (-torch.arange(64).double() / 64)
    cos, sin = (f(t)[:, None] for f in (torch.cos, torch.sin))
    q = a[:, :(heads + kv) * dh].reshape(tail, heads + kv, 2, 64)
    turned = torch.stack([q[:, :, 0] * cos - q[:, :, 1] * sin, q[:, :, 0] * sin + q[:, :, 1] * cos], 2).reshape(tail, -1)
    check("rotary", y[-tail:].float().cpu().numpy(), torch.cat([turned, a[:, (heads + kv) * dh:]], 1).numpy(), S.HALF_STEP["bf16"])
    st.close()
