"""Sequence operators (rotary positions, windowed attention) on the GPU against the fp64 oracle: gradients block by block, cut sums of
many rounds, and the places in an operator graph that choose buffers and kernels of their own.

Tolerances count roundings, a half step h each (bf16 2^-8, fp32 2^-24), l2-relative per tensor.  One attention as in
test_gpu_sequence_ops: output and dV 2 h, dQ and dK 3 h in bf16; 64 + 4 sqrt(n) half steps in fp32.  Graphs in bf16 against the oracle that
rounds what operators store, so that what differs is what a kernel rounds inside and a stored value that falls to the other
side: one h for each operator that a tensor has come through, and two more for an attention among them.  The max-norm guard is five times
the bar, as everywhere."""
import numpy as np
import pytest

from oracle import gpp_oracle as O
from tests import sequence_util as S

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2406_17145_amd.binding")
import torch  # noqa: E402

from paper_2406_17145_amd import workloads as W  # noqa: E402

H = S.HALF_STEP["bf16"]


def check(label, got, ref, bar):
    e2, em = S.rel(got, ref)
    assert e2 <= bar and em <= 5 * bar, f"{label}: l2 {e2:.3e} max {em:.3e} bar {bar:.3e}"


def check_blocks(label, got, ref, heads, kv, dh, dtype, n):
    """dQ, dK and dV by themselves."""
    h = S.HALF_STEP[dtype]
    q, k = heads * dh, (heads + kv) * dh
    for name, at, steps in (("dQ", slice(0, q), 3), ("dK", slice(q, k), 3), ("dV", slice(k, None), 2)):
        check(f"{label} {name}", got[:, at], ref[:, at], (steps if dtype == "bf16" else 64 + 4 * n ** 0.5) * h)


def lengths(values):
    return {1: lambda r, s: np.resize(np.array(values), s)}


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("bf16", 20), ("f32", 64), ("f32", 96)])
@pytest.mark.parametrize("b,seq,heads,kv,window,sinks,causal,values", [
    (2, 5, 4, 2, 3, 1, True, None), (3, 70, 4, 1, 0, 0, True, [70, 1, 33]), (2, 150, 6, 3, 17, 40, False, None), (2, 150, 2, 2, 64, 2, True, [150, 66]),
    (1, 600, 4, 2, 100, 3, True, None), (4, 1, 2, 1, 0, 0, False, None)])
def test_gradient_blocks(dtype, dh, b, seq, heads, kv, window, sinks, causal, values):
    """dQ, dK and dV of each sample."""
    ops = S.attention_ops(b, seq, heads, kv, dh, window=window, sinks=sinks, causal=causal, dtype=dtype, lengths=values is not None)
    batch, gout = S.draw(ops, b, 21, lengths(values) if values else None)
    got, ref = S.gpu(ops, b, batch, gout), S.oracle(ops, b, batch, gout)
    for k in range(b):
        rows = slice(k * seq, (k + 1) * seq)
        check_blocks(f"sample {k}", got[1][rows], ref[1][rows], heads, kv, dh, dtype, seq)


@pytest.mark.parametrize("b,seq,heads,kv,dh,dtype,values", [(3, 1500, 6, 3, 96, "f32", None), (5, 1300, 8, 1, 64, "bf16", None), (1, 3000, 8, 2, 128, "bf16", None),
                                                            (5, 1300, 8, 1, 64, "bf16", [1300, 0, 1, 700, 129])])
def test_cut_blocks_of_causal_rows(b, seq, heads, kv, dh, dtype, values):
    """Causal without a window: blocks of keys in more parts than run at once, which go round the XCDs block by block."""
    ops = S.attention_ops(b, seq, heads, kv, dh, causal=True, dtype=dtype, lengths=values is not None)
    d, keep = B.build_desc(ops, b)
    cut = [s["blocks"] for s in B.gpp_stage_describe(d) if s["kernel"] == "attention_bwd_dkv"]
    assert len(cut) == 2 and cut[0] > 256 and cut[0] % 2 == b * kv * ((seq + 127) // 128) % 2      # units (an odd number of parts), joins
    batch, gout = S.draw(ops, b, 22, lengths(values) if values else None)
    got, ref = S.gpu(ops, b, batch, gout), S.oracle(ops, b, batch, gout)
    check_blocks("gradient", got[1], ref[1], heads, kv, dh, dtype, seq)
    again = S.gpu(ops, b, batch, gout, slots=2)
    assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])


# ---- operator graphs ----------------------------------------------------------------------------------------------
class Graph:
    """A list of operators in bf16, S rows a sample."""
    def __init__(self, seq):
        self.ops, self.seq, self.params, self.rng = [], seq, {}, np.random.default_rng(31)

    def add(self, kind, inputs=(), **kw):
        self.ops.append(dict(kind=kind, inputs=list(inputs), dtype=kw.pop("dtype", "bf16"), **kw))
        return len(self.ops) - 1

    def input(self, feat, seq=None, **kw):
        return self.add("input", out_features=feat, seq_len=self.seq if seq is None else seq, rows_extra=0, **kw)

    def linear(self, x, out, act="none"):
        feat = self.ops[x]["out_features"]
        i = self.add("linear", [x], in_features=feat, out_features=out, act=act, bias=True)
        self.params[i] = {"W": W.round_to_bf16(self.rng.standard_normal((out, feat)) / feat ** 0.5), "b": self.rng.standard_normal(out).astype(np.float32)}
        return i

    def rotary(self, x, pos, heads, dh, pairs=(10, 6), **kw):
        return self.add("rotary", [x, pos], out_features=self.ops[x]["out_features"], heads=heads, head_dim=dh, axis_pairs=list(pairs), base=100.0,
                        seq_len=self.seq, **kw)

    def attention(self, x, heads, kv, dh, lengths=None, **kw):
        return self.add("attention_window", [x] if lengths is None else [x, lengths], out_features=heads * dh, heads=heads, kv_heads=kv, head_dim=dh,
                        seq_len=self.seq, **kw)

    def concat(self, *xs):
        return self.add("concat", xs, out_features=sum(self.ops[x]["out_features"] for x in xs))

    def kernels(self, b, flags=0):
        d, keep = B.build_desc(self.ops, b, flags=flags)
        return [(s["pass"], s["kernel"], s["records"]) for s in B.gpp_stage_describe(d) if s["kernel"] != "loss_sum"]

    def compare(self, b, batch, steps, flags=0, blocks=None):
        """Outputs, input gradients (blocks: of input i the Q, K and V columns by themselves) and parameter gradients, to `steps` h."""
        ora = O.OracleStage(self.ops, b, self.params, model_storage=True)
        stash = ora.forward(batch)
        gout = {i: W.round_to_bf16(self.rng.standard_normal(stash.values[i].shape)) for i in ora.output_ids}
        ref = ora.backward(stash, gout)
        st = B.Stage(self.ops, b, self.params, slots=2, flags=flags)
        st.grad_reset()
        outs, _ = st.forward(0, batch)
        gin = st.backward(0, gout)
        if flags & B.FLAG_GROUPED_DW:
            st.backward_weights()
        st.sync_status()
        for i, t in zip(st.output_ids, outs):
            check(f"output {i}", t.float().cpu().numpy(), stash.values[i], steps * H)
        for i, t in zip(st.input_ids, gin):
            if t is None:
                continue
            got = t.float().cpu().numpy()
            for at in (blocks or {}).get(i, [slice(None)]):
                check(f"gradient of {i} {at}", got[:, at], ref[i][:, at], steps * H)
        grads = st.grads_numpy()
        for i in self.params:
            check(f"dW {i}", grads[i]["W"], ora.grads[i]["W"], steps * H)
            check(f"db {i}", grads[i]["b"], ora.grads[i]["b"], steps * H)
        st.close()


FLAGS = [0, 1, 4]      # (1: the row-parallel kernels; 4: weight gradients of a group, gradients per slot)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("front", [33, 40])
def test_merge_of_a_rotary_in_place_and_an_attention(front, flags):
    """A rotary behind a layer and an attention, each read by a merge only, at columns off 16 bytes (33) and on (40): their results lie in
    the merge, the rotary's gradient, and that of its layer, too where it is on 16 bytes."""
    g, b, seq = Graph(24), 3, 24
    x, pos, length = g.input(192), g.input(2, dtype="i32"), g.input(1, 1, dtype="i32")
    first = g.linear(x, front)
    turned = g.rotary(g.linear(x, 192), pos, 4, 32)
    seen = g.attention(x, 2, 2, 32, length, window=7, sinks=2, causal=True)
    g.linear(g.concat(first, turned, seen), 64)
    rng = np.random.default_rng(32)
    batch = {x: W.round_to_bf16(rng.standard_normal((b * seq, 192))), pos: rng.integers(0, 500, (b * seq, 2)).astype(np.int32),
             length: np.array([[24], [0], [13]], np.int32)}
    # merge's layer, rotary, its layer, three sums; an attention
    g.compare(b, batch, 8, flags)


@pytest.mark.parametrize("flags", FLAGS)
def test_merge_of_rotaries_in_place_inside_a_merge(flags):
    """Rotaries in place in a merge, which an attention and another merge read."""
    g, b, seq = Graph(20), 2, 20
    x, pos = g.input(96), g.input(2, dtype="i32")
    one = g.rotary(g.linear(x, 64), pos, 2, 32)
    two = g.rotary(g.linear(x, 128), pos, 4, 32, pairs=(5, 3), pairing="neighbours")
    merge = g.concat(one, two)
    seen = g.attention(merge, 2, 2, 32, window=6)
    g.concat(merge, seen)
    rng = np.random.default_rng(33)
    batch = {x: W.round_to_bf16(rng.standard_normal((b * seq, 96))), pos: rng.integers(0, 500, (b * seq, 2)).astype(np.int32)}
    # attention (2 more), sum, rotary, layer, sum
    g.compare(b, batch, 8, flags)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("other", ["rotary", "layer", "input", "activated layer"])
def test_sum_of_a_rotary_in_place(other, flags):
    """A rotary behind a layer that only an addition reads: the sum's gradient goes to both addends, the rotary turns one of its own."""
    g, b, seq = Graph(20), 2, 20
    x, pos = g.input(96), g.input(2, dtype="i32")
    turned = g.rotary(g.linear(x, 96), pos, 3, 32)
    second = {"rotary": lambda: g.rotary(g.linear(x, 96), pos, 2, 32, pairs=(4, 4)), "layer": lambda: g.linear(x, 96), "input": lambda: x,
              "activated layer": lambda: g.linear(x, 96, "gelu")}[other]()
    total = g.add("add", [second, turned], out_features=96)
    g.linear(total, 32)
    g.add("add", [total, x], out_features=96)
    rng = np.random.default_rng(34)
    batch = {x: W.round_to_bf16(rng.standard_normal((b * seq, 96))), pos: rng.integers(0, 500, (b * seq, 2)).astype(np.int32)}
    # layer, sum, rotary, layer, three sums
    g.compare(b, batch, 7, flags)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("first,second", [([24, 3, 0], [7, 24, 24]), ([7, 24, 24], [24, 3, 0])])
def test_two_attentions_with_lengths_of_their_own_share_an_input(first, second, flags):
    """The stage keeps one copy of the rows for both: what one does not see the other does."""
    g, b, seq = Graph(24), 3, 24
    x, one, two = g.input(256), g.input(1, 1, dtype="i32"), g.input(1, 1, dtype="i32")
    g.attention(x, 2, 1, 64, one, window=9, causal=True)
    g.attention(x, 4, 2, 32, two, window=0, causal=False)
    rng = np.random.default_rng(35)
    batch = {x: W.round_to_bf16(rng.standard_normal((b * seq, 256))), one: np.array(first, np.int32).reshape(3, 1), two: np.array(second, np.int32).reshape(3, 1)}
    # an attention and a sum
    g.compare(b, batch, 4, flags, blocks={x: [slice(0, 128), slice(128, 192), slice(192, 256)]})


def test_more_inputs_and_outputs_than_a_launch_has_pointers_for():
    """Forty branches: the first 32 inputs and outputs are the caller's own tensors in the launches, the others are copied."""
    g, b, seq, feeds = Graph(9), 2, 9, {}
    rng = np.random.default_rng(36)
    for k in range(40):
        x = g.input(128)
        feeds[x] = W.round_to_bf16(rng.standard_normal((b * seq, 128)))
        if k % 3 == 0:
            p = g.input(2, dtype="i32")
            feeds[p] = rng.integers(0, 500, (b * seq, 2)).astype(np.int32)
            g.rotary(x, p, 3, 32)
        elif k % 3 == 1:
            n = g.input(1, 1, dtype="i32")
            feeds[n] = rng.integers(0, seq + 1, (b, 1)).astype(np.int32)
            g.attention(x, 2, 1, 32, n, window=4, causal=True)
        else:
            g.attention(x, 4, 2, 16, window=3, sinks=1)
    kernels = g.kernels(b)
    assert [n for p, k, n in kernels if (p, k) == ("forward", "attention_fwd")] == [26]
    assert ("forward", "elt_fwd", 14) in kernels and ("backward", "elt_bwd", 14) in kernels      # the rotaries
    copies = sum(n for p, k, n in kernels if (p, k) == ("forward", "elt_fwd")) - 14
    inputs = sum(op["kind"] == "input" for op in g.ops)
    assert copies == (inputs - 32) + (40 - 32)
    # an attention
    g.compare(b, feeds, 3)


@pytest.mark.parametrize("dh", [32, 64, 96, 128])
@pytest.mark.parametrize("b,seq", [(2, 150), (24, 400)])
def test_branches_that_see_few_keys_and_many_share_a_launch(b, seq, dh):
    """Of one launch's branches some keep the lower half of their output and some do not; one backward launch for all, or several."""
    g, rng, feeds = Graph(seq), np.random.default_rng(38), {}
    for window, causal in ((3, True), (0, True), (5, False), (90, False)):
        x = g.input(4 * dh)
        feeds[x] = W.round_to_bf16(rng.standard_normal((b * seq, 4 * dh)))
        g.attention(x, 2, 1, dh, window=window, causal=causal)
    # an attention
    g.compare(b, feeds, 3, blocks={x: [slice(0, 2 * dh), slice(2 * dh, 3 * dh), slice(3 * dh, None)] for x in feeds})


def test_branches_of_more_threads_than_a_launch_has():
    """Three attentions on a million single tokens each, in launches of their own: a token sees itself, so its output is V, dV is dO and
    the rest of the gradient is zero.  Then rotary positions of 2^27 rows."""
    b, n, heads, dh = 1 << 20, 3, 7, 8
    ops = [{**op, "inputs": [p + 2 * k for p in op["inputs"]]} for k in range(n) for op in S.attention_ops(b, 1, heads, heads, dh)]
    st = B.Stage(ops, b, {})
    gen = torch.Generator(device="cuda").manual_seed(37)
    x = [torch.empty(b, 3 * heads * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(n)]
    dy = [torch.empty(b, heads * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(n)]
    y, dx = [torch.empty_like(t) for t in dy], [torch.empty_like(t) for t in x]
    ptr = lambda ts: [t.data_ptr() for t in ts]  # noqa: E731
    B.gpp_stage_forward(st.handle, 0, ptr(x), ptr(y), None, st.stream())
    B.gpp_stage_backward(st.handle, 0, ptr(dy), ptr(dx), st.stream())
    torch.cuda.synchronize()
    v = slice(2 * heads * dh, None)
    for k in range(n):
        assert torch.equal(y[k], x[k][:, v]) and torch.equal(dx[k][:, v], dy[k]) and not dx[k][:, :2 * heads * dh].any()
    st.close()
    del st, x, dy, y, dx
    rows = 127 * b
    ops = [{**op, "inputs": [p + 3 * k for p in op["inputs"]]} for k in range(n) for op in S.rotary_ops(b, 127, 1, 2, (1,), grad=False)]
    st = B.Stage(ops, b, {})
    x = [torch.empty(rows, 2, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(n)]
    pos = [torch.arange(rows, dtype=torch.int32, device="cuda") % 1000 + k for k in range(n)]
    y = [torch.empty_like(t) for t in x]
    B.gpp_stage_forward(st.handle, 0, [t.data_ptr() for k in range(n) for t in (x[k], pos[k])], ptr(y), None, st.stream())
    torch.cuda.synchronize()
    for k in range(n):
        for at in (slice(0, 4096), slice(rows // 2, rows // 2 + 4096), slice(rows - 4096, rows)):
            a, t = x[k][at].double(), pos[k][at].double()
            want = torch.stack([a[:, 0] * t.cos() - a[:, 1] * t.sin(), a[:, 0] * t.sin() + a[:, 1] * t.cos()], 1)
            check("rotary", y[k][at].float().cpu().numpy(), want.cpu().numpy(), H)
    st.close()


@pytest.mark.parametrize("flags", [0, 1])
@pytest.mark.parametrize("b,seq,heads,kv,dh,window,causal", [(40, 2, 8, 2, 80, 0, False), (2, 234, 8, 1, 128, 2, False), (30, 7, 4, 4, 64, 2, False), (16, 4, 16, 4, 32, 3, True),
                                                             (40, 3, 16, 8, 96, 0, True), (3, 1400, 4, 2, 64, 3, True)])
def test_gradients_of_queries_that_see_few_keys(b, seq, heads, kv, dh, window, causal, flags):
    """dP - rowsum(dO * O) loses what rounding O took off where O is nearly one of the few values, so the lower half of O is kept.  What is left
    are the roundings of the score gradients and of the result (of the probabilities and of the result in dV).  The relative
    errors of a rounding to 8 bits are spread evenly over +-2^-8 / m, m the value's mantissa from 1 to 2, evenly on a logarithmic scale:
    2^-8 sqrt(1/3 * 3 / (8 ln 2)) = 0.00166 in the root mean square.  Two of them are 0.00235; a fifth of that is allowed on top
    for tensors of some thousand values, and for the fp32 sums.  Without the lower half dQ is off by 0.0029 to 0.0037."""
    ops = S.attention_ops(b, seq, heads, kv, dh, window=window, causal=causal)
    batch, gout = S.draw(ops, b, 23)
    got, ref = S.gpu(ops, b, batch, gout, flags=flags), S.oracle(ops, b, batch, gout)
    rms = 2.0 ** -8 * (1 / (8 * np.log(2))) ** 0.5
    q, k = heads * dh, (heads + kv) * dh
    for name, at in (("dQ", slice(0, q)), ("dK", slice(q, k)), ("dV", slice(k, None))):
        e2, _ = S.rel(got[1][:, at], ref[1][:, at])
        print(f"{name} {e2:.5f}")
        assert e2 <= 1.2 * 2 ** 0.5 * rms, f"{name}: {e2:.5f}"
