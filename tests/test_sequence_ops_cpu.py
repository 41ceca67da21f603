"""Rotary positions and windowed attention without a GPU: pins of the oracle (finite differences, autograd, closed forms), what the
planner refuses, and which buffers and launches a stage of them has."""
import copy

import numpy as np
import pytest
import torch

from oracle import gpp_oracle as O
from paper_2406_17145_amd import binding as B
from paper_2406_17145_amd import workloads as W
from tests import sequence_util as S


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2406_17145_amd.build import build_library
        build_library(verbose=False)
    return B.load()


CASES = [dict(b=2, seq=7, heads=4, kv=2, dh=4, window=3, sinks=2, causal=True, lengths=True),
         dict(b=2, seq=6, heads=2, kv=2, dh=3, window=2, sinks=4, causal=False),
         dict(b=1, seq=9, heads=3, kv=1, dh=4, window=0, causal=True),
         dict(b=3, seq=5, heads=2, kv=1, dh=4, window=9, sinks=1, causal=False, lengths=True, scale=0.3),
         dict(b=2, seq=1, heads=2, kv=2, dh=4, window=1, causal=True)]


def lengths_of(seq):
    return {1: lambda r, s: r.integers(0, seq + 1, s)}


@pytest.mark.parametrize("case", CASES)
def test_window_oracle_against_differences(case):
    ops = S.attention_ops(dtype="f32", **case)
    batch, gout = S.draw(ops, case["b"], 1, lengths_of(case["seq"]))
    _, grad = S.oracle(ops, case["b"], batch, gout)
    x = batch[0].astype(np.float64)
    rng = np.random.default_rng(2)
    for _ in range(25):
        at, h = (rng.integers(x.shape[0]), rng.integers(x.shape[1])), 1e-5
        side = []
        for s in (h, -h):
            y = x.copy()
            y[at] += s
            st = O.OracleStage(ops, case["b"], {})
            side.append((st.forward({**batch, 0: y}).values[len(ops) - 1] * gout[len(ops) - 1]).sum())
        assert abs((side[0] - side[1]) / (2 * h) - grad[at]) <= 1e-7 * max(1.0, abs(grad[at]))


@pytest.mark.parametrize("case", CASES)
def test_window_oracle_against_autograd(case):
    """The library routine with an explicit mask, key / value heads repeated, one sample at a time."""
    ops = S.attention_ops(dtype="f32", **case)
    batch, gout = S.draw(ops, case["b"], 3, lengths_of(case["seq"]))
    out, grad = S.oracle(ops, case["b"], batch, gout)
    b, s, hq, hk, dh = (case[k] for k in ("b", "seq", "heads", "kv", "dh"))
    x = torch.tensor(batch[0], dtype=torch.float64, requires_grad=True)
    y = torch.zeros(b * s, hq * dh, dtype=torch.float64)
    n = batch[1].reshape(-1) if case.get("lengths") else [s] * b
    total = torch.zeros((), dtype=torch.float64)
    for k in range(b):
        m = int(n[k])
        if m == 0:
            continue
        r = x[k * s:k * s + m].reshape(m, hq + 2 * hk, dh).transpose(0, 1)
        rep = lambda t: t.repeat_interleave(hq // hk, 0)  # noqa: E731
        i = torch.arange(m)
        back = i[:, None] - i[None, :]
        seen = torch.ones(m, m, dtype=torch.bool) if not case["window"] else (back.abs() < case["window"]) | (i[None, :] < case.get("sinks", 0))
        if case["causal"]:
            seen = seen & (back >= 0)
        o = torch.nn.functional.scaled_dot_product_attention(r[:hq], rep(r[hq:hq + hk]), rep(r[hq + hk:]), attn_mask=seen,
                                                             scale=case.get("scale") or None).transpose(0, 1).reshape(m, hq * dh)
        y[k * s:k * s + m] = o.detach()
        total = total + (o * torch.tensor(gout[len(ops) - 1][k * s:k * s + m])).sum()
    total.backward() if total.requires_grad else None
    assert np.abs(out - y.numpy()).max() <= 1e-12
    assert np.abs(grad - (x.grad.numpy() if x.grad is not None else 0.0)).max() <= 1e-12


def test_window_oracle_closed_forms():
    ops = S.attention_ops(1, 6, 1, 1, 2, window=1, causal=True, dtype="f32")
    batch, gout = S.draw(ops, 1, 4)
    out, grad = S.oracle(ops, 1, batch, gout)
    assert np.array_equal(out, batch[0][:, 4:].astype(np.float64))         # each token sees itself only
    assert np.array_equal(grad[:, :4], np.zeros((6, 4))) and np.array_equal(grad[:, 4:], gout[1].astype(np.float64))
    # no window, both sides: the plain attention operator
    ops = S.attention_ops(2, 5, 2, 2, 3, dtype="f32")
    batch, gout = S.draw(ops, 2, 5)
    plain = [ops[0], dict(kind="attention", inputs=[0], out_features=6, heads=2, seq_len=5, dtype="f32")]
    for a, c in zip(S.oracle(ops, 2, batch, gout), S.oracle(plain, 2, batch, gout)):
        assert np.abs(a - c).max() <= 1e-13


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("ladder", ["shared", "per_axis"])
def test_rotary_oracle(pairing, ladder):
    ops = S.rotary_ops(2, 5, 3, 14, (3, 1, 2), rest=4, base=100.0, pairing=pairing, ladder=ladder, dtype="f32")
    batch, gout = S.draw(ops, 2, 6, {1: lambda r, s: r.integers(-50, 1 << 20, s)})
    out, grad = S.oracle(ops, 2, batch, gout)
    x = batch[0].astype(np.float64)
    # norms of the turned blocks and every other column stay; the gradient is the transpose: <out, g> = <x, grad>
    for h in range(3):
        assert np.allclose(np.linalg.norm(out[:, 14 * h:14 * h + 12], axis=1), np.linalg.norm(x[:, 14 * h:14 * h + 12], axis=1), rtol=1e-13)
        assert np.array_equal(out[:, 14 * h + 12:14 * h + 14], x[:, 14 * h + 12:14 * h + 14])
    assert np.array_equal(out[:, 42:], x[:, 42:])
    assert abs((out * gout[2]).sum() - (x * grad).sum()) <= 1e-10
    # scores of turned queries and keys depend on differences of positions only
    shifted = {**batch, 1: batch[1] + np.array([[7, 3, 11]], np.int32)}
    again, _ = S.oracle(ops, 2, shifted, gout)
    dot = lambda y: y[:, :12] @ y[:, 14:26].T  # noqa: E731
    assert np.abs(dot(out) - dot(again)).max() <= 1e-8 * np.abs(dot(out)).max()
    # complex numbers: the first pair of the first axis turns by the position itself
    second = 1 if pairing == "neighbours" else 6
    z = (x[:, 0] + 1j * x[:, second]) * np.exp(1j * batch[1][:, 0].astype(np.float64))
    assert np.abs(out[:, 0] - z.real).max() <= 1e-9 and np.abs(out[:, second] - z.imag).max() <= 1e-9


def _status(ops, b=4):
    d, keep = B.build_desc(ops, b)
    with pytest.raises(B.GppError) as e:
        B.gpp_stage_workspace_bytes(d)
    return e.value.status


def _changed(ops, at, **kw):
    ops = copy.deepcopy(ops)
    ops[at].update(kw)
    return ops


def test_window_refusals(lib):
    ops = S.attention_ops(4, 16, 4, 2, 64, window=3, causal=True, lengths=True)
    d, keep = B.build_desc(ops, 4)
    assert B.gpp_stage_workspace_bytes(d) > 0
    for kw, want in [(dict(kv_heads=3), B.GPP_ERR_SHAPE), (dict(kv_heads=0), B.GPP_ERR_SHAPE), (dict(heads=0), B.GPP_ERR_SHAPE),
                     (dict(head_dim=32), B.GPP_ERR_SHAPE), (dict(head_dim=0), B.GPP_ERR_SHAPE), (dict(out_features=512), B.GPP_ERR_SHAPE),
                     (dict(seq_len=15), B.GPP_ERR_SHAPE), (dict(seq_len=0), B.GPP_ERR_SHAPE), (dict(window=-1), B.GPP_ERR_INVALID_ARG),
                     (dict(sinks=-1), B.GPP_ERR_INVALID_ARG), (dict(scale=-1.0), B.GPP_ERR_INVALID_ARG),
                     (dict(scale=float("nan")), B.GPP_ERR_INVALID_ARG), (dict(scale=1e300), B.GPP_ERR_INVALID_ARG),
                     (dict(inputs=[0, 0]), B.GPP_ERR_BAD_GRAPH), (dict(inputs=[]), B.GPP_ERR_BAD_GRAPH), (dict(inputs=[0, 1, 1]), B.GPP_ERR_BAD_GRAPH),
                     (dict(dtype="i32"), B.GPP_ERR_UNSUPPORTED)]:
        assert _status(_changed(ops, 2, **kw)) == want, kw
    assert _status(_changed(ops, 1, out_features=2)) == B.GPP_ERR_SHAPE
    assert _status(_changed(ops, 1, seq_len=2)) == B.GPP_ERR_SHAPE
    assert _status(_changed(ops, 1, dtype="f32")) == B.GPP_ERR_BAD_GRAPH
    assert _status(_changed(ops, 0, out_features=500)) == B.GPP_ERR_SHAPE
    assert _status(S.attention_ops(4, 4, 1, 1, 264)) == B.GPP_ERR_UNSUPPORTED
    assert _status(S.attention_ops(64, 1 << 20, 1, 1, 8), 64) == B.GPP_ERR_UNSUPPORTED


def test_rotary_refusals(lib):
    ops = S.rotary_ops(4, 16, 6, 64, (8, 12, 12), rest=128)
    d, keep = B.build_desc(ops, 4)
    assert B.gpp_stage_workspace_bytes(d) > 0
    for kw, want in [(dict(heads=0), B.GPP_ERR_SHAPE), (dict(heads=9), B.GPP_ERR_SHAPE), (dict(head_dim=0), B.GPP_ERR_SHAPE),
                     (dict(out_features=448), B.GPP_ERR_SHAPE), (dict(axis_pairs=[8, 12, 13]), B.GPP_ERR_SHAPE),
                     (dict(axis_pairs=[8, 12]), B.GPP_ERR_SHAPE), (dict(axis_pairs=[0, 0, 0]), B.GPP_ERR_INVALID_ARG),
                     (dict(axis_pairs=[8, 0, 12, 4]), B.GPP_ERR_INVALID_ARG), (dict(axis_pairs=[8, -1, 12]), B.GPP_ERR_INVALID_ARG),
                     (dict(base=0.0), B.GPP_ERR_INVALID_ARG), (dict(base=float("inf")), B.GPP_ERR_INVALID_ARG),
                     (dict(dtype="f32"), B.GPP_ERR_UNSUPPORTED), (dict(inputs=[0]), B.GPP_ERR_BAD_GRAPH), (dict(inputs=[0, 0]), B.GPP_ERR_BAD_GRAPH)]:
        assert _status(_changed(ops, 2, **kw)) == want, kw
    assert _status(_changed(ops, 1, seq_len=15)) == B.GPP_ERR_SHAPE
    assert _status(_changed(ops, 1, dtype="f32")) == B.GPP_ERR_BAD_GRAPH
    assert _status(S.rotary_ops(4, 4, 1, 2048, (1000,))) == B.GPP_ERR_UNSUPPORTED


def test_refusals_at_the_ends_of_ranges(lib):
    ops = S.attention_ops(4, 16, 4, 2, 64)
    for scale in (1e-50, 1e-40, 2e38):          # fp32 holds no such factor, or no product with log2 e
        assert _status(_changed(ops, 1, scale=scale)) == B.GPP_ERR_INVALID_ARG
    for scale in (1e-30, 1e30):
        d, keep = B.build_desc(_changed(ops, 1, scale=scale), 4)
        assert B.gpp_stage_workspace_bytes(d) > 0
    b = 1 << 20
    for heads, want in ((16, B.GPP_ERR_UNSUPPORTED), (8, B.GPP_ERR_UNSUPPORTED), (7, None)):      # single tokens: workgroups of a launch
        ops = S.attention_ops(b, 1, heads, heads, 8)
        if want is not None:
            assert _status(ops, b) == want
        else:
            d, keep = B.build_desc(ops, b)
            assert B.gpp_stage_workspace_bytes(d) > 0
    with pytest.raises(ValueError):
        B.build_desc(S.rotary_ops(4, 16, 6, 64, (1, 1, 1, 1, 1)), 4)
    assert _status(S.rotary_ops(1, 1 << 29, 1, 2, (1,)), 1) == B.GPP_ERR_UNSUPPORTED      # more workgroups than a launch has


def _launches(ops, b):
    d, keep = B.build_desc(ops, b)
    # (without loss operators the loss sum writes a zero where the caller asks for one)
    return [(s["pass"], s["kernel"]) for s in B.gpp_stage_describe(d) if s["kernel"] != "loss_sum"], B.gpp_stage_workspace_bytes(d)


def test_a_stage_of_one_operator_works_on_the_callers_tensors(lib):
    """No copies in or out: two launches for a rotary, for an attention forward (which keeps Q, K and V)
    and backward, the gradients in one launch of few workgroups or two."""
    steps, size = _launches(S.rotary_ops(2, 64, 6, 64, (8, 12, 12), rest=128), 2)
    assert steps == [("forward", "elt_fwd"), ("backward", "elt_bwd")]
    assert size < 64 * 1024          # positions (rows padded to 64) and tables: no tensor of [128, 512]
    steps, size = _launches(S.attention_ops(2, 64, 4, 2, 64, window=9, lengths=True, grad=False), 2)
    assert steps == [("forward", "attention_fwd")] and size < 8192
    steps, _ = _launches(S.attention_ops(2, 64, 4, 2, 64, window=9, lengths=True), 2)
    assert steps == [("forward", "attention_fwd"), ("backward", "attention_bwd_dkv")]
    steps, _ = _launches(S.attention_ops(16, 1024, 8, 2, 64, window=9), 16)
    assert steps == [("forward", "attention_fwd"), ("backward", "attention_bwd_dq"), ("backward", "attention_bwd_dkv")]


def test_a_layer_in_front_of_a_rotary_shares_its_buffers(lib):
    kw = dict(micro_batch=2, n_branches=1, n_layers=1, d_model=128, heads=2, d_ff=128, seq_len=16, axis_pairs=[(16, 16)])
    turned, plain = W.mmt(**kw), W.mmt(**{**kw, "axis_pairs": [(16, 16)]})
    at = next(i for i, o in enumerate(plain.ops) if o["kind"] == "rotary")
    plain.ops[at - 1]["act"] = "gelu"       # keeps its output: buffers of their own
    size = []
    for wl in (turned, plain):
        d, keep = B.build_desc(wl.ops, wl.micro_batch)
        size.append(B.gpp_stage_workspace_bytes(d))
    assert size[1] - size[0] >= 3 * 32 * 384 * 2        # value, gradient, stashed derivative of [32, 384]


def test_partition_costs_count_the_visible_pairs():
    from types import SimpleNamespace
    from paper_2406_17145_amd import bench_partition as P
    for seq, window, sinks, causal in [(2048, 0, 0, True), (2048, 0, 0, False), (2048, 100, 30, True), (2048, 100, 0, False), (2048, 2048, 9, True)]:
        ops = S.attention_ops(1, seq, 8, 2, 128, window=window, sinks=sinks, causal=causal)
        _, t, _, _ = P.op_costs(SimpleNamespace(ops=ops, micro_batch=1))
        seen = O.window_mask(seq, ops[1]).sum()
        assert abs(t[1] - max(4 * 3.5 * seen * 1024 / P.MFMA_RATE, seq * 1024 * 2 * (4 * 1.5 + 4) / P.MEM_RATE)) <= 1e-12 * t[1]
