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
