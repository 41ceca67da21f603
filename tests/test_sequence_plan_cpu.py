"""Plans of stages with several sequence operators (rotary positions, windowed attention), without a GPU: launches and memory."""
import pytest

from paper_2406_17145_amd import binding as B
from tests import sequence_util as S


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2406_17145_amd.build import build_library
        build_library(verbose=False)
    return B.load()


def branches(one, n):
    """n copies of an operator graph beside each other."""
    return [{**op, "inputs": [p + k * len(one) for p in op["inputs"]]} for k in range(n) for op in one]


def launches(ops, b):
    d, keep = B.build_desc(ops, b)
    return [s for s in B.gpp_stage_describe(d) if s["kernel"] != "loss_sum"]


@pytest.mark.parametrize("op", ["attention", "attention of one type on the matrix cores", "rotary"])
@pytest.mark.parametrize("grad", [False, True])
def test_launches_of_many_records_stay_below_2_to_the_32_threads(lib, op, grad):
    """Each of the three branches may have a launch of its own (7 * 2^20 workgroups of up to 512 threads, rotary 2^23 - 2^16 of 256);
    one launch of all three would have 5.6e9 threads or more."""
    b = 1 << 20
    if op == "rotary":
        one, threads, each = S.rotary_ops(b, 127, 1, 2, (1,), grad=grad), 256, 127 * b // 16
    else:
        mixed = op == "attention"
        one = S.attention_ops(b, 1, 7, 7, 12 if mixed else 8, grad=grad)
        threads, each = (256 if mixed else 512), 7 * b
    for n in (1, 2, 3):
        steps = launches(branches(one, n), b)
        for direction in ("forward", "backward") if grad else ("forward",):
            here = [s for s in steps if s["pass"] == direction]
            assert here and all(s["blocks"] * threads < 1 << 32 for s in here)
            for kernel in {s["kernel"] for s in here}:
                mine = [s for s in here if s["kernel"] == kernel]
                assert sum(s["records"] for s in mine) == n and sum(s["blocks"] for s in mine) == n * each


def test_branches_share_a_launch_where_they_fit(lib):
    for one in (S.attention_ops(4, 100, 4, 2, 64, window=9), S.rotary_ops(4, 100, 6, 64, (8, 12, 12))):
        assert [s["records"] for s in launches(branches(one, 5), 4)] == [5, 5]


@pytest.mark.parametrize("seq,window,sinks,causal", [(2048, 5, 300, False), (300, 20, 1000, False), (64, 64, 64, False), (64, 1, 64, False),
                                                     (90, 7, 8, False), (2048, 5, 300, True), (300, 20, 1000, True)])
def test_partition_costs_count_first_tokens_on_both_sides(monkeypatch, seq, window, sinks, causal):
    """Queries see first tokens ahead of a two-sided window too (by the operations alone)."""
    from types import SimpleNamespace
    from oracle import gpp_oracle as O
    from paper_2406_17145_amd import bench_partition as P
    ops = S.attention_ops(1, seq, 8, 2, 128, window=window, sinks=sinks, causal=causal)
    monkeypatch.setattr(P, "MEM_RATE", 1e30)
    _, t, _, _ = P.op_costs(SimpleNamespace(ops=ops, micro_batch=1))
    want = 4 * 3.5 * O.window_mask(seq, ops[1]).sum() * 1024 / P.MFMA_RATE
    assert abs(t[1] - want) <= 1e-12 * want


def cut_sums(ops, b):
    """Bytes of workspace beyond the tensors of a single attention whose gradient is wanted: its cut sums and, below 64 KB, tables."""
    up = lambda v: (v + 63) // 64 * 64  # noqa: E731
    x, a = ops[0], ops[-1]
    rows, size = b * x["seq_len"], 2 if x["dtype"] == "bf16" else 4
    d, keep = B.build_desc(ops, b)
    return B.gpp_stage_workspace_bytes(d) - rows * (up(x["out_features"]) + up(a["out_features"])) * size - 2 * up(rows * a["heads"]) * 4


def test_levels_share_the_memory_of_cut_sums(lib):
    """Three attentions in a row: the parts of one are joined before those of the next are written."""
    chain, parts, alone = [], [], []
    for heads, kv in ((16, 4), (12, 2), (4, 4)):
        one = S.attention_ops(4, 512, heads, kv, 64, window=100, causal=False)
        d, keep = B.build_desc(one, 4)
        alone.append(B.gpp_stage_workspace_bytes(d))
        parts.append(cut_sums(one, 4))
        chain = chain + [{**one[1], "inputs": [len(chain) - 1]}] if chain else one
    assert sum(parts) - max(parts) > 8 << 20
    d, keep = B.build_desc(chain, 4)
    # (one's output is the next one's input: a gradient of it in the place of the copy of the caller's rows)
    assert B.gpp_stage_workspace_bytes(d) <= sum(alone) - sum(parts) + max(parts) + (64 << 10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 700, 300), (False, 4000, 0)])
@pytest.mark.parametrize("b,seq,heads,kv,dh", [(1, 32768, 4, 1, 128), (1, 32768, 2, 1, 32), (1, 23721, 8, 2, 32), (2, 4096, 8, 2, 128), (1, 16384, 16, 2, 128),
                                               (3, 1500, 6, 3, 96), (5, 2000, 8, 1, 64), (1, 100000, 32, 1, 64), (64, 700, 4, 4, 80), (4, 512, 16, 4, 64)])
def test_memory_of_cut_sums_is_bounded(lib, dtype, causal, window, sinks, b, seq, heads, kv, dh):
    """64 MB or twice the gradient, whichever is more, and a megabyte for everything else."""
    gradient = b * seq * (heads + 2 * kv) * dh * (2 if dtype == "bf16" else 4)
    ops = S.attention_ops(b, seq, heads, kv, dh, window=window, sinks=sinks, causal=causal, dtype=dtype)
    assert cut_sums(ops, b) <= max(64 << 20, 2 * gradient) + (1 << 20)


@pytest.mark.parametrize("causal,window,sinks,kept", [(True, 40, 0, True), (True, 60, 0, False), (False, 20, 0, True), (False, 30, 0, False), (True, 20, 20, True),
                                                      (True, 20, 40, False), (True, 1, 0, False), (False, 1, 0, False), (False, 1, 1, True), (True, 0, 0, False)])
def test_lower_half_of_the_output_is_kept_for_few_keys(lib, causal, window, sinks, kept):
    """In bf16; fp32 has none."""
    seq, heads, kv, dh = 16384, 8, 8, 64
    size = seq * heads * dh * 2
    for dtype in ("bf16", "f32"):
        ops = S.attention_ops(1, seq, heads, kv, dh, window=window, sinks=sinks, causal=causal, dtype=dtype)
        d, keep = B.build_desc(ops, 1)
        used = sum(s["kernel"] == "attention_bwd_dkv" for s in B.gpp_stage_describe(d)) > 1        # (cut sums beside it)
        extra = cut_sums(ops, 1)
        if not used:
            assert abs(extra - (size if kept and dtype == "bf16" else 0)) < 64 << 10
        else:
            assert extra >= (size if kept and dtype == "bf16" else 0)
