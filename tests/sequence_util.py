"""Single-operator stages of the sequence operators (rotary positions, windowed attention), their inputs and their comparison
with the fp64 oracle."""
import numpy as np

from oracle import gpp_oracle as O
from paper_2406_17145_amd import workloads as W

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def attention_ops(b, seq, heads, kv, dh, window=0, sinks=0, causal=False, lengths=False, dtype="bf16", out_dtype=None, scale=0.0,
                  grad=True):
    ops = [dict(kind="input", inputs=[], out_features=(heads + 2 * kv) * dh, seq_len=seq, dtype=dtype, rows_extra=0,
                role="data" if grad else "frozen")]
    if lengths:
        ops.append(dict(kind="input", inputs=[], out_features=1, seq_len=1, dtype="i32", rows_extra=0, role="lengths"))
    ops.append(dict(kind="attention_window", inputs=[0, 1] if lengths else [0], out_features=heads * dh, heads=heads, kv_heads=kv,
                    head_dim=dh, window=window, sinks=sinks, causal=causal, scale=scale, seq_len=seq, dtype=out_dtype or dtype))
    return ops


def rotary_ops(b, seq, heads, dh, pairs, rest=0, base=10000.0, pairing="halves", ladder="shared", dtype="bf16", grad=True):
    feat = heads * dh + rest
    return [dict(kind="input", inputs=[], out_features=feat, seq_len=seq, dtype=dtype, rows_extra=0, role="data" if grad else "frozen"),
            dict(kind="input", inputs=[], out_features=len(pairs), seq_len=seq, dtype="i32", rows_extra=0, role="positions"),
            dict(kind="rotary", inputs=[0, 1], out_features=feat, heads=heads, head_dim=dh, axis_pairs=list(pairs), base=base,
                 pairing=pairing, ladder=ladder, seq_len=seq, dtype=dtype)]


def draw(ops, b, seed, samplers=None):
    """Inputs and the gradient of the last operator's output, exactly representable in their types."""
    rng = np.random.default_rng(seed)

    def tensor(op, rows):
        a = rng.standard_normal((rows, op["out_features"])).astype(np.float32)
        return W.round_to_bf16(a) if op["dtype"] == "bf16" else a
    batch = {}
    for i, op in enumerate(ops):
        if op["kind"] != "input":
            continue
        rows = b * op["seq_len"] + op["rows_extra"]
        if op["dtype"] == "i32":
            batch[i] = np.ascontiguousarray((samplers or {})[i](rng, (rows, op["out_features"])), dtype=np.int32)
        else:
            batch[i] = tensor(op, rows)
    return batch, {len(ops) - 1: tensor(ops[-1], b * ops[0]["seq_len"])}


def oracle(ops, b, batch, gout, rounded=True):
    st = O.OracleStage(ops, b, {}, model_storage=False)
    s = st.forward(batch)
    return s.values[len(ops) - 1], st.backward(s, gout).get(0)


def rel(got, ref):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all(), "shape or not finite"
    n, m = np.linalg.norm(ref), np.abs(ref).max() if ref.size else 0.0
    if n == 0.0:
        return float(np.linalg.norm(got)), float(np.abs(got).max() if got.size else 0.0)
    return float(np.linalg.norm(got - ref) / n), float(np.abs(got - ref).max() / m)


def gpu(ops, b, batch, gout, slots=1, flags=0, slot=0):
    from paper_2406_17145_amd import binding as B
    st = B.Stage(ops, b, {}, slots=slots, flags=flags)
    outs, _ = st.forward(slot, batch)
    gin = st.backward(slot, gout)
    st.sync_status()
    res = outs[0].float().cpu().numpy(), None if gin[0] is None else gin[0].float().cpu().numpy()
    st.close()
    return res
