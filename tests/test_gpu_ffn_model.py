"""Stages with token-wise layers (LINEAR, GATED; kept values in the tensors' type and in 8 bits) against the oracle: training
steps, partitions, the asynchronous pipeline, captured steps, traces and guard zones."""
import numpy as np
import pytest

import oracle
import synth
from helpers import TOL_BF16, TOL_FP32, clear_batch, gpu_step_split, make_gpu, rel_err, to_dev
from oracle import schedule as S

pytestmark = pytest.mark.gpu
F = pytest.importorskip("paper_2110_02781_b200")


def nets(kept=0, precision=0, **kw):
    ls, cfg = synth.token_ffn(kept=kept, precision=precision, **kw)
    return ls, cfg, synth.init_params(70, ls), synth.init_state(ls)


def border_distance(om):
    """Smallest distance, in steps, of a value that is kept in 8 bits from a rounding border: float32 and float64 then keep the
    same codes."""
    worst = 1.0
    for i, l in enumerate(om.layers):
        if l.k != 8 or l.kind not in (synth.KIND["LINEAR"], synth.KIND["GATED"]) or om.saved.get(i) is None:
            continue
        x = om.out[i - 1]
        for w in (om.p[i] if l.kind == synth.KIND["GATED"] else om.p[i][:1]):
            z = x @ w + (om.p[i][1] if l.kind == synth.KIND["LINEAR"] and l.has_bias else 0.0)
            for a in range(0, z.shape[-1], 32):
                v = z[..., a:a + 32]
                top = np.abs(v).max(-1, keepdims=True)
                q = np.abs(v / np.exp2(np.floor(np.log2(top)) - 6))
                q = q[q < 127]
                worst = min(worst, float(np.abs(q - np.floor(q) - 0.5).min()))
    return worst


def clear(ls, cfg, params, state, margin=1e-4):
    """The first batch whose kept values keep that distance (float32 noise there: 1e-6 of a value of at most 128 steps)."""
    for t in range(400):
        om = oracle.OracleModel(ls, cfg, params, state)
        x, y = synth.make_batch(70, cfg, t)
        om.forward(0, om.L, x, y)
        if border_distance(om) >= margin:
            return x, y
    raise RuntimeError("no clear batch")


@pytest.mark.parametrize("kept,points", [(0, None), (0, [0, 1, 2, 4]), (8, None), (8, [0, 2, 3, 4])])
def test_training_steps_match_the_oracle(kept, points):
    ls, cfg, params, state = nets(kept, batch=2, tokens=5, in_c=12, d=24, f=40)
    x, y = clear(ls, cfg, params, state) if kept else synth.make_batch(70, cfg)
    om = oracle.OracleModel(ls, cfg, params, state)
    gm = make_gpu(ls, cfg, 70)
    pts = points or [0, gm.L]
    gm.ftp_set_partition(pts)
    loss = gm.ftp_train_step(to_dev(x), to_dev(y), cfg["lr"])
    ref = om.step(pts, x, y)
    assert abs(loss - ref) <= TOL_FP32 * abs(ref)
    for u in range(gm.L):
        assert rel_err(gm.ftp_get_tensor(F.T_GRADS, u), om.unit_grads(u)) <= TOL_FP32, u
        assert rel_err(gm.ftp_get_tensor(F.T_WEIGHTS, u), om.unit_params(u)) <= TOL_FP32, u
    gm.ftp_check_guards()
    gm.ftp_check_device_status()
    gm.close()


@pytest.mark.parametrize("precision", [0, 1])
@pytest.mark.parametrize("kept", [0, 8])
def test_stage_grouping_changes_no_bit(precision, kept):
    ls, cfg, params, state = nets(kept, precision, batch=3, tokens=50, in_c=20, d=72, f=136)
    x, y = synth.make_batch(70, cfg)
    import torch
    xd = to_dev(x, torch.bfloat16 if precision else None)
    out = []
    for pts in ([0, 4], [0, 1, 2, 3, 4]):
        gm = make_gpu(ls, cfg, 70)
        gm.ftp_set_partition(pts)
        loss, _, _ = gpu_step_split(gm, pts, xd, to_dev(y), cfg["lr"])
        out.append((loss, [gm.ftp_get_tensor(F.T_GRADS, u) for u in range(gm.L)]))
        gm.ftp_check_guards()
        gm.close()
    assert out[0][0] == out[1][0]
    assert all(np.array_equal(a, b) for a, b in zip(out[0][1], out[1][1]))


@pytest.mark.parametrize("kept", [0, 8])
@pytest.mark.parametrize("cin,f", [(64, 96), (40, 100), (33, 70)])
def test_a_feed_forward_unit_in_bf16(kept, cin, f):
    """Forward and backward of one unit [GATED, LINEAR + bias + residual of the unit's input] on given boundary tensors."""
    import torch
    K, A, L = synth.KIND, synth.ACT, synth.Layer
    ls = [L(0, K["LINEAR"], cin, cin, 0, 1, 0, 0, 0, -1), L(1, K["GATED"], cin, f, kept, 1, 0, A["SILU"], 0, -1),
          L(1, K["LINEAR"], f, cin, kept, 1, 0, 0, 1, 0), L(2, K["GAP"], cin, cin, 0, 1, 0, 0, 0, -1), L(2, K["FC"], cin, 3, 1, 1, 0, 0, 1, -1),
          L(2, K["SOFTMAX_CE"], 3, 3, 0, 1, 0, 0, 0, -1)]
    cfg = synth.config(2, cin, 1, 35, 3, precision=1)
    params = synth.init_params(71, ls)
    params[2][1] = synth.rng_stream(71, "misc").standard_normal(cin).astype(np.float32)
    om = oracle.OracleModel(ls, cfg, params, synth.init_state(ls))
    gm = F.Model(ls, cfg)
    gm.load_params(params, synth.init_state(ls))
    g = synth.rng_stream(72, "misc")
    x = oracle.model.round_bf16(g.standard_normal((2, 1, 35, cin)))
    go = oracle.model.round_bf16(g.standard_normal((2, 1, 35, cin)))
    out, gin = (torch.empty((2, 1, 35, cin), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xd, god = to_dev(x, torch.bfloat16), to_dev(go, torch.bfloat16)      # a stage's input stays valid until its backward pass
    gm.ftp_run_stage_forward(1, 2, xd, out)
    gm.ftp_run_stage_backward(1, 2, god, gin)
    want = om.forward(1, 2, x)
    want_gin = om.backward(1, 2, go)
    assert rel_err(out.float().cpu().numpy(), want) <= TOL_BF16
    assert rel_err(gin.float().cpu().numpy(), want_gin) <= TOL_BF16
    assert rel_err(gm.ftp_get_tensor(F.T_GRADS, 1), om.unit_grads(1)) <= TOL_BF16
    gm.ftp_check_guards()
    gm.ftp_check_device_status()
    gm.close()


def test_async_pipeline_with_token_layers():
    from paper_2110_02781_b200.async_pipeline import AsyncPipeline
    ls, cfg, params, state = nets(0, batch=2, tokens=6, in_c=12, d=24, f=40)
    points, nb = [0, 1, 2, 4], 6
    op = S.AsyncPipeline(ls, cfg, params, state, points, 1)
    batches = [synth.make_batch(70, cfg, t) for t in range(nb)]
    ref = op.run(batches, cfg["lr"])
    gp = AsyncPipeline(ls, cfg, points, params, state, 1)
    got = gp.run([(to_dev(x), to_dev(y)) for x, y in batches], cfg["lr"])
    assert gp.log == op.log
    for b in range(nb):
        assert abs(got[b] - ref[b]) <= 5 * TOL_FP32 * abs(ref[b]), b
    for u in range(gp.L):                                            # several updates of drift, not one
        assert rel_err(gp.master.ftp_get_tensor(F.T_WEIGHTS, u), op.master.unit_params(u)) <= 1e-3, u
    gp.close()


def test_eight_bits_shrink_what_a_batch_in_flight_holds():
    big = dict(batch=8, tokens=512, in_c=64, d=256, f=1024)
    for precision, es in ((1, 2), (0, 4)):
        full, eight = (F.ftp_workspace_bytes(*synth.token_ffn(kept=k, precision=precision, **big))[0] for k in (0, 8))
        kept = 8 * 512 * (256 + 2 * 2 * 1024)                        # values before the activations: the first layer's, two per block
        saved = kept * (es - 33 / 32)
        assert abs((full - eight) - saved) <= 0.01 * saved


def test_captured_step_traces_and_profile():
    import torch
    ls, cfg, params, state = nets(8, 1, batch=2, tokens=40, in_c=32, d=64, f=128)
    x, y = synth.make_batch(70, cfg)
    xd, yd = to_dev(x, torch.bfloat16), to_dev(y)
    a, b = make_gpu(ls, cfg, 70), make_gpu(ls, cfg, 70)
    for m in (a, b):
        m.ftp_train_step(xd, yd, cfg["lr"])
    before = a.ftp_launch_count()
    a.ftp_train_step(xd, yd, cfg["lr"], want_loss=False)
    assert a.ftp_launch_count() - before >= 20
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        b.ftp_train_step(xd, yd, cfg["lr"], want_loss=False)
    graph.replay()
    torch.cuda.synchronize()
    for u in range(a.L):
        assert np.array_equal(a.ftp_get_tensor(F.T_WEIGHTS, u), b.ftp_get_tensor(F.T_WEIGHTS, u)), u
    del graph
    a.ftp_trace_enable(True)
    a.ftp_train_step(xd, yd, cfg["lr"])
    names = [r["kernel"] for r in a.ftp_trace_read()]
    assert names.count("gated_fwd") == names.count("gated_bwd") == 2 and names.count("linear_fwd") == names.count("linear_bwd") == 3
    a.ftp_trace_enable(False)
    f, bw, ob = a.ftp_profile_layers(2, xd, yd)
    assert (f > 0).all() and (bw > 0).all() and ob[0] == 2 * 40 * 64 * 2
    for m in (a, b):
        m.ftp_check_guards()
        m.close()


def mixed_net():
    """Token-wise layers among the other kinds: with RELU and RELU6, and residuals from a convolution, a batch norm that a gated
    block reads too, a linear op (read by an ADD_RESIDUAL), a sum and the unit's input."""
    K, A, d = synth.KIND, synth.ACT, 20
    L = lambda unit, kind, cin=d, cout=d, k=0, act="NONE", bias=0, src=-1, pad=0: synth.Layer(unit, K[kind], cin, cout, k, 1, pad, A[act], bias, src)  # noqa: E731
    ls = [L(0, "CONV1D", 12, d, 3, pad=1, bias=1), L(0, "LINEAR", act="RELU", bias=1, src=0),
          L(1, "BN"), L(1, "GATED", d, 36, act="RELU6"), L(1, "LINEAR", 36, d, src=2), L(1, "BN"), L(1, "ADD_RESIDUAL", src=4), L(1, "LINEAR", act="RELU6", src=6),
          L(2, "LINEAR", act="GELU", src=7), L(2, "ACT", act="RELU"), L(2, "GATED", act="RELU"), L(2, "LINEAR", src=9, bias=1),
          L(3, "GAP"), L(3, "FC", d, 5, 1, bias=1), L(3, "SOFTMAX_CE", 5, 5)]
    return ls, synth.config(2, 12, 1, 6, 5)


@pytest.mark.parametrize("points", [None, [0, 1, 2, 3, 4]])
def test_residuals_from_layers_of_every_kind(points):
    ls, cfg = mixed_net()
    params, state = synth.init_params(73, ls), synth.init_state(ls)
    probe = oracle.OracleModel(ls, cfg, params, state)
    x, y, _ = clear_batch(probe, 73, cfg)
    om = oracle.OracleModel(ls, cfg, params, state)
    gm = F.Model(ls, cfg)
    gm.load_params(params, state)
    pts = points or [0, gm.L]
    gm.ftp_set_partition(pts)
    loss = gm.ftp_train_step(to_dev(x), to_dev(y), cfg["lr"])
    ref = om.step(pts, x, y)
    assert abs(loss - ref) <= TOL_FP32 * abs(ref)
    for u in range(gm.L):
        assert rel_err(gm.ftp_get_tensor(F.T_GRADS, u), om.unit_grads(u)) <= TOL_FP32, u
        assert rel_err(gm.ftp_get_tensor(F.T_WEIGHTS, u), om.unit_params(u)) <= TOL_FP32, u
    gm.ftp_check_guards()
    gm.ftp_check_device_status()
    gm.close()


@pytest.mark.parametrize("kept,precision", [(8, 0), (0, 1), (8, 1)])
def test_async_pipeline_with_values_kept_in_8_bits(kept, precision):
    """Several micro-batches in flight.  A kept value next to a rounding border may land on the other side (1/64 of its block's
    largest): held to the bf16 tolerance, and to the same bits when the run is repeated."""
    import torch
    from paper_2110_02781_b200.async_pipeline import AsyncPipeline
    ls, cfg, params, state = nets(kept, precision, batch=2, tokens=6, in_c=16, d=24, f=40)
    points, nb = [0, 1, 2, 4], 6
    op = S.AsyncPipeline(ls, cfg, params, state, points, 1)
    batches = [synth.make_batch(70, cfg, t) for t in range(nb)]
    if precision:
        batches = [(oracle.model.round_bf16(x), y) for x, y in batches]
    ref = op.run(batches, cfg["lr"])
    runs = []
    for _ in range(2):
        gp = AsyncPipeline(ls, cfg, points, params, state, 1)
        got = gp.run([(to_dev(x, torch.bfloat16 if precision else None), to_dev(y)) for x, y in batches], cfg["lr"])
        assert gp.log == op.log
        for b in range(nb):
            assert abs(got[b] - ref[b]) <= TOL_BF16 * abs(ref[b]), b
        for u in range(gp.L):
            assert rel_err(gp.master.ftp_get_tensor(F.T_WEIGHTS, u), op.master.unit_params(u)) <= TOL_BF16, u
        runs.append((list(got), [gp.master.ftp_get_tensor(F.T_WEIGHTS, u) for u in range(gp.L)]))
        gp.close()
    assert runs[0][0] == runs[1][0] and all(np.array_equal(a, b) for a, b in zip(runs[0][1], runs[1][1]))
