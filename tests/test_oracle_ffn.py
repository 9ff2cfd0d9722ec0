"""The oracle's token-wise layers (LINEAR, GATED, 8-bit kept values) pinned on the CPU: against torch's autograd in float64
and against differences of the loss."""
import numpy as np
import pytest
import torch

import oracle
import synth
from oracle import ops


@pytest.mark.parametrize("act", [0, 1, 2, 3, 4])
def test_activations_match_torch(act):
    z = torch.randn(200, dtype=torch.float64, requires_grad=True)
    f = {0: lambda v: v, 1: torch.relu, 2: torch.nn.functional.relu6, 3: torch.nn.functional.gelu, 4: torch.nn.functional.silu}[act]
    y = f(z)
    y.sum().backward()
    zn = z.detach().numpy()
    assert np.allclose(ops.act_fwd(zn, act), y.detach().numpy(), rtol=1e-12, atol=1e-14)
    assert np.allclose(ops.act_bwd(zn, np.ones_like(zn), act), z.grad.numpy(), rtol=1e-12, atol=1e-14)


def test_eight_bits_worked_example():
    x = np.zeros((1, 33))
    x[0, :4] = [100.0, 1.6, -0.4, 127.9]      # largest 127.9: scale 2^(6-6) = 1
    x[0, 32] = -3.0                             # its own block: scale 2^(1-6)
    out = ops.through_8_bits(x)
    assert out[0, :4].tolist() == [100.0, 2.0, -0.0, 127.0] and out[0, 32] == -3.0
    assert np.array_equal(ops.through_8_bits(out), out)


def _torch_loss(ls, params, x, labels):
    """The network in torch: float64, autograd."""
    K = synth.KIND
    acts = {0: lambda v: v, 3: torch.nn.functional.gelu, 4: torch.nn.functional.silu}
    outs = {-1: x}
    for i, l in enumerate(ls):
        h, p = outs[i - 1], params[i]
        if l.kind == K["LINEAR"]:
            y = acts[l.act](h @ p[0] + p[1])
            if l.residual_src >= 0:
                y = y + outs[l.residual_src]
        elif l.kind == K["GATED"]:
            y = acts[l.act](h @ p[0]) * (h @ p[1])
        elif l.kind == K["BN"]:
            mu, var = h.mean((0, 1, 2)), h.var((0, 1, 2), unbiased=False)
            y = (h - mu) / torch.sqrt(var + 1e-5) * p[0] + p[1]
        elif l.kind == K["GAP"]:
            y = h.mean((1, 2), keepdim=True)
        elif l.kind == K["FC"]:
            y = h.reshape(h.shape[0], -1) @ p[0].reshape(l.cin, l.cout) + p[1]
        else:
            return torch.nn.functional.cross_entropy(h, labels)
        outs[i] = y


def test_network_gradients_match_autograd():
    ls, cfg = synth.token_ffn()
    params = synth.init_params(60, ls)
    om = oracle.OracleModel(ls, cfg, params, synth.init_state(ls))
    x, y = synth.make_batch(60, cfg)
    om.forward(0, om.L, x, y)
    om.backward(0, om.L)
    tp = [[torch.tensor(a, dtype=torch.float64, requires_grad=True) for a in arrs] for arrs in params]
    loss = _torch_loss(ls, tp, torch.tensor(x, dtype=torch.float64), torch.tensor(y, dtype=torch.int64))
    loss.backward()
    assert abs(float(loss.detach()) - float(om.loss)) < 1e-12
    for i, arrs in enumerate(tp):
        for k, t in enumerate(arrs):
            assert np.allclose(om.g[i][k], t.grad.numpy(), rtol=1e-9, atol=1e-12), (i, k)


def test_kept_values_only_change_the_backward_pass():
    grads, losses = [], []
    for kept in (0, 8):
        ls, cfg = synth.token_ffn(kept=kept)
        om = oracle.OracleModel(ls, cfg, synth.init_params(61, ls), synth.init_state(ls))
        x, y = synth.make_batch(61, cfg)
        om.forward(0, om.L, x, y)
        om.backward(0, om.L)
        losses.append(float(om.loss))
        grads.append(np.concatenate([g.reshape(-1) for arrs in om.g for g in arrs]))
    assert losses[0] == losses[1]
    off = np.linalg.norm(grads[0] - grads[1]) / np.linalg.norm(grads[0])
    assert 0 < off < 1 / 32                    # a code is off by at most half a step of 1/64 of the block's largest value
