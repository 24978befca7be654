"""The operators of a training step together, as a program uses them: a small network whose linear layers run in microscaled 4 bits
forward and backward, gradients clipped by their global norm, Muon on the matrices, AdamW on the rest. Each stage is held against
fp64 formulas on the values that the stage before it produced."""
import numpy as np
import pytest
import torch

import oracle
from oracle import mx4, optim

E = 2.0 ** -24


class Recorder:
    def __init__(self):
        self.calls = []

    def defl_grad_norm(self, grads, max_norm, step=None):
        self.calls.append(("norm", list(grads), max_norm, step))
        return "clip"

    def defl_muon_step_batched(self, W, M, G, lr, mu, k, p, J, sched, **kw):
        self.calls.append(("muon", W, G, k, kw["grad_scale"], kw.get("nesterov")))

    def defl_adamw_step(self, group, grads, lr, step, grad_scale=None, **kw):
        self.calls.append(("adamw", group, list(grads), lr, step, grad_scale, kw))


def test_one_norm_for_both_kinds():
    """Host logic of the whole-model step (a recording stand-in for the context, no GPU)."""
    from paper_2609_21102_b200 import grouping
    rec = Recorder()
    clip = grouping.optimizer_step_groups(rec, {(4, 8): "W", (8, 8): "V"}, {(4, 8): "MW", (8, 8): "MV"}, {(4, 8): "GW", (8, 8): None}, 0.02, 0.95,
                                          1, 1, 1, [[1.0, 0.0, 0.0]], "rest", ["g0", None], 1e-3, "t", max_norm=2.0, adamw={"eps": 1e-6},
                                          nesterov=False)
    assert clip == "clip"
    assert rec.calls == [("norm", ["GW", "g0"], 2.0, "t"), ("muon", "W", "GW", 1, "clip", False), ("muon", "V", None, 1, "clip", False),
                         ("adamw", "rest", ["g0", None], 1e-3, "t", "clip", {"eps": 1e-6})]


@pytest.mark.parametrize("kw,rest_grads", [(dict(nesterov=True), ["g0", "g1"]), (dict(), ["g0"]), (dict(), ["g0", "g1", "g2"])])
def test_refused_step_changes_nothing(kw, rest_grads):
    """A group without a gradient under the Nesterov look-ahead, and gradients that are too few or too many: no call is made, so that neither the
    counter nor a weight has moved; the Muon groups alone refuse the same."""
    from paper_2609_21102_b200 import grouping

    class Rest:
        sizes = [10, 20]
    rec = Recorder()
    groups = ({(4, 8): "W", (8, 8): "V"}, {(4, 8): "MW", (8, 8): "MV"}, {(4, 8): "GW", (8, 8): None}, 0.02, 0.95, 1, 1, 1, [[1.0, 0.0, 0.0]])
    with pytest.raises(ValueError):
        grouping.optimizer_step_groups(rec, *groups, Rest(), rest_grads, 1e-3, "t", **kw)
    if kw:
        with pytest.raises(ValueError):
            grouping.muon_step_groups(rec, *groups, **kw)
    assert rec.calls == []


def test_gradients_from_a_generator():
    """The norm and the step read the same gradients, also where they come one after the other."""
    from paper_2609_21102_b200 import grouping
    rec = Recorder()
    grouping.optimizer_step_groups(rec, {}, {}, {}, 0.02, 0.95, 1, 1, 1, [[1.0, 0.0, 0.0]], "rest", (g for g in ("g0", None, "g2")), 1e-3, "t")
    assert [c[0] for c in rec.calls] == ["norm", "adamw"]
    assert rec.calls[0][1] == ["g0", "g2"] and rec.calls[1][2] == ["g0", None, "g2"]


def _dq(X, fmt):
    return np.stack([mx4.round_trip(x, fmt) for x in X])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("eight", [False, True])
def test_two_layer_network(fmt, eight):
    """y = relu(x w1^T + b1) w2^T + b2, L = mean (y - t)^2 / 2; w1 and w2^T share a stacked group."""
    from paper_2609_21102_b200 import binding, grouping
    ctx = binding.Context(0)
    rng = np.random.default_rng(1)
    T, d, h = 192, 64, 160
    x = torch.tensor(rng.standard_normal((1, T, d)), dtype=torch.bfloat16).cuda()
    target = torch.tensor(rng.standard_normal((T, d)), dtype=torch.float32).cuda()
    W = torch.tensor(rng.standard_normal((2, h, d)) / np.sqrt(d), dtype=torch.float32).cuda()          # w1 [h, d] and w2 stored as [h, d]
    Mom = torch.zeros(2, h, d, device="cuda")
    G = torch.full((2, h, d), float("nan"), device="cuda")
    biases = [torch.zeros(h, device="cuda"), torch.zeros(d, device="cuda")]
    if eight:
        moments = [[torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in (h, d)] for _ in range(2)]
        scales = [[torch.zeros(1, device="cuda") for _ in range(2)] for _ in range(2)]
    else:
        moments, scales = [[torch.zeros(n, device="cuda") for n in (h, d)] for _ in range(2)], [None, None]
    rest = binding.AdamWGroup(biases, moments[0], moments[1], *scales)
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    sched = [list(binding.MUON_QUINTIC)] * 5
    for t in range(1, 4):
        W0, Mom0, b0 = W.double().cpu().numpy(), Mom.double().cpu().numpy(), [b.double().cpu().numpy() for b in biases]
        state0 = [(optim.load8(m.double().cpu().numpy(), s.double().cpu().numpy()), optim.load8(r.double().cpu().numpy(), q.double().cpu().numpy()) ** 2)
                  for m, r, s, q in zip(moments[0], moments[1], *scales)] if eight else \
                 [(m.double().cpu().numpy(), v.double().cpu().numpy()) for m, v in zip(*moments)]
        # forward
        xq, xt = ctx.defl_mx4_quantize(x, fmt, both=True)
        w1, w1t = ctx.defl_mx4_quantize(W[:1], fmt, both=True)
        w2t, w2 = ctx.defl_mx4_quantize(W[1:], fmt, both=True)          # stored [h, d]: blocks along d, and of the transpose along h
        z = ctx.defl_mx4_gemm(xq, w1)
        a = torch.relu(z + biases[0])
        a16 = a.to(torch.bfloat16)
        aq, at = ctx.defl_mx4_quantize(a16, fmt, both=True)
        y = ctx.defl_mx4_gemm(aq, w2, out_dtype=torch.float32)[0] + biases[1]
        dy = ((y - target) / T)
        dy16 = dy[None].to(torch.bfloat16)
        # backward; the weights' gradients go straight into the stacked buffer
        dq, dt = ctx.defl_mx4_quantize(dy16, fmt, both=True)
        da = ctx.defl_mx4_gemm(dq, w2t)
        ctx.defl_mx4_gemm(at, dt, out=G[1:])                            # w2 is stored transposed, so is its gradient: a^T dy
        dz = da * (a > 0)
        zq, zt = ctx.defl_mx4_quantize(dz, fmt, both=True)
        ctx.defl_mx4_gemm(zt, xt, out=G[:1])
        gb = [dz[0].float().sum(0), dy16[0].float().sum(0)]
        # the products against fp64 on the rounded matrices (sums of K terms: K 2^-23 of the magnitudes; bf16 half a unit)
        for have, p, q, K in ((z, x, W[:1], d), (y - biases[1], a16, W[1:].transpose(1, 2), h), (da, dy16, W[1:], d),
                              (G[1:], a16.transpose(1, 2), dy16.transpose(1, 2), T), (G[:1], dz.transpose(1, 2), x.transpose(1, 2), T)):
            P, Q = _dq(p.double().cpu().numpy(), fmt), _dq(q.double().cpu().numpy(), fmt)
            want, size = P @ Q.transpose(0, 2, 1), np.abs(P) @ np.abs(Q).transpose(0, 2, 1)
            extra = 2.0 ** -8 * np.abs(want) if have.dtype == torch.bfloat16 else 0.0
            slack = 2.0 ** -22 * np.abs(biases[1].double().cpu().numpy()) if have.ndim == 2 else 0.0      # y was formed with the bias and freed of it
            assert np.all(np.abs(have.double().cpu().numpy() - want) <= 1.1 * (K * 2.0 ** -23 + 2.0 ** -20) * size + extra + slack + 1e-30)
        grads64 = [g.double().cpu().numpy() for g in (G, *gb)]
        Om = torch.randn(2, d, 8, generator=torch.Generator().manual_seed(t)).cuda()
        clip = grouping.optimizer_step_groups(ctx, {(h, d): W}, {(h, d): Mom}, {(h, d): G}, 0.02, 0.9, 4, 4, 1, sched, rest, gb, 1e-2, count,
                                              max_norm=0.05, adamw=dict(weight_decay=0.1, stochastic=eight, seed=7), nesterov=True, sketch=Om, gamma=1.01)
        norm, c = optim.grad_norm(grads64, 0.05)
        assert int(count) == t and abs(float(clip[0]) - norm) <= 6 * E * norm and abs(float(clip[1]) - c) <= 7 * E * c and c < 1
        c = float(clip[1])
        for i in range(2):
            # the gradient as both sides see it: scaled in fp32
            g = (G[i].cpu() * clip[1].cpu()).double().numpy()
            w, m = oracle.muon_step(W0[i], Mom0[i], g, 0.02, 0.9, 4, 8, Om[i].double().cpu().numpy(), 1, [oracle.MUON_QUINTIC] * 5, nesterov=True,
                                    storage="f32", gamma=1.01)
            step = w - W0[i]
            assert np.linalg.norm(W[i].double().cpu().numpy() - w) <= 2e-3 * np.linalg.norm(step) + E * np.linalg.norm(w)      # the Muon step's bar
        for i in range(2):
            p, m, v = optim.adamw(b0[i], grads64[1 + i], *state0[i], t, 1e-2, 0.9, 0.999, 1e-8, 0.1, c)
            # thirteen roundings of the step, three of the weight, the moment's own eight (which its parts share out between them)
            big = 1e-2 / (1 - 0.9 ** t) / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8) * (np.abs(0.9 * state0[i][0]) + np.abs(0.1 * c * grads64[1 + i]))
            assert np.all(np.abs(biases[i].double().cpu().numpy() - p) <= 1.1 * E * (3 * np.abs(b0[i]) + 22 * big) + 1e-30)
    assert ctx.defl_device_wait_status() == 0
    ctx.close()
