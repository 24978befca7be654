"""defl_adamw_step and defl_grad_norm on the GPU against the fp64 oracle, element by element.

Bounds (E = 2^-24, half a unit of fp32): the factor c and each constant of the step are fp32 (E each), every operation rounds
once (E), so with a = |beta1 m|, b = |(1 - beta1) c g|
  m: c g 2E, (1 - beta1) and its product 2E, beta1 and its product 2E, the sum E of at most a + b -> E (3a + 5b)
  v: all terms positive: (c g)^2 5E, constant and product 2E, sum E                             -> 8E v
  sqrt(v): 4E + E; its product with 1 / sqrt(1 - beta2^t) and the sum with eps: 2E more         -> 7E of the denominator
  p: decay factor, product, sum: 3E |p|; step: m's error over the denominator + (7 + 1 of the step size + 4 of the quotient, whose
     documented error is 2 units, + 1 of the sum = 13) E |step|
A tenth more covers the second order. Stored bf16 adds half a unit, 2^-8.
"""
import numpy as np
import pytest
import torch

from oracle import optim

E = 2.0 ** -24
B1, B2, EPS, WD, LR = 0.9, 0.999, 1e-8, 0.1, 1e-2
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_21102_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


def _gen(seed):
    return np.random.default_rng(seed)


class Problem:
    """A list of tensors with states, on the GPU, and the same in fp64."""

    def __init__(self, sizes, p_dtype, g_dtype, eight, seed, offset=0, copies=False, fresh=False):
        rng = _gen(seed)
        self.sizes, self.eight = sizes, eight
        self.p, self.g, self.m, self.v, self.ms, self.vs, self.c = [], [], [], [], [], [], []
        self.p64, self.g64, self.m64, self.v64 = [], [], [], []

        def dev(x, dtype):
            t = torch.empty(x.size + offset, dtype=dtype, device="cuda")[offset:]
            t.copy_(torch.tensor(x).to(dtype))
            return t
        for n in sizes:
            p = dev(rng.standard_normal(n), p_dtype)
            size = np.exp(2 * rng.standard_normal(n))
            g = dev(size * rng.standard_normal(n) * (rng.random(n) < 0.8), g_dtype)
            root = np.zeros(n) if fresh else size * (0.3 + rng.random(n))
            m = 0.5 * root * rng.standard_normal(n)
            self.p.append(p)
            self.g.append(g)
            if eight:
                (qm, sm), (qv, sv) = optim.store8(m, None, False), optim.store8(root, None, True)
                self.m.append(dev(qm, torch.float8_e4m3fn))
                self.v.append(dev(qv, torch.float8_e4m3fn))
                self.ms.append(torch.tensor(sm, dtype=F32, device="cuda"))
                self.vs.append(torch.tensor(sv, dtype=F32, device="cuda"))
                self.m64.append(optim.load8(qm, sm.astype(np.float32).astype(np.float64)))
                self.v64.append(optim.load8(qv, sv.astype(np.float32).astype(np.float64)) ** 2)
            else:
                self.m.append(dev(m, F32))
                self.v.append(dev(root * root, F32))
                self.m64.append(self.m[-1].double().cpu().numpy())
                self.v64.append(self.v[-1].double().cpu().numpy())
            self.c.append(torch.zeros(n + offset, dtype=BF16, device="cuda")[offset:] if copies else None)
            self.p64.append(p.double().cpu().numpy())
            self.g64.append(g.double().cpu().numpy())

    def group(self):
        from paper_2609_21102_b200 import binding
        return binding.AdamWGroup(self.p, self.m, self.v, self.ms if self.eight else None, self.vs if self.eight else None, copies=self.c)

    def check(self, t, c=1.0, stochastic=False, seed=0, lr=LR, skip=()):
        for i, n in enumerate(self.sizes):
            if i in skip or n == 0:
                continue
            p0, g0, m0, v0 = self.p64[i], self.g64[i], self.m64[i], self.v64[i]
            p, m, v = optim.adamw(p0, g0, m0, v0, t, lr, B1, B2, EPS, WD, c)
            low, high = optim.random_bits(seed, t, i, n)
            held = 4 * E if self.eight else 0.0          # code times scale, squared: two roundings each
            err_m = 1.1 * E * ((4 if self.eight else 3) * np.abs(B1 * m0) + 5 * np.abs((1 - B1) * c * g0))
            err_v = 1.1 * (8 * E + held) * v
            step = np.abs(p - (1 - lr * WD) * p0)
            denom = lr / (1 - B1 ** t) / (np.sqrt(v / (1 - B2 ** t)) + EPS)
            err_p = 1.1 * (3 * E * np.abs(p0) + denom * err_m + (13 * E + held) * step) + 1e-40
            got = self.p[i].double().cpu().numpy()
            if self.p[i].dtype == F32:
                assert np.all(np.abs(got - p) <= err_p), (i, n, np.max(np.abs(got - p) / err_p))
                if self.c[i] is not None:
                    assert torch.equal(self.c[i], self.p[i].to(BF16))
            elif stochastic:
                want = optim.bf16_stochastic(p, high)
                spacing = np.ldexp(1.0, np.frexp(np.maximum(np.abs(p), 2.0 ** -126))[1] - 8)
                off = got != want
                # only where the error of p moves it over the border, and then to the neighbour
                border = np.abs(np.abs(p) / spacing + high / 65536.0 - np.rint(np.abs(p) / spacing + high / 65536.0)) * spacing
                assert np.all(border[off] <= err_p[off]) and np.all(np.abs(got - want)[off] <= 2 * spacing[off])
            else:
                assert np.all(np.abs(got - p) <= np.abs(p) * 2.0 ** -8 + err_p * (1 + 2.0 ** -8))
            if not self.eight:
                assert np.all(np.abs(self.m[i].double().cpu().numpy() - m) <= err_m + 1e-45)
                assert np.all(np.abs(self.v[i].double().cpu().numpy() - v) <= err_v + 1e-45)
                continue
            for q, scale, x, err, bits, keep in ((self.m[i], self.ms[i], m, err_m, low, False),
                                                 (self.v[i], self.vs[i], np.sqrt(v), 0.6 * err_v / np.sqrt(np.maximum(v, 1e-300)) + E * np.sqrt(v), high, True)):
                want, s64 = optim.store8(x, bits if stochastic else None, keep)
                y, _ = optim.scaled_blocks(x)
                big = np.repeat(s64, 256)[:n] * 448.0
                got_s = scale.double().cpu().numpy()
                err_blocks = np.zeros(s64.size * 256)
                err_blocks[:n] = err
                worst = err_blocks.reshape(-1, 256).max(axis=1) / 448.0
                assert np.all(np.abs(got_s - s64) <= worst + 2 * E * s64 + 1e-45)
                got = q.double().cpu().numpy()
                # y's error: the value's own and the largest's, in units of y, and three roundings
                rel = np.repeat(worst, 256)[:n] * 448.0 / np.where(big > 0, big, 1.0)
                err_y = np.where(big > 0, err * 448.0 / np.where(big > 0, big, 1.0), 0.0) + y * (rel + 4 * E)
                d = optim.e4m3_spacing(y)
                u = bits / 65536.0 if stochastic else 0.5
                where = y / d + u
                # (the 16 bits are added where fp32 holds 20 below the cut: y is first rounded to 2^-23 of itself, or of 2^-6)
                border = np.abs(where - np.rint(where)) * d
                off = got != want
                assert np.all(border[off] <= err_y[off] + 2.0 ** -29), (i, int(off.sum()))
                assert np.all(np.abs(got - want)[off] <= 2 * d[off])


SIZES = [1, 255, 256, 257, 0, 2048, 2049, 5000, 7]


@pytest.mark.gpu
@pytest.mark.parametrize("p_dtype", [F32, BF16])
@pytest.mark.parametrize("g_dtype", [F32, BF16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_step_matches_oracle(ctx, p_dtype, g_dtype, eight, stochastic, offset):
    pr = Problem(SIZES, p_dtype, g_dtype, eight, 11, offset, copies=p_dtype == F32)
    ctx.defl_adamw_step(pr.group(), pr.g, LR, 7, betas=(B1, B2), eps=EPS, weight_decay=WD, stochastic=stochastic, seed=123)
    pr.check(7, stochastic=stochastic, seed=123)


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
def test_first_step_from_zero_moments(ctx, eight):
    pr = Problem([300, 1000], F32, F32, eight, 12, fresh=True)
    ctx.defl_adamw_step(pr.group(), pr.g, LR, 1, betas=(B1, B2), eps=EPS, weight_decay=WD, stochastic=True, seed=5)
    pr.check(1, stochastic=True, seed=5)


@pytest.mark.gpu
def test_more_tensors_than_one_launch_holds(ctx):
    rng = _gen(13)
    sizes = [int(x) for x in rng.integers(1, 700, 1000)]
    pr = Problem(sizes, F32, BF16, True, 13)
    before = ctx.defl_launch_count()
    ctx.defl_adamw_step(pr.group(), pr.g, LR, 3, betas=(B1, B2), eps=EPS, weight_decay=WD, stochastic=True, seed=9)
    assert ctx.defl_launch_count() - before == 3           # 438 a launch
    pr.check(3, stochastic=True, seed=9)


@pytest.mark.gpu
def test_mixed_types_and_missing_gradients(ctx):
    from paper_2609_21102_b200 import binding
    a, b = Problem([400, 33], F32, BF16, False, 14), Problem([500, 257], BF16, F32, True, 15)
    group = binding.AdamWGroup(a.p + b.p, a.m + b.m, a.v + b.v, [None, None] + b.ms, [None, None] + b.vs)
    before = [x.clone() for x in (a.p[1], a.m[1], a.v[1])]
    ctx.defl_adamw_step(group, [a.g[0], None] + b.g, LR, 4, betas=(B1, B2), eps=EPS, weight_decay=WD)
    assert all(torch.equal(x, y) for x, y in zip(before, (a.p[1], a.m[1], a.v[1])))
    a.check(4, skip=(1,))
    b.check(4)
    none = binding.AdamWGroup([], [], [])
    ctx.defl_adamw_step(none, [], LR, 1)                   # an empty list is a step


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
def test_clipped_step_with_device_scalars(ctx, eight):
    """Norm, factor and step counter stay on the device; a gradient that is not finite leaves everything as it was."""
    pr = Problem([1000, 513, 4097], F32, BF16, eight, 16)
    group = pr.group()
    step = torch.full((1,), 6, dtype=torch.int64, device="cuda")
    lr = torch.full((1,), LR, dtype=F32, device="cuda")
    clip = ctx.defl_grad_norm(pr.g, 2.0, step=step)
    norm, c = optim.grad_norm(pr.g64, 2.0)
    assert int(step) == 7
    # fp64 sums of fp32 sums of eight squares (7 additions, 8 products: at most 8 E of the sum, 4 E of its root), one last rounding
    assert abs(float(clip[0]) - norm) <= 6 * E * norm and abs(float(clip[1]) - c) <= 7 * E * c and c < 0.5
    ctx.defl_adamw_step(group, pr.g, lr, step, betas=(B1, B2), eps=EPS, weight_decay=WD, grad_scale=clip, stochastic=True, seed=3)
    pr.check(7, c=float(clip[1]), stochastic=True, seed=3, lr=float(np.float32(LR)))
    held = [x.clone() for x in pr.p + pr.m + pr.v]
    for bad in (float("nan"), float("inf"), float("-inf")):
        pr.g[1][77] = bad
        ctx.defl_grad_norm(pr.g, 2.0, out=clip, step=step)
        ctx.defl_adamw_step(group, pr.g, lr, step, grad_scale=clip, stochastic=True)
        assert int(step) == 7 and float(clip[1]) == 0.0
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(held, pr.p + pr.m + pr.v))


@pytest.mark.gpu
def test_gradient_not_finite_without_the_gate(ctx):
    """Only its own element with 32-bit moments, its block with 8-bit ones; weights beside it are updated."""
    for eight in (False, True):
        pr = Problem([1024], F32, F32, eight, 17)
        pr.g[0][300] = float("nan")
        ctx.defl_adamw_step(pr.group(), pr.g, LR, 2, betas=(B1, B2), eps=EPS, weight_decay=WD)
        bad = torch.isnan(pr.p[0])
        assert bad.sum() == 1 and bool(bad[300])
        if eight:
            assert torch.isnan(pr.ms[0]).tolist() == [False, True, False, False] and torch.isnan(pr.vs[0]).tolist() == [False, True, False, False]
        else:
            assert torch.isnan(pr.m[0]).sum() == 1 and torch.isnan(pr.v[0]).sum() == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", [[], [0], [1], [7, 8, 9], [8191, 8192, 8193], [100003], list(range(1, 200)), [3] * 1500])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_matches_oracle(ctx, dtype, sizes, offset):
    rng = _gen(18)
    g = []
    for n in sizes:
        t = torch.empty(n + offset, dtype=dtype, device="cuda")[offset:]
        t.copy_(torch.tensor(rng.standard_normal(n)))
        g.append(t)
    norm, c = optim.grad_norm([x.double().cpu().numpy() for x in g], 1.5)
    a = ctx.defl_grad_norm(g, 1.5)
    b = ctx.defl_grad_norm(g, 1.5)
    assert torch.equal(a, b)
    assert abs(float(a[0]) - norm) <= 6 * E * norm and abs(float(a[1]) - c) <= 7 * E * c


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e18, 1e30])
def test_norm_of_extreme_gradients(ctx, size):
    """Squares that fp32 cannot hold: the norm itself can be held."""
    x = torch.tensor(_gen(19).standard_normal(5000) * size, dtype=F32, device="cuda")
    norm, _ = optim.grad_norm([x.double().cpu().numpy()], 0.0)
    got = ctx.defl_grad_norm([x], 0.0)
    # squares that fp32 holds without their last bits (below 2^-126) appear only beside sums above 1e-30
    assert abs(float(got[0]) - norm) <= 7 * E * norm and float(got[1]) == 1.0


@pytest.mark.gpu
def test_captured_steps_and_other_streams(ctx):
    """Norm and step in a graph: replays advance the counter and give what eager steps give; two graphs of one context may run
    at the same time on two streams (each has its own scratch)."""
    def eager(pr, n):
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        group = pr.group()
        for _ in range(n):
            clip = ctx.defl_grad_norm(pr.g, 1.0, step=step)
            ctx.defl_adamw_step(group, pr.g, LR, step, grad_scale=clip, stochastic=True, seed=4)
        torch.cuda.synchronize()
    want = [Problem([70000, 300], F32, BF16, True, s, fresh=True) for s in (20, 21)]
    have = [Problem([70000, 300], F32, BF16, True, s, fresh=True) for s in (20, 21)]
    for pr in want:
        eager(pr, 5)
    graphs = []
    for pr in have:
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        group, clip = pr.group(), torch.zeros(2, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.defl_grad_norm(pr.g, 1.0, out=clip, step=step)
            ctx.defl_adamw_step(group, pr.g, LR, step, grad_scale=clip, stochastic=True, seed=4)
        graphs.append((g, torch.cuda.Stream(), group, clip, step))
    torch.cuda.synchronize()
    for _ in range(5):
        for g, st, *_ in graphs:
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for a, b, (*_, step) in zip(want, have, graphs):
        assert int(step) == 5
        for x, y in zip(a.p + a.m + a.v + a.ms + a.vs, b.p + b.m + b.v + b.ms + b.vs):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.gpu
def test_muon_takes_the_factor(ctx):
    """Mom <- mu Mom + c Grad: the same as a call with the scaled gradient; c = 0 drops a gradient that is not finite."""
    from paper_2609_21102_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(22)
    r = lambda: torch.randn(2, 64, 96, generator=g, device="cuda")  # noqa: E731
    W, M, G = r(), r(), r()
    clip = ctx.defl_grad_norm([G], 0.5)
    sched = [list(binding.MUON_QUINTIC)] * 5
    a, b = (W.clone(), M.clone()), (W.clone(), M.clone())
    ctx.defl_muon_step_batched(*a, G, LR, 0.95, 4, 4, 1, sched, nesterov=True, grad_scale=clip)
    ctx.defl_muon_step_batched(*b, G * clip[1], LR, 0.95, 4, 4, 1, sched, nesterov=True)
    assert torch.equal(a[1], b[1]) and torch.equal(a[0], b[0])
    G[0, 3, 3] = float("nan")
    ctx.defl_grad_norm([G], 0.5, out=clip)
    m = a[1].clone()
    ctx.defl_muon_step_batched(*a, G, LR, 0.95, 4, 4, 1, sched, grad_scale=clip)
    assert torch.equal(a[1], torch.tensor(0.95, dtype=F32).item() * m)


@pytest.mark.gpu
def test_a_parameter_that_has_moved(ctx):
    """A group made before a parameter was given other memory is refused, and what it points to is still there."""
    from paper_2609_21102_b200 import binding
    p = torch.nn.Parameter(torch.ones(1000, device="cuda"))
    group = binding.AdamWGroup([p], [torch.zeros(1000, device="cuda")], [torch.zeros(1000, device="cuda")])
    g = torch.ones(1000, device="cuda")
    ctx.defl_adamw_step(group, [g], LR, 1)
    old = group._memory[0][0]
    assert old.data_ptr() == p.data_ptr() and torch.all(p != 1)
    p.data = p.data.clone()
    kept = p.detach().clone()
    with pytest.raises(ValueError):
        ctx.defl_adamw_step(group, [g], LR, 2)
    assert torch.equal(p.detach(), kept) and torch.equal(old, kept)


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["first moment", "second moment", "first moment's scales", "second moment's scales", "copy"])
def test_a_moment_that_has_moved(ctx, which):
    """What belongs to a parameter and was given other memory since its group was made is refused, by its name, and nothing is updated."""
    from paper_2609_21102_b200 import binding
    e8 = torch.float8_e4m3fn
    f = lambda n, dtype=F32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    parts = {"parameter": f(700), "first moment": f(700, e8), "second moment": f(700, e8), "first moment's scales": f(3),
             "second moment's scales": f(3), "copy": f(700, BF16)}
    group = binding.AdamWGroup([f(9)] + [parts["parameter"]], [f(9)] + [parts["first moment"]], [f(9)] + [parts["second moment"]],
                               [None, parts["first moment's scales"]], [None, parts["second moment's scales"]], copies=[None, parts["copy"]])
    grads = [torch.ones(9, device="cuda"), torch.ones(700, device="cuda")]
    ctx.defl_adamw_step(group, grads, LR, 1)
    moved = parts[which]
    moved.data = moved.data.clone()
    held = [t.clone() for t in list(group.params) + list(parts.values())]
    with pytest.raises(ValueError, match="%s 1 has other memory" % which):
        ctx.defl_adamw_step(group, grads, LR, 2)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, list(group.params) + list(parts.values())))
    for name, place in (("params", 0), ("exp_avg", 1)):      # another tensor in its place would not be seen either
        with pytest.raises(TypeError):
            getattr(group, name)[place] = moved
        with pytest.raises(AttributeError):
            setattr(group, name, [moved])


@pytest.mark.gpu
def test_moments_that_share_a_buffer(ctx):
    """Views of one buffer: another place in it, and a buffer that was given other memory itself, are refused; a view of all of a tensor's own
    memory is that memory. What moved before the first step is seen by it."""
    from paper_2609_21102_b200 import binding
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    flat, p, g = f(1000), f(100), torch.ones(100, device="cuda")
    m, v = flat[:100], flat[100:200]
    group = binding.AdamWGroup([p], [m], [v])
    m.data = flat[200:300]
    with pytest.raises(ValueError, match="first moment 0"):
        ctx.defl_adamw_step(group, [g], LR, 1)               # (the first one)
    m.data = flat[:100]
    ctx.defl_adamw_step(group, [g], LR, 1)
    assert torch.all(m > 0)
    v.data = flat[300:400]
    held = p.clone()
    with pytest.raises(ValueError, match="second moment 0"):
        ctx.defl_adamw_step(group, [g], LR, 2)
    v.data = flat[100:200]
    ctx.defl_adamw_step(group, [g], LR, 2)
    assert not torch.equal(p, held)
    held.copy_(p)
    flat.untyped_storage().resize_(4 * 2000)
    with pytest.raises(ValueError, match="moment 0"):
        ctx.defl_adamw_step(group, [g], LR, 3)
    assert torch.equal(p, held)
    own = f(100)
    group = binding.AdamWGroup([p], [own], [f(100)])
    own.data = own.data[:50]
    ctx.defl_adamw_step(group, [g], LR, 1)
    assert torch.all(own > 0)


@pytest.mark.gpu
def test_context_of_a_device_without_a_number():
    """torch.device("cuda") is the first device, as the tensors that were made on it say; they are not refused."""
    from paper_2609_21102_b200 import binding
    c = binding.Context(torch.device("cuda"))
    f = lambda: torch.ones(300, device="cuda")  # noqa: E731
    p, g = f(), f()
    clip = c.defl_grad_norm([g], 1.0)
    c.defl_adamw_step(binding.AdamWGroup([p], [f()], [f()]), [g], torch.full((1,), LR, device="cuda"), 1, grad_scale=clip)
    W, G = torch.randn(1, 32, 48, device="cuda"), torch.randn(1, 32, 48, device="cuda")
    c.defl_muon_step_batched(W, torch.zeros_like(W), G, LR, 0.9, 2, 2, 1, [list(binding.MUON_QUINTIC)] * 2, grad_scale=clip)
    assert torch.all(p < 1) and torch.isfinite(W).all()
    c.close()


@pytest.mark.gpu
def test_smallest_eps(ctx):
    """An eps below fp32's normal numbers is zero; where both moments are, the quotient is then NaN, as 0 / 0 is."""
    from paper_2609_21102_b200 import binding
    for eps, dead in ((0.0, True), (1e-40, True), (2e-38, False)):
        p, m, v = (torch.full((512,), x, device="cuda") for x in (1.0, 0.0, 0.0))
        g = torch.zeros(512, device="cuda")
        g[::2] = 0.5
        ctx.defl_adamw_step(binding.AdamWGroup([p], [m], [v]), [g], LR, 1, eps=eps, weight_decay=0.0)
        # the first step is lr in the gradient's direction: a reciprocal, two products and a difference
        assert float((p[::2].double() - (1 - LR)).abs().max()) <= 8 * 2.0 ** -24
        assert torch.isnan(p[1::2]).all() if dead else torch.all(p[1::2] == 1)


@pytest.mark.gpu
def test_refusals(ctx):
    from paper_2609_21102_b200 import binding
    f = lambda n, dtype=F32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    group = binding.AdamWGroup([f(10)], [f(10)], [f(10)])
    with pytest.raises(ValueError):
        ctx.defl_adamw_step(group, [], LR, 1)
    with pytest.raises(ValueError):
        ctx.defl_adamw_step(group, [f(11)], LR, 1)
    with pytest.raises(ValueError):
        ctx.defl_adamw_step(group, [torch.zeros(10)], LR, 1)
    with pytest.raises(ValueError):
        ctx.defl_adamw_step(group, [f(20)[::2]], LR, 1)
    with pytest.raises(TypeError):
        ctx.defl_adamw_step(group, [f(10, torch.float16)], LR, 1)
    for kw in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(eps=float("nan")),
               dict(weight_decay=float("inf"))):
        with pytest.raises(binding.DeflError) as e:
            ctx.defl_adamw_step(group, [f(10)], LR, **{"step": 1, **kw})
        assert e.value.code == -1
    for lr in (float("nan"), float("inf")):
        with pytest.raises(binding.DeflError):
            ctx.defl_adamw_step(group, [f(10)], lr, 1)
    for bad in (f(1), f(2, torch.int64)):
        with pytest.raises(ValueError):
            ctx.defl_adamw_step(group, [f(10)], LR, bad)
        with pytest.raises(ValueError):
            ctx.defl_grad_norm([f(10)], 1.0, step=bad)
    with pytest.raises(ValueError):
        ctx.defl_grad_norm([f(10)], 1.0, out=f(3))
    with pytest.raises(binding.DeflError):
        ctx.defl_grad_norm([f(10)], float("nan"))
    x = f(100)
    with pytest.raises(ValueError):                        # one tensor twice, or two that share elements
        binding.AdamWGroup([x, x], [f(100), f(100)], [f(100), f(100)])
    with pytest.raises(ValueError):
        binding.AdamWGroup([x[:60], x[50:]], [f(60), f(50)], [f(60), f(50)])
    e8 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        binding.AdamWGroup([f(300)], [f(300, e8)], [f(300, e8)])
    with pytest.raises(ValueError):
        binding.AdamWGroup([f(300)], [f(300, e8)], [f(300, e8)], [f(1)], [f(2)])
    with pytest.raises(TypeError):
        binding.AdamWGroup([f(300)], [f(300, e8)], [f(300)], [f(2)], [f(2)])
    with pytest.raises(TypeError):
        binding.AdamWGroup([f(300, torch.float16)], [f(300)], [f(300)])


def test_refusals_without_a_device():
    from paper_2609_21102_b200 import binding, build
    import ctypes
    build.build()
    with pytest.raises(ValueError):
        binding.AdamWGroup([torch.zeros(3)], [torch.zeros(3)], [torch.zeros(3)])
    with pytest.raises(ValueError):
        binding.AdamWGroup([torch.zeros(3)], [], [])
    L = binding.lib()
    assert L.defl_adamw_step(None, None, 0, None) == -1
    assert L.defl_grad_norm(None, None, 0, ctypes.c_float(1.0), None, None, None) == -1
    assert L.defl_grad_norm_work_bytes(-1) == 0
    one = L.defl_grad_norm_work_bytes(1)
    assert one == L.defl_grad_norm_work_bytes(1300) == L.defl_grad_norm_work_bytes(1301) // 2
    # the table is laid out as the C structure is: 7 pointers, a 64-bit count, three ints and padding
    assert binding._ADAMW_TENSOR.itemsize == 80
    # a context that is closed refuses (no device: none can be made), and so does a list that is none
    with pytest.raises(TypeError):
        binding._native().grad_norm(0, 0, 5, 1.0, None, None)
    with pytest.raises(ValueError):
        binding._native().grad_norm(0, 0, [torch.zeros(3)], 1.0, None, None)
    with pytest.raises(TypeError):
        binding._native().grad_norm(0, 0, [3], 1.0, None, None)
    with pytest.raises(ValueError):
        binding._native().adamw_step(0, 0, 0, [torch.zeros(3)], [], 1e-3, 1, 0.9, 0.999, 1e-8, 0.0, None, False, 0)


def test_a_group_is_not_copied():
    """A copy would hold the addresses of the original's table and tensors, and outlive them."""
    import copy
    import pickle
    from paper_2609_21102_b200 import binding
    group = binding.AdamWGroup([], [], [])
    for f in (copy.copy, copy.deepcopy, pickle.dumps):
        with pytest.raises(TypeError):
            f(group)
