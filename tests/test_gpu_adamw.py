"""AdamW over lists of tensors, against the definition in 64 bits.

Tolerances.  m and v are two products and a sum of fp32 numbers: 4 * 2^-24 of their magnitudes' sum (v: one product more, and with
8-bit states the squared root, two more).  The update is a quotient of those with a root, a product and a sum, the quotient by the hardware's
division (2 units): 24 * 2^-24 of its magnitude, plus what m's and v's errors move it (half of v's), and the parameter itself two
roundings.  A code of 8 bits is off by less than one step of its scale (it is rounded up or down by a threshold).
"""
import math

import pytest

U = 2.0 ** -24
BLOCK = 256


class Case:
    def __init__(self, sizes, q8, grad="fp32", copies=False, decay=0.01, decayed=None, offset=0, done=0, seed=0, clip=None, lr_scale=None, **hyper):
        import torch
        from paper_2408_11500_b200 import binding as B
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.sizes, self.q8, self.decay, self.done = sizes, q8, decay, done
        self.decayed = decayed or [True] * len(sizes)

        def rand(n, std, t=torch.float32):
            return (torch.randn(n + 8, generator=g, device="cuda") * std).to(t)[offset:offset + n]
        gt = {"fp32": lambda i: torch.float32, "bf16": lambda i: torch.bfloat16, "mixed": lambda i: (torch.float32, torch.bfloat16)[i % 2]}[grad]
        self.p, self.g = [rand(n, 0.1) for n in sizes], [rand(n, 1e-2, gt(i)) for i, n in enumerate(sizes)]
        self.m_scale = self.v_scale = None
        if q8:
            self.m = [torch.randint(-127, 128, (n + 8,), generator=g, device="cuda").to(torch.int8)[offset:offset + n] for n in sizes]
            self.v = [torch.randint(0, 256, (n + 8,), generator=g, device="cuda").to(torch.uint8)[offset:offset + n] for n in sizes]
            self.m_scale, self.v_scale = ([torch.rand(-(-n // BLOCK), generator=g, device="cuda") * s + s for n in sizes] for s in (1e-4, 1e-4))
        else:
            self.m, self.v = [rand(n, 1e-2) for n in sizes], [rand(n, 1e-2).square() for n in sizes]
            if offset:
                self.v = [torch.cat([t.new_zeros(offset), t])[offset:] for t in self.v]
        self.copies = [torch.full((n + 8,), float("nan"), device="cuda", dtype=torch.bfloat16)[offset:offset + n] if i % 3 != 2 else None
                       for i, n in enumerate(sizes)] if copies else None
        self.step = torch.tensor([done, 0], dtype=torch.int64, device="cuda")
        self.norm, self.factor = None, 1.0
        max_norm = math.inf
        if clip is not None:
            norm = math.sqrt(sum(float(t.double().square().sum()) for t in self.g))
            self.norm, max_norm = torch.tensor([norm], device="cuda"), clip * norm
            self.factor = min(1.0, max_norm / float(self.norm))
        self.hyper = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)
        self.hyper.update(hyper)
        self.lr_scale = torch.tensor([lr_scale], device="cuda") if lr_scale is not None else None
        self.d = B.make_adamw_desc(self.p, self.g, self.m, self.v, self.m_scale, self.v_scale, copies=self.copies, weight_decay=decay, decayed=self.decayed,
                                   max_norm=max_norm, lr_scale=self.lr_scale, **self.hyper)

    def values(self):
        """m and sqrt(v) as 64-bit numbers."""
        import torch
        if not self.q8:
            return [t.double() for t in self.m], [t.double().sqrt() for t in self.v]
        spread = lambda s, n: torch.repeat_interleave(s.double(), BLOCK)[:n]   # noqa: E731
        return ([t.double() * spread(s, t.numel()) for t, s in zip(self.m, self.m_scale)], [t.double() * spread(s, t.numel()) for t, s in zip(self.v, self.v_scale)])

    def go(self, stream=None):
        from paper_2408_11500_b200 import binding as B
        B.slicegcn_adamw_step(self.d, self.step, self.norm, stream)

    def check_step(self):
        """Runs one step and compares."""
        import torch
        h, t = self.hyper, int(self.step[0]) + 1
        m0, r0 = self.values()
        p0 = [t.double().clone() for t in self.p]
        self.go()
        assert self.step.tolist() == [t, 0]
        m1, r1 = self.values()
        rate = h["lr"] * (float(self.lr_scale) if self.lr_scale is not None else 1.0)
        for i, g in enumerate(self.g):
            g = g.double() * self.factor
            m = h["beta1"] * m0[i] + (1 - h["beta1"]) * g
            v = h["beta2"] * r0[i] ** 2 + (1 - h["beta2"]) * g ** 2
            root, denom = v.sqrt(), (v / (1 - h["beta2"] ** t)).sqrt() + h["eps"]
            move = rate * m / (1 - h["beta1"] ** t) / denom
            em = 6 * U * (h["beta1"] * m0[i].abs() + (1 - h["beta1"]) * g.abs())
            keep = 1 - rate * (self.decay if self.decayed[i] else 0.0)
            want = p0[i] * keep - move
            bound = 4 * U * p0[i].abs() + 2 * U * want.abs() + (40 * U) * move.abs() + rate / (1 - h["beta1"] ** t) * em / denom + 1e-38
            off = (self.p[i].double() - want).abs()
            assert bool((off <= bound).all()), (i, float((off / bound).max()))
            if self.copies and self.copies[i] is not None:
                assert torch.equal(self.copies[i], self.p[i].to(torch.bfloat16))
            if self.q8:
                n = g.numel()
                for name, got, exact, scale, codes in (("m", m1[i], m, self.m_scale[i], 127), ("v", r1[i], root, self.v_scale[i], 255)):
                    nb = -(-n // BLOCK)
                    top = torch.nn.functional.pad(exact.abs(), (0, nb * BLOCK - n)).view(nb, BLOCK).amax(1)
                    # (the state's cancellation: beta1 m + (1 - beta1) g of opposite signs)
                    assert bool(((scale.double() - top / codes).abs() <= 8 * U * top / codes + 2e-2 / codes * U + 1.2e-38).all()), name
                    step = torch.repeat_interleave(scale.double(), BLOCK)[:n]
                    assert bool(((got - exact).abs() <= step * (1 + 1e-5) + (em if name == "m" else 0)).all()), name
                assert bool((self.v[i][root > 1e-37] > 0).all())
            else:
                assert bool(((m1[i] - m).abs() <= em + 1e-44).all()) and bool(((r1[i] - root).abs() <= 8 * U * root + 1e-22).all())


SIZES = [[1], [5, 0, 3], [255, 256, 257, 4096, 4097], [128 * 32, 32, 256 * 40, 40, 7], [200_003, 64, 65_536, 13, 100], [33] * 40, [130] * 300, [3_000_001, 8]]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=[str(k) for k in range(len(SIZES))])
@pytest.mark.parametrize("grad", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("q8", [False, True], ids=["f32", "q8"])
def test_steps(sizes, grad, q8):
    for done, offset, kw in ((0, 0, {}), (999, 1, dict(copies=True, clip=0.3)), (7, 4, dict(copies=True, clip=2.0, lr_scale=0.25, decayed=[i % 2 == 0 for i in range(len(sizes))])),
                             (100_000, 0, dict(beta1=0.0, beta2=0.5, eps=1e-3, decay=0.0))):
        c = Case(sizes, q8, grad, offset=offset, done=done, seed=done, **kw)
        c.check_step()
        c.check_step()


@pytest.mark.gpu
@pytest.mark.parametrize("q8", [False, True], ids=["f32", "q8"])
def test_neighbours_keep_their_values(q8):
    """Elements before and behind a tensor, in every array, stay as they are."""
    import torch
    from paper_2408_11500_b200 import binding as B
    n, lead = 777, 3
    types = [torch.float32, torch.float32] + ([torch.int8, torch.uint8] if q8 else [torch.float32] * 2) + [torch.bfloat16]
    bufs = [torch.full((n + 20,), 9, dtype=t, device="cuda") for t in types]
    scales = [torch.full((-(-n // BLOCK) + 4,), 9.0, device="cuda") for _ in range(2)] if q8 else [None, None]
    views, blocks = [t[lead:lead + n] for t in bufs], [[t[2:2 + -(-n // BLOCK)]] if q8 else None for t in scales]
    d = B.make_adamw_desc([views[0]], [views[1]], [views[2]], [views[3]], *blocks, copies=[views[4]])
    B.slicegcn_adamw_step(d, torch.zeros(2, dtype=torch.int64, device="cuda"))
    for t in bufs:
        assert bool((t[:lead] == 9).all()) and bool((t[lead + n:] == 9).all())
    for t in scales if q8 else []:
        assert bool((t[:2] == 9).all()) and bool((t[-2:] == 9).all())


@pytest.mark.gpu
def test_slow_averages_move():
    """A root that falls by less than a step of its code each time falls as the 32-bit one does, on average."""
    import torch
    n = 1 << 16
    c = Case([n], True, done=10_000, beta2=0.999, lr=0.0)
    c.m[0].zero_()
    c.v[0].random_(50, 256)
    c.v[0][::BLOCK] = 255
    c.v_scale[0].fill_(1e-3)
    c.g[0].zero_()
    c.g[0][::BLOCK] = 0.255                      # the blocks' largest roots stay, and with them the scales
    start = c.values()[1][0]
    for _ in range(100):
        c.go()
    end = c.values()[1][0]
    rest = torch.arange(n, device="cuda") % BLOCK != 0
    fall = float((end[rest].mean() / start[rest].mean()))
    # 65,000 independent thresholds: the mean's deviation is 100 steps' worth of half a code, sqrt(100) / 2 / 150 / 255, below 2e-4
    assert abs(fall - 0.999 ** 50) < 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("q8", [False, True], ids=["f32", "q8"])
def test_special_gradients(q8):
    """No gradient at all, infinities and NaN in one block, and a norm that is not finite."""
    import torch
    c = Case([600, 40], q8, done=3, decay=0.1)
    for t in c.g + c.m + c.v:
        t.zero_()
    before = [t.clone() for t in c.p]
    c.go()
    for a, b in zip(before, c.p):
        assert bool(((b - a * (1 - 1e-3)).abs() <= 2 * U * a.abs()).all())
    c.g[0][300], c.g[0][301] = float("inf"), float("nan")
    before = c.p[0].clone()
    c.go()
    assert bool(torch.isfinite(c.p[0][:256]).all()) and bool(torch.isfinite(c.p[0][512:]).all()) and bool(torch.isfinite(c.p[1]).all())
    assert not bool(torch.isfinite(c.values()[0][0][300:302]).any()) and bool(torch.isfinite(c.values()[0][0][:256]).all())
    assert bool(torch.isnan(c.p[0][301])) and bool(torch.isfinite(c.p[0][302:512]).all())
    if q8:
        assert not bool(torch.isfinite(c.values()[0][0][256:512]).any()) and not bool(torch.isfinite(c.values()[1][0][256:512]).any())
    for bad in (float("inf"), float("nan")):
        a, b = Case([300], q8, seed=5), Case([300], q8, seed=5, clip=0.5)
        b.norm.fill_(bad)
        a.go(), b.go()
        assert torch.equal(a.p[0], b.p[0])


@pytest.mark.gpu
def test_tiny_factor_keeps_digits():
    """Gradients of 1e30 against a limit that takes them to 1e-9: the factor itself is below the normal numbers."""
    import torch
    from paper_2408_11500_b200 import binding as B
    g = torch.full((300,), 3e38, device="cuda")
    p, m, v = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    norm = torch.tensor([3.2e38], device="cuda")
    d = B.make_adamw_desc([p], [g], [m], [v], max_norm=1e-3)
    B.slicegcn_adamw_step(d, torch.zeros(2, dtype=torch.int64, device="cuda"), norm)
    want = 0.1 * float(g[0].double()) * (1e-3 / float(norm.double()))
    assert bool(((m.double() - want).abs() <= 4 * U * want).all())


@pytest.mark.gpu
@pytest.mark.parametrize("q8", [False, True], ids=["f32", "q8"])
def test_captured_and_on_a_side_stream(q8):
    """A captured step that is replayed advances the count and gives what eager steps give."""
    import torch
    a, b = (Case([5000, 77], q8, "mixed", seed=3, clip=0.5, copies=True) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.go(torch.cuda.current_stream().cuda_stream)
    for _ in range(4):
        a.go()
        graph.replay()
    torch.cuda.synchronize()
    assert a.step.tolist() == b.step.tolist() == [4, 0]
    for x, y in zip(a.p + a.m + a.v, b.p + b.m + b.v):
        assert torch.equal(x, y)


@pytest.mark.gpu
def test_empty_list_counts_its_step():
    import torch
    from paper_2408_11500_b200 import binding as B
    step = torch.tensor([4, 0], dtype=torch.int64, device="cuda")
    B.slicegcn_adamw_step(B.make_adamw_desc([], [], [], []), step)
    assert step.tolist() == [5, 0]
