"""Gradient norm, AdamW step and moments read out, against the float64 checker; codes, scales and 32-bit moments bit for bit.

Tolerances.  Moments are formed by single roundings in float32, which numpy makes alike.  The parameter's step from them: root,
product, sum, quotient, product and difference, each off by at most 2^-24 of its result (the two factors from 1 - beta^t as well), so 10 x 2^-24 of
the step and 2 x 2^-24 of the parameter; then half a unit of the storage type.
"""
import numpy as np
import pytest
import torch

from oracle import training_oracle as orc

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24
SIZES = [1, 2, 7, 8, 9, 31, 255, 256, 257, 511, 2047, 2048, 2049, 4096, 5003, 10000]


@pytest.fixture(scope="module")
def gh():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gpu_helpers
    return gpu_helpers


class Buffers:
    """Tensors as pieces of one buffer of each kind, `gap` elements between them that have to stay as they are."""

    def __init__(self, sizes, gap):
        self.sizes, self.gap = sizes, gap
        self.starts = np.concatenate([[0], np.cumsum(np.asarray(sizes) + gap)[:-1]]).astype(int) + gap
        self.total = int(sum(sizes) + gap * (len(sizes) + 1))

    def put(self, arrays, dtype):
        flat = torch.full((self.total,), 77, dtype=torch.float32).to(dtype)
        for a, s, x in zip(self.starts, self.sizes, arrays):
            flat[a:a + s] = torch.from_numpy(np.ascontiguousarray(x)).to(dtype)
        return flat.to("cuda")

    def pieces(self, flat):
        return [flat[a:a + s] for a, s in zip(self.starts, self.sizes)]

    def get(self, flat):
        host = flat.cpu()
        keep = torch.ones(self.total, dtype=torch.bool)
        out = []
        for a, s in zip(self.starts, self.sizes):
            keep[a:a + s] = False
            out.append(host[a:a + s])
        assert (host[keep].float() == 77).all(), "written outside the tensors"
        return out


def wide(x):
    return x.float().numpy().astype(np.float64)


class Model:
    """A table of tensors with its host copies."""

    def __init__(self, seed, sizes, param, grad, master, bits, gap=1, decay=None, spread=3):
        import paper_2602_14338_amd as aero
        rng = np.random.default_rng(seed)
        self.kind, self.bits = (param, grad, master), bits
        self.b = Buffers(sizes, gap)
        self.blocks = Buffers([(s + 255) // 256 for s in sizes], gap)
        new = lambda sigma: [(rng.normal(0, sigma, s) * 10.0 ** rng.uniform(-spread, 0, s)).astype(np.float32) for s in sizes]   # noqa: E731
        w, g = new(1.0), new(1e-2)
        self.m = new(1e-3)
        self.v = [np.abs(x) ** 2 for x in new(1e-3)]
        flat = dict(param=self.b.put(w, TORCH[param]), grad=self.b.put(g, TORCH[grad]))
        self.g = [wide(x).astype(np.float32) for x in self.b.get(flat["grad"])]
        if master:
            flat["master"] = self.b.put(w, torch.float32)
            self.p = w
        else:
            self.p = [wide(x).astype(np.float32) for x in self.b.get(flat["param"])]
        if bits == 32:
            flat["exp_avg"], flat["exp_avg_sq"] = self.b.put(self.m, torch.float32), self.b.put(self.v, torch.float32)
        else:
            half = lambda x: np.full(len(x), 0.5)   # noqa: E731
            for name, top, first in (("exp_avg", orc.TOP1, True), ("exp_avg_sq", orc.TOP2, False)):
                values = self.m if first else self.v
                scales = [orc.scale_of(x, top) for x in values]
                codes = [orc.codes_of(x, s, half(x), first) for x, s in zip(values, scales)]
                flat[name] = self.b.put([c.astype(np.int8 if first else np.uint8) for c in codes], torch.int8 if first else torch.uint8)
                flat[name + "_scale"] = self.blocks.put(scales, torch.float32)
                values[:] = [orc.values_of(c, s, first) for c, s in zip(codes, scales)]
        self.flat = flat
        self.decay = decay if decay is not None else [1.0] * len(sizes)
        cut = lambda k: (self.blocks if k.endswith("scale") else self.b).pieces(flat[k])   # noqa: E731
        self.entries = [dict(zip(flat, x), decay=d) for x, d in zip(zip(*(cut(k) for k in flat)), self.decay)]
        self.table = aero.TensorTable(self.entries)

    def check(self, steps_before, how, factor=1.0, first_tensor=0, rate=1.0):
        """The device's buffers after one more step than the host's, which then takes it too."""
        param, grad, master = self.kind
        get = {k: (self.blocks if k.endswith("scale") else self.b).get(x) for k, x in self.flat.items()}
        lr = how["lr"] * rate
        t = steps_before + 1
        for k in range(len(self.b.sizes)):
            n = self.b.sizes[k]
            m, v = orc.moments32(self.m[k], self.v[k], self.g[k], factor, how["beta1"], how["beta2"])
            m64, v64 = m.astype(np.float64), v.astype(np.float64)
            step = (m64 / (1 - how["beta1"] ** t)) / (np.sqrt(v64 / (1 - how["beta2"] ** t)) + float(np.float32(how["eps"])))
            want = self.p[k].astype(np.float64) * (1 - lr * how["weight_decay"] * self.decay[k]) - lr * step
            tol = 2 * U * np.abs(self.p[k]) + 10 * U * lr * np.abs(step) + U * np.abs(want) + 1e-45
            if master:
                got = get["master"][k].numpy()
                assert (np.abs(got - want) <= tol).all()
                assert torch.equal(get["param"][k], get["master"][k].to(TORCH[param]))
                self.p[k] = got
            else:
                got = wide(get["param"][k])
                random = how["stochastic"] and param == "bf16"
                ulp = (2 if random else 1) * HALF_ULP[param]
                assert (np.abs(got - want) <= tol + ulp * (np.abs(want) + tol) + 1e-40).all()
                if random and n >= 2000:   # neither up nor down on the whole
                    off = (got - want) / np.abs(want)
                    assert abs(off.mean()) <= 5 * HALF_ULP["bf16"] / np.sqrt(n)
                self.p[k] = got.astype(np.float32)
            if self.bits == 32:
                assert np.array_equal(get["exp_avg"][k].numpy(), m) and np.array_equal(get["exp_avg_sq"][k].numpy(), v)
                self.m[k], self.v[k] = m, v
                continue
            h = orc.random_bits(how["seed"], steps_before, first_tensor + k, n)
            u1, u2 = (((h & 0xffff) + 0.5) / 65536, ((h >> 16) + 0.5) / 65536) if how["stochastic"] else (np.full(n, 0.5),) * 2
            for name, x, top, first, u in (("exp_avg", m, orc.TOP1, True, u1), ("exp_avg_sq", v, orc.TOP2, False, u2)):
                scale = orc.scale_of(x, top)
                codes = orc.codes_of(x, scale, u, first)
                assert np.array_equal(get[name + "_scale"][k].numpy(), scale), (name, k)
                assert np.array_equal(get[name][k].numpy().astype(int), codes), (name, k)
                (self.m if first else self.v)[k] = orc.values_of(codes, scale, first)


def how_of(**more):
    return dict(dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, seed=0x700000123, stochastic=False), **more)


def words(step=0, factor=None, rate=None):
    one = lambda x: None if x is None else torch.full((1,), x, device="cuda")   # noqa: E731
    return torch.full((1,), step, dtype=torch.int32, device="cuda"), one(factor), one(rate)


KINDS = [("f32", 0), ("bf16", 0), ("bf16", 1), ("f16", 1)]


@pytest.mark.parametrize("param,master", KINDS)
@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("stochastic", [False, True])
def test_steps(gh, param, master, grad, bits, stochastic):
    import paper_2602_14338_amd as aero
    model = Model([bits, master, len(grad)], SIZES, param, grad, master, bits, gap=1, decay=[k % 3 * 0.5 for k in range(len(SIZES))])
    how = how_of(stochastic=stochastic)
    step, factor, rate = words(0, 0.625, 0.5)
    for t in range(3):
        aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step, factor, rate)
        torch.cuda.synchronize()
        assert step.item() == t + 1
        model.check(t, how, factor=0.625, rate=0.5)
    assert torch.equal(model.flat["grad"], model.b.put(model.g, TORCH[grad]))


@pytest.mark.parametrize("gap", [0, 3, 8])
@pytest.mark.parametrize("bits", [32, 8])
def test_alignments(gh, gap, bits):
    import paper_2602_14338_amd as aero
    model = Model([gap, bits], [2048, 5, 256, 3001, 4097], "bf16", "bf16", 1, bits, gap=gap)
    how = how_of(weight_decay=0.0)
    step, *_ = words(99)
    aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step)
    torch.cuda.synchronize()
    model.check(99, how)


@pytest.mark.parametrize("steps", [0, 1, 999, 10 ** 6, 2 ** 31 - 2])
def test_counts_of_steps(gh, steps):
    import paper_2602_14338_amd as aero
    model = Model(7, [300], "f32", "f32", 0, 8)
    how = how_of(beta1=0.95, beta2=0.9999, stochastic=True)
    step, *_ = words(steps)
    aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step)
    torch.cuda.synchronize()
    assert step.item() == steps + 1
    model.check(steps, how)


def test_no_momentum_and_no_rate(gh):
    import paper_2602_14338_amd as aero
    for how in (how_of(beta1=0.0, beta2=0.0), how_of(lr=0.0)):
        model = Model(8, [700], "bf16", "f32", 0, 8)
        step, *_ = words()
        aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step)
        torch.cuda.synchronize()
        model.check(0, how)


@pytest.mark.parametrize("param,master,bits", [("f32", 0, 32), ("f32", 0, 8), ("bf16", 1, 32), ("f16", 1, 8)])
@pytest.mark.parametrize("rate,weight_decay,decay,n", [(1e-6, 0.01, 1.0, 20000), (1e-6, 0.1, 1.0, 20000), (2e-6, 0.1, 1.0, 20000), (1e-6, 0.1, 0.5, 20000),
                                                       (1e-6, 0.01, 1.0, 4500000)])
def test_decay_at_small_rates(gh, param, master, bits, rate, weight_decay, decay, n):
    """Weights of 0.55 to 0.95 over 200 steps of about `rate`, with decay and without, whose moments are the same: their means differ by what decays,
    f = rate weight_decay decay of the weight a step, though that is less than a unit of the weight (2^-24).  Each of the steps on either side rounds by up to half
    a unit, evenly, as the gradients are others every time: 5 standard deviations of the mean, sqrt(2 steps / 12 n) units.  (But for the first, which moves every weight by
    the rate itself, whatever its gradient: 1e-6 are 16.78 units, 17 with or without a decay of 0.13 units, and so on every weight: half a unit on either side.)  The weights move by
    4 x 200 rates at most (|m| / sqrt v <= 4 with these moments), their decay by that share of itself; f is rounded by 2^-24 of itself, as are the products."""
    from paper_2602_14338_amd import optim
    steps = 200 if n < 100000 else 60
    gen = torch.Generator(device="cuda").manual_seed(9)
    start = (0.55 + 0.4 * torch.rand(n, generator=gen, device="cuda")).to(TORCH[param])
    g = torch.zeros(n, device="cuda")
    factor = torch.full((1,), 2.0 ** -10, device="cuda")
    opts = [optim.AdamW([start.clone()], [g], lr=rate * 2.0 ** 10, betas=(0.9, 0.99), weight_decay=x, decay=[decay], bits=bits) for x in (weight_decay, 0.0)]
    for _ in range(steps):
        g.normal_(generator=gen)
        for o in opts:
            o.step(lr_factor=factor)
    ends = [(o.table.entries[0]["master" if master else "param"]).double() for o in opts]
    f = rate * weight_decay * decay
    moved = float((ends[1] - start.double()).abs().max())
    assert moved <= 4 * steps * rate
    want = (1 - (1 - f) ** steps) * start.double().mean().item()
    got = (ends[1] - ends[0]).mean().item()
    tol = U + 5 * np.sqrt(steps / 6 / n) * U + want * (4 * steps * rate / 0.55 + 4 * U)
    assert abs(got - want) <= tol, (got, want, tol)
    assert tol < 0.15 * want


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_zero_and_tiny_ones(gh, bits):
    """All zeros, blocks of zeros beside others, numbers whose squares are below the smallest scale: no NaN, and what the checker says."""
    import paper_2602_14338_amd as aero
    model = Model(9, [600, 256, 1000], "f32", "f32", 0, bits)
    model.g = [np.zeros(600, np.float32), np.full(256, 1e-22, np.float32), np.where(np.arange(1000) < 500, 0, 1e-13).astype(np.float32)]
    model.flat["grad"].copy_(model.b.put(model.g, torch.float32))
    for k in ("exp_avg", "exp_avg_sq"):
        for piece in model.b.pieces(model.flat[k]):
            piece.zero_()
    model.m = [np.zeros(s, np.float32) for s in model.b.sizes]
    model.v = [np.zeros(s, np.float32) for s in model.b.sizes]
    step, *_ = words()
    for t in range(2):
        aero.aero_adamw_step(model.table, aero.AdamWParams(**how_of()), step)
        torch.cuda.synchronize()
        model.check(t, how_of())


@pytest.mark.parametrize("param,master", KINDS)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-19, 1e-12])
def test_smallest_eps(gh, param, master, bits, eps):
    """Moments of 0 leave a weight to its decay alone, whatever eps is; second moments below 2^-126 (gradients of 3e-19 and less) count as what they are."""
    import paper_2602_14338_amd as aero
    sizes = [700, 256, 1500, 5000]
    model = Model(19, sizes, param, "f32", master, bits)
    rng = np.random.default_rng(20)
    some = (rng.normal(0, 1, 5000) * 10.0 ** rng.uniform(-22, -15, 5000)).astype(np.float32)
    model.g = [np.zeros(700, np.float32), np.full(256, 3e-19, np.float32), np.where(np.arange(1500) % 3 == 0, np.float32(-2e-20), np.float32(0)), some]
    model.flat["grad"].copy_(model.b.put(model.g, torch.float32))
    for k in ("exp_avg", "exp_avg_sq"):
        for piece in model.b.pieces(model.flat[k]):
            piece.zero_()
    model.m = [np.zeros(s, np.float32) for s in sizes]
    model.v = [np.zeros(s, np.float32) for s in sizes]
    how = how_of(eps=eps)
    step, *_ = words()
    for t in range(2):
        aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step)
        torch.cuda.synchronize()
        # what the step is made on (squares below 2^-149 are 0 in 32 bits, and m over eps may be beyond fp16)
        assert all(torch.isfinite(x.float()).all() for x in model.b.pieces(model.flat["master" if master else "param"]))
        model.check(t, how)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_bad_gradient_and_the_norm_in_front(gh, bits, bad):
    """Through the norm a bad gradient stops the step, which leaves everything as it was; without it the elements, or their block's moments, are NaN."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    model = Model(10, [1000, 30], "f32", "f32", 0, bits)
    model.entries[0]["grad"][300] = bad
    before = {k: x.clone() for k, x in model.flat.items()}
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device="cuda")
    aero.aero_grad_norm(model.table, 1.0, 1.0, norm, factor, ws)
    step, *_ = words(4)
    aero.aero_adamw_step(model.table, aero.AdamWParams(**how_of()), step, factor)
    torch.cuda.synchronize()
    assert torch.isnan(factor).all() and not torch.isfinite(norm).any() and step.item() == 4
    for k, x in model.flat.items():
        assert torch.equal(x.view(torch.uint8), before[k].view(torch.uint8)), k
    aero.aero_adamw_step(model.table, aero.AdamWParams(**how_of()), step)
    torch.cuda.synchronize()
    e = model.entries[0]
    assert step.item() == 5 and not torch.isfinite(e["param"][300]) and torch.isfinite(e["param"][:300]).all() and torch.isfinite(e["param"][301:]).all()
    if bits == 8:
        assert torch.isnan(e["exp_avg_scale"]).tolist() == [False, True, False, False] == torch.isnan(e["exp_avg_sq_scale"]).tolist()


def test_one_table_of_everything(gh):
    """Tensors of all kinds in one table: each is stepped as by itself, with its own place in the list for its random bits; empty ones and
    gradients without parameters among them."""
    import paper_2602_14338_amd as aero
    models = [Model([k, bits], [257, 2050], p, g, m, bits) for k, (p, m) in enumerate(KINDS) for g in ("f32", "bf16", "f16") for bits in (8, 32)]
    entries = [e for m in models for e in m.entries]
    lone = torch.randn(5000, device="cuda")
    entries.insert(0, dict(grad=lone))
    entries.append(dict(grad=torch.empty(0, device="cuda")))
    order = np.random.default_rng(1).permutation(len(entries))
    order = [0] + [k for k in order if k != 0]
    table = aero.TensorTable([entries[k] for k in order])
    how = how_of(stochastic=True)
    step, *_ = words(2)
    aero.aero_adamw_step(table, aero.AdamWParams(**how), step)
    torch.cuda.synchronize()
    assert step.item() == 3
    at = 1
    for m in models:
        # tensors of a model may stand anywhere: look each up by itself
        places = [order.index(at + k) for k in range(2)]
        at += 2
        got = {k: x.clone() for k, x in m.flat.items()}
        for k in range(2):
            one = Model.__new__(Model)
            one.__dict__.update(m.__dict__)
            one.b, one.blocks = Buffers([m.b.sizes[k]], 0), Buffers([m.blocks.sizes[k]], 0)
            one.m, one.v, one.p, one.g, one.decay = [m.m[k]], [m.v[k]], [m.p[k]], [m.g[k]], [1.0]
            one.flat = {n: (m.blocks if n.endswith("scale") else m.b).pieces(x)[k].clone() for n, x in got.items()}
            one.check(2, how, first_tensor=places[k])


def test_tables_without_parameters(gh):
    import paper_2602_14338_amd as aero
    table = aero.TensorTable([dict(grad=torch.ones(10, device="cuda"))])
    step, factor, _ = words(3, 0.5)
    aero.aero_adamw_step(table, aero.AdamWParams(), step, factor)
    assert step.item() == 4
    empty = torch.empty(0, device="cuda")
    aero.aero_adamw_moments(table, empty, empty)


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_read_out(gh, bits):
    import paper_2602_14338_amd as aero
    model = Model(12, SIZES, "bf16", "bf16", 0, bits, gap=3)
    n = sum(SIZES)
    for dtype in (torch.float32, torch.bfloat16):
        out = [torch.full((n + 2,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        aero.aero_adamw_moments(model.table, out[0][1:n + 1], out[1][1:n + 1])
        torch.cuda.synchronize()
        for got, want in zip(out, (model.m, model.v)):
            assert got[0] == got[-1] == 7.0
            assert torch.equal(got[1:n + 1].cpu(), torch.from_numpy(np.concatenate(want)).to(dtype))


@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [7, 9], SIZES, [300000, 1, 5000], [6000001]])
def test_norm(gh, grad, sizes):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    b = Buffers(sizes, 1)
    rng = np.random.default_rng(sizes)
    flat = b.put([rng.normal(0, 1, s).astype(np.float32) for s in sizes], TORCH[grad])
    table = aero.TensorTable([dict(grad=x) for x in b.pieces(flat)])
    exact = np.sqrt(sum((wide(x) ** 2).sum() for x in b.get(flat)))
    ws = torch.full((aero.aero_workspace_bytes(binding.OP_GRAD_NORM),), 0x5a, dtype=torch.uint8, device="cuda")
    for scale, most in ((1.0, 1.0), (0.5, 1e9), (-0.25, 0.0), (2.0, float(exact)), (0.0, 1.0)):
        norm, factor = torch.full((1,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
        aero.aero_grad_norm(table, scale, most, norm, factor, ws)
        torch.cuda.synchronize()
        want = abs(scale) * exact
        assert abs(norm.item() - want) <= 2 * U * want
        f = scale * min(1.0, most / want) if most > 0 and want > 0 else scale
        assert abs(factor.item() - f) <= 2 * U * abs(f)
        again = torch.zeros(1, device="cuda")
        aero.aero_grad_norm(table, scale, most, again, None, ws)
        assert again.item() == norm.item()


@pytest.mark.parametrize("sizes", [[70000, 333, 90000, 5000], [524288], [524289]])
def test_norm_is_new_every_time(gh, sizes):
    """Call after call on gradients that change in between, without a wait: each result is its own gradients'."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    flat = torch.randn(sum(sizes), device="cuda")
    table = aero.TensorTable([dict(grad=x) for x in flat.split(sizes)])
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device="cuda")
    got, want = torch.zeros(300, device="cuda"), torch.zeros(300, dtype=torch.float64, device="cuda")
    for k in range(300):
        flat.mul_(-0.97 if k % 3 else 1.1)
        aero.aero_grad_norm(table, 1.0, 0.0, got[k:k + 1], None, ws)
        want[k] = flat.double().square().sum().sqrt()
    assert bool(((got.double() - want).abs() <= 2 * U * want).all())


def test_norm_of_large_and_tiny_gradients(gh):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device="cuda")
    for x in (3e38, 1e-40, 1e25):
        g = torch.full((3000,), x, device="cuda")
        norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        aero.aero_grad_norm(aero.TensorTable([dict(grad=g)]), 1.0, 1.0, norm, factor, ws)
        want = np.sqrt(3000.0) * float(g[0].double())
        assert norm.item() == float(np.float32(want)) if want > 3.4e38 else abs(norm.item() - want) <= 2 * U * want + 2.0 ** -149
        assert abs(factor.item() - min(1.0, 1.0 / want)) <= 2 * U * min(1.0, 1.0 / want) + 2.0 ** -149


def test_offsets_beyond_32_bits(gh):
    """A tensor of more than 2^31 elements: its last blocks are stepped right."""
    import paper_2602_14338_amd as aero
    n, tail = (1 << 31) + 4096 + 77, 256 + 77
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(2)
    w, dg = (torch.from_numpy(rng.normal(0, s, tail).astype(np.float32)).bfloat16() for s in (1.0, 1e-2))
    p[n - tail:], g[n - tail:] = w.cuda(), dg.cuda()
    blocks = (n + 255) // 256
    e = dict(param=p, grad=g, exp_avg=torch.zeros(n, dtype=torch.int8, device="cuda"), exp_avg_sq=torch.zeros(n, dtype=torch.uint8, device="cuda"),
             exp_avg_scale=torch.zeros(blocks, device="cuda"), exp_avg_sq_scale=torch.zeros(blocks, device="cuda"))
    how = how_of(stochastic=True)
    step, *_ = words()
    aero.aero_adamw_step(aero.TensorTable([e]), aero.AdamWParams(**how), step)
    torch.cuda.synchronize()
    m, v = orc.moments32(np.zeros(tail, np.float32), np.zeros(tail, np.float32), dg.float().numpy(), 1.0, how["beta1"], how["beta2"])
    at = np.arange(n - tail, n, dtype=np.uint64)
    of = int(orc.mix((how["seed"] & 0xffffffff) ^ int(orc.mix((how["seed"] >> 32) ^ int(orc.mix(0))))))
    h = orc.mix(int(orc.mix(of)) + at)
    for name, x, top, first, u in (("exp_avg", m, orc.TOP1, True, ((h & 0xffff) + 0.5) / 65536), ("exp_avg_sq", v, orc.TOP2, False, ((h >> 16) + 0.5) / 65536)):
        scale = orc.scale_of(x, top)
        assert np.array_equal(e[name + "_scale"][blocks - 2:].cpu().numpy(), scale)
        assert np.array_equal(e[name][n - tail:].cpu().numpy().astype(int), orc.codes_of(x, scale, u, first))
        assert not e[name][:n - tail].any() and not e[name + "_scale"][:blocks - 2].any()
    want = w.double().numpy() * (1 - how["lr"] * how["weight_decay"]) - how["lr"] * np.sign(dg.double().numpy())
    assert np.abs(p[n - tail:].double().cpu().numpy() - want).max() <= 2.0 ** -7 * np.abs(want).max()
    assert not p[:n - tail].any()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_where_one_launch_ends(gh, bits, more):
    """As many elements as one launch takes (1024 or 2048 to each of 4096 workgroups), one fewer, one more; and the norm's 1024 chunks of 2048."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    model = Model(13, [4096 * (1024 if bits == 32 else 2048) + more], "bf16", "bf16", 0, bits)
    how = how_of(stochastic=True)
    step, factor, _ = words(5, 1.5)
    aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step, factor)
    torch.cuda.synchronize()
    assert step.item() == 6
    model.check(5, how, factor=1.5)
    g = torch.randn(1024 * 2048 + more, device="cuda")
    norm = torch.zeros(1, device="cuda")
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device="cuda")
    aero.aero_grad_norm(aero.TensorTable([dict(grad=g)]), 1.0, 0.0, norm, None, ws)
    want = g.double().square().sum().sqrt().item()
    assert abs(norm.item() - want) <= 2 * U * want


def test_a_step_that_does_not_take_place_in_many_launches(gh):
    import paper_2602_14338_amd as aero
    models = [Model([3, bits], [5000], "bf16", "f32", m, bits) for m in (0, 1) for bits in (8, 32)]
    table = aero.TensorTable([e for m in models for e in m.entries])
    before = [{k: x.clone() for k, x in m.flat.items()} for m in models]
    for bad in (float("nan"), float("inf"), -float("inf")):
        step, factor, _ = words(9, bad)
        aero.aero_adamw_step(table, aero.AdamWParams(**how_of()), step, factor)
        torch.cuda.synchronize()
        assert step.item() == 9
        for m, held in zip(models, before):
            for k, x in m.flat.items():
                assert torch.equal(x, held[k]), k
    step, factor, _ = words(9, 1.0)
    aero.aero_adamw_step(table, aero.AdamWParams(**how_of()), step, factor)
    torch.cuda.synchronize()
    assert step.item() == 10
    for k, m in enumerate(models):
        m.check(9, how_of(), first_tensor=k)


@pytest.mark.parametrize("bits,sizes", [(32, [5000, 33, 2048]), (8, [5000, 33, 2048]), (32, [4300000, 7]), (8, [8500000, 7])])
def test_captured_replayed_and_on_another_stream(gh, bits, sizes):
    """Norm and step in a graph: every replay is one more step, with its own count and random bits."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    how = how_of(stochastic=True)
    a, b = (Model(14, sizes, "bf16", "bf16", 0, bits) for _ in range(2))
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_GRAD_NORM), dtype=torch.uint8, device="cuda")
    norm, factor, rate = (torch.ones(1, device="cuda") for _ in range(3))
    sa, sb = words()[0], words()[0]

    def call(model, step):
        aero.aero_grad_norm(model.table, 1.0, 0.01, norm, factor, ws)
        aero.aero_adamw_step(model.table, aero.AdamWParams(**how), step, factor, rate)
    call(a, sa)
    call(b, sb)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(a, sa)
    for k in range(3):
        rate.fill_(1.0 / (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        call(b, sb)
        torch.cuda.synchronize()
        assert sa.item() == sb.item() == k + 2
        for name in a.flat:
            assert torch.equal(a.flat[name], b.flat[name]), name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(a, sa)
    side.synchronize()
    call(b, sb)
    torch.cuda.synchronize()
    for name in a.flat:
        assert torch.equal(a.flat[name], b.flat[name]), name


def test_binding_refuses(gh):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    new = lambda dtype=torch.float32, n=300: torch.zeros(n, dtype=dtype, device="cuda")   # noqa: E731
    good = dict(param=new(), grad=new(), exp_avg=new(), exp_avg_sq=new())
    small = dict(param=new(), grad=new(), exp_avg=new(torch.int8), exp_avg_sq=new(torch.uint8), exp_avg_scale=new(n=2), exp_avg_sq_scale=new(n=2))
    table = aero.TensorTable([good, small])
    for more in (dict(param=new().cpu()), dict(grad=None), dict(exp_avg=new(torch.int8)), dict(exp_avg=None), dict(param=new(n=299)), dict(master=new()),
                 dict(param=new(torch.float16)), dict(param=new(torch.float64)), dict(grad=new(n=600)[::2]), dict(moment=new()), dict(decay=float("nan"))):
        with pytest.raises(aero.AeroError):
            aero.TensorTable([good, dict(good, **more)])
    for more in (dict(exp_avg=new()), dict(exp_avg_scale=new(n=1)), dict(exp_avg_sq_scale=None), dict(exp_avg_sq=new(torch.int8))):
        with pytest.raises(aero.AeroError):
            aero.TensorTable([dict(small, **more)])
    with pytest.raises(aero.AeroError):
        aero.TensorTable([])
    flat = new(n=900)
    for more in ([good, dict(good)], [dict(good, exp_avg_sq=good["exp_avg"])], [dict(good, param=good["grad"])],
                 [dict(good, param=flat[:300]), dict(small, param=flat[299:599])], [dict(good, param=flat[10:310], grad=flat[:300])]):
        with pytest.raises(aero.AeroError, match="overlaps"):
            aero.TensorTable(more)
    aero.TensorTable([dict(good, param=flat[:300]), dict(small, param=flat[300:600], grad=good["grad"]), dict(grad=good["grad"])])   # a gradient twice is read twice
    step, *_ = words()
    aero.aero_adamw_step(table, aero.AdamWParams(), step)
    for call in (lambda: aero.aero_adamw_step(table, aero.AdamWParams(eps=0.0), step), lambda: aero.aero_adamw_step(table, aero.AdamWParams(), step.long()),
                 lambda: aero.aero_adamw_step(table, aero.AdamWParams(), step, new(torch.float64, 1)), lambda: aero.aero_adamw_step(table, aero.AdamWParams(), None),
                 lambda: aero.aero_adamw_moments(table, new(n=599), new(n=600)), lambda: aero.aero_adamw_moments(table, new(torch.float16, 600), new(torch.float16, 600)),
                 lambda: aero.aero_adamw_moments(table, new(n=600), new(torch.bfloat16, 600)),
                 lambda: aero.aero_grad_norm(table, float("nan"), 1.0, new(n=1), new(n=1), new(torch.uint8, 1 << 16)),
                 lambda: aero.aero_grad_norm(table, 1.0, 1.0, new(n=1), new(n=1), new(torch.uint8, 16)),
                 lambda: aero.aero_grad_norm(table, 1.0, 1.0, new(n=1).double(), new(n=1), new(torch.uint8, 1 << 16))):
        with pytest.raises(aero.AeroError):
            call()
    assert step.item() == 1 and binding.OP_GRAD_NORM == 10
