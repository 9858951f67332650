"""The loss on pairs of rollouts against the float64 checker, from log-probs and from logits.

Tolerances.  A row's log-partition carries the roundings of its exponentials' arguments (numbers of the size of |z| and the offset, 2^-24 each,
8 max|z| of them in all), of a thread's additions (V / 64 at most) and of the exponential itself; row(V, z) bounds it.  A token's difference is
rounded once to 32 bits, and so is a pair's share of a slope; sums of both are exact.  With |l''| <= c an error e of a margin is at
most c e of l' (c = 1/4 for the logistic form, 2 / beta^2 for the square one; the hinge's steps are kept away from).  Outputs
round once by half a unit of their type.
"""
import numpy as np
import pytest
import torch

from oracle import training_oracle as orc

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f8": 2.0 ** -4}
HALF_LEAST = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25, "f8": 2.0 ** -10}
U = 2.0 ** -24
KIND = {"logistic": orc.LOGISTIC, "hinge": orc.HINGE, "square": orc.SQUARE}


@pytest.fixture(scope="module")
def gh():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gpu_helpers
    return gpu_helpers


def row(V, zmax):
    return U * (V / 64 + 8 * zmax + 64)


def wide(t):
    return t.cpu().float().double().numpy()


def on(x, dtype=None):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x if dtype is None else np.asarray(x, dtype))).to("cuda")


def stored(values, dtype, ld=None, off=0):
    """[T, V] values in the storage type with pitch ld, NaN behind column V, `off` elements behind a 256-byte boundary; and as stored."""
    T, V = values.shape
    ld = ld or V
    host = torch.full((T, ld), float("nan"))
    host[:, :V] = torch.from_numpy(np.asarray(values, np.float32))
    host = host.to(TORCH[dtype])
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[host.element_size()]
    flat = torch.zeros(T * ld + off, dtype=raw)
    flat[off:] = host.reshape(-1).view(raw)
    return flat.to("cuda").view(TORCH[dtype])[off:], wide(host)[:, :V]


def sevens(n, dtype, off=0):
    host = torch.full((n + off,), 7.0).to(TORCH[dtype])
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[host.element_size()]
    return host.view(raw).to("cuda").view(TORCH[dtype])[off:]


def params_of(how):
    import paper_2602_14338_amd as aero
    return aero.PreferenceParams(**how)


def curve(how):
    return {orc.LOGISTIC: 0.25, orc.HINGE: 0.0, orc.SQUARE: 2 / how["beta"] ** 2}[how["kind"]]


def bounds(want, count, size, chosen, rejected, weight, how, each):
    """Tolerances of ratio, margin, slope and loss; size[r] = sum |d| of a rollout's tokens, `each` = error of a token's log-prob."""
    loss, m, ratio, slope, *_ = want
    R = len(ratio)
    t_ratio = count * each + U * size
    if how["average"]:
        t_ratio = t_ratio / np.maximum(count, 1)
    t_ratio = t_ratio + U * np.abs(ratio)
    t_slope, t_loss, t_m = np.zeros(R), 0.0, np.zeros(len(chosen))
    for p in range(len(chosen)):
        c, j = chosen[p], rejected[p]
        w = weight[p] if weight is not None else 1.0 / len(chosen)
        if not (0 <= c < R and 0 <= j < R) or w == 0:
            continue
        e = how["beta"] * (t_ratio[c] + t_ratio[j])
        t_m[p] = e + U * abs(m[p])
        x = m[p] - how["margin"]
        if how["kind"] == orc.HINGE:
            assert abs(x - 1.0) > 2 * e, "a pair at the hinge's corner"
        k = abs(orc.pair_slope(how["kind"], x, how["beta"], how["smoothing"]))
        share = how["beta"] * abs(w) * (curve(how) * e + 2 * U * k)
        t_slope[c] += share
        t_slope[j] += share
        t_loss += abs(w) * (k * e + curve(how) * e * e + 4 * U * abs(orc.pair_value(how["kind"], x, how["beta"], how["smoothing"])))
    if how["average"]:
        t_slope = t_slope / np.maximum(count, 1)
    return t_ratio, t_m, t_slope + 2 * U * np.abs(slope), t_loss + U * abs(loss)


def near(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    nan, inf = np.isnan(want), np.isinf(want)
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[inf], want[inf])
    ok = ~nan & ~inf
    tol = np.broadcast_to(tol, want.shape)
    assert (np.abs(got[ok] - want[ok]) <= tol[ok] + 1e-37).all(), float(np.max(np.abs(got[ok] - want[ok]) - tol[ok]))


def batch(seed, T, R, P, shape="packed", V=None):
    """Tokens of R rollouts: one behind the other, in turn, or anywhere; an eighth of them padding."""
    rng = np.random.default_rng(seed)
    if shape == "packed":
        rollout = np.sort(rng.integers(0, R, T)) if R else np.full(T, -1)
    elif shape == "turns":
        rollout = np.arange(T) % max(R, 1)
    else:
        rollout = rng.integers(0, max(R, 1), T)
    rollout = np.where(rng.random(T) < 0.125, -1, rollout).astype(np.int32)
    chosen, rejected = (rng.integers(0, max(R, 1), P).astype(np.int32) for _ in range(2))
    weight = rng.uniform(0.2, 1.5, P).astype(np.float32) / max(P, 1)
    return rng, rollout, chosen, rejected, weight


def how_of(kind="logistic", average=0, beta=0.3, smoothing=0.1, margin=0.2):
    return dict(kind=KIND[kind], average=average, beta=float(np.float32(beta)), smoothing=float(np.float32(smoothing)), margin=float(np.float32(margin)))


# ------------------------------------------------------------------------------------------------ from log-probs
def run_terms(lp, ref, rollout, R, chosen, rejected, weight, how, sink=True):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    T, P = len(lp), len(chosen)
    loss, err = torch.full((1,), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    m, s, d = (torch.full((n,), 7.0, device="cuda") if sink else None for n in (P, R, R))
    ws = torch.full((aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS, T=T, R=R, Q=P),), 0x5a, dtype=torch.uint8, device="cuda")
    aero.aero_preference_loss(on(lp, np.float32), T, on(ref, np.float32) if ref is not None else None, on(rollout), R, on(chosen), on(rejected),
                              on(weight) if weight is not None else None, P, params_of(how), loss, m, s, d, ws, err)
    torch.cuda.synchronize()
    host = lambda t: None if t is None else t.cpu().numpy().astype(np.float64)   # noqa: E731
    return host(loss), host(m), host(s), host(d), int(err.item())


def check_terms(seed, T, R, P, shape="packed", ref=True, weights=True, **kw):
    rng, rollout, chosen, rejected, weight = batch(seed, T, R, P, shape)
    lp = -rng.exponential(1.0, T).astype(np.float32)
    rf = (lp + rng.normal(0, 0.3, T)).astype(np.float32) if ref else None
    how = how_of(**kw)
    weight = weight if weights else None
    want = orc.preference(lp.astype(np.float64), None if rf is None else rf.astype(np.float64), rollout, R, chosen, rejected, weight, **how)
    count = want[4]
    size = np.zeros(R)
    np.add.at(size, rollout[rollout >= 0], np.abs(lp.astype(np.float64) - (0 if rf is None else rf))[rollout >= 0])
    t_ratio, t_m, t_slope, t_loss = bounds(want, count, size, chosen, rejected, weight, how, 0.0)
    loss, m, s, d, err = run_terms(lp, rf, rollout, R, chosen, rejected, weight, how)
    assert err == 0
    near(s, want[2], t_ratio)
    near(m, want[1], t_m)
    near(d, want[3], t_slope)
    near(loss, [want[0]], t_loss)


@pytest.mark.parametrize("kind", ["logistic", "hinge", "square"])
@pytest.mark.parametrize("average", [0, 1])
@pytest.mark.parametrize("T,R,P,shape", [(1, 1, 1, "packed"), (1, 2, 1, "packed"), (63, 3, 2, "packed"), (65, 2, 5, "turns"), (1000, 16, 8, "packed"),
                                         (4097, 256, 300, "packed"), (5000, 257, 64, "packed"), (4096, 64, 4097, "turns"), (3000, 100, 50, "mixed"),
                                         (16384, 7, 40, "packed"), (16385, 7, 40, "packed"), (8192, 9, 4096, "packed"), (8193, 256, 4096, "turns"), (20000, 3000, 2000, "mixed")])
def test_terms(gh, T, R, P, shape, kind, average):
    check_terms([T, R, P], T, R, P, shape, kind=kind, average=average)


@pytest.mark.parametrize("T,R,P", [(300, 10, 6), (18000, 300, 200)])
def test_terms_without_reference_and_weights(gh, T, R, P):
    check_terms(T, T, R, P, ref=False, weights=False, beta=0.01)
    check_terms(T + 1, T, R, P, ref=False, smoothing=0.0, margin=-0.5, beta=0.02)


def test_terms_of_nothing(gh):
    for T, R, P in ((0, 0, 0), (0, 4, 2), (10, 0, 0), (10, 4, 0), (0, 300, 5000)):
        rng, rollout, chosen, rejected, weight = batch(T, T, R, P)
        loss, m, s, d, err = run_terms(np.zeros(T), None, rollout, R, chosen, rejected, weight, how_of())
        want = orc.preference(np.zeros(T), None, rollout, R, chosen, rejected, weight, **how_of())
        assert err == 0
        near(loss, [want[0]], 8 * U * abs(want[0]))
        near(m, want[1], 0)
        near(s, want[2], 0)
        near(d, want[3], 8 * U * np.abs(want[3]) + 2 * U * 0.3 * weight.sum() if P else 0)
    run_terms(np.zeros(10), None, np.zeros(10, np.int32), 4, np.array([0], np.int32), np.array([1], np.int32), None, how_of(), sink=False)


@pytest.mark.parametrize("T,R,P", [(40, 8, 6), (20000, 300, 6)])
def test_indices_out_of_range(gh, T, R, P):
    """A rollout index beyond R in a token or a pair is flagged, a negative one is not; either takes no part."""
    rng, rollout, *_ = batch(1, T, R, P)
    lp = -rng.exponential(1.0, T).astype(np.float32)
    chosen, rejected = np.array([0, -1, 2, 3, 1, 5], np.int32), np.array([1, 2, -7, 3, 4, 1], np.int32)
    want = orc.preference(lp.astype(np.float64), None, rollout, R, chosen, rejected, None, **how_of())
    loss, m, s, d, err = run_terms(lp, None, rollout, R, chosen, rejected, None, how_of())
    assert err == 0 and m[1] == m[2] == 0.0 and m[3] == 0.0 and abs(loss[0] - want[0]) < 1e-5
    near(d, want[3], 1e-6)
    chosen[4] = R
    assert run_terms(lp, None, rollout, R, chosen, rejected, None, how_of())[4] == 4
    chosen[4] = 1
    rollout[T // 2] = R + 3
    got = run_terms(lp, None, rollout, R, chosen, rejected, None, how_of())
    want = orc.preference(lp.astype(np.float64), None, rollout, R, chosen, rejected, None, **how_of())
    assert got[4] == 4 and abs(got[0][0] - want[0]) < 1e-5


@pytest.mark.parametrize("T,R", [(60, 6), (20000, 300)])
@pytest.mark.parametrize("kind", ["logistic", "hinge", "square"])
def test_log_probs_that_are_not_finite(gh, T, R, kind):
    rollout = (np.arange(T) * R // T).astype(np.int32)
    lp = np.full(T, -1.0, np.float32)
    first = [int(np.argmax(rollout == r)) for r in range(6)]
    lp[first[0]] = -np.inf
    lp[first[1]] = np.nan
    lp[first[2]] = np.inf
    lp[first[3]], lp[first[3] + 1] = np.inf, -np.inf
    chosen, rejected = np.array([0, 4, 1, 2, 3], np.int32), np.array([4, 0, 4, 4, 4], np.int32)
    for weight in (None, np.array([1, 1, 0, 1, 0], np.float32)):
        for smoothing in (0.0, 0.1):
            how = how_of(kind, smoothing=smoothing)
            with np.errstate(all="ignore"):
                want = orc.preference(lp.astype(np.float64), None, rollout, R, chosen, rejected, weight, **how)
            loss, m, s, d, _ = run_terms(lp, None, rollout, R, chosen, rejected, weight, how)
            near(s, want[2], 1e-4)
            near(m, want[1], 1e-4)
            near(loss, [want[0]], 1e-5)
            near(d, want[3], 1e-5)


@pytest.mark.parametrize("T,R", [(60, 6), (3000, 6), (20000, 300)])
@pytest.mark.parametrize("packed", [True, False])
def test_log_probs_of_the_lowest_value(gh, T, R, packed):
    """Finite tokens whose sum is beyond 32 bits: log ratios are formed in 64, margins are finite where beta makes them so, and 0 between rollouts alike."""
    rollout = np.sort(np.arange(T) % R).astype(np.int32) if packed else (np.arange(T) % R).astype(np.int32)
    lp = np.full(T, -1.0, np.float32)
    low = np.finfo(np.float32).min
    of = [np.nonzero(rollout == r)[0] for r in range(6)]
    lp[of[0][:3]] = lp[of[1][-3:]] = lp[of[2][:2]] = lp[of[4]] = low
    lp[of[3][:2]], lp[of[5][[0, 1, 5]]] = -low, [low, low, -low]
    chosen, rejected = np.array([0, 2, 1, 3, 4, 5], np.int32), np.array([1, 0, 2, 4, 5, 2], np.int32)
    weight = np.array([0.5, 1.0, 2.0, 1.0, 0.25, 1.0], np.float32) / 1024
    how = how_of(beta=2.0 ** -20, margin=0.0)
    want = orc.preference(lp.astype(np.float64), None, rollout, R, chosen, rejected, weight, **how)
    count, size = np.bincount(rollout, minlength=R), np.zeros(R)
    np.add.at(size, rollout, np.abs(lp.astype(np.float64)))
    t_ratio, t_m, t_slope, t_loss = bounds(want, count, size, chosen, rejected, weight, how, 0.0)
    loss, m, s, d, err = run_terms(lp, None, rollout, R, chosen, rejected, weight, how)
    with np.errstate(over="ignore"):
        near(s, want[2].astype(np.float32), t_ratio)
    near(m, want[1], t_m)
    assert m[0] == 0.0
    near(loss, [want[0]], t_loss)
    # far from a margin of 0 the logistic form's slope is -1 or 0, less the smoothing
    slope = np.zeros(R)
    for p in range(1, 6):
        k = how["beta"] * weight[p] * (how["smoothing"] - (1.0 if want[1][p] < 0 else 0.0))
        slope[chosen[p]] += k
        slope[rejected[p]] -= k
    k = how["beta"] * weight[0] * (how["smoothing"] - 0.5)
    slope[0] += k
    slope[1] -= k
    near(d, slope, 8 * U * how["beta"] * weight.sum())


@pytest.mark.parametrize("T,R,P", [(4000, 50, 300), (30000, 500, 6000)])
def test_terms_do_not_depend_on_order(gh, T, R, P):
    """Tokens and pairs in another order leave the same bits, in slopes whose terms differ by many magnitudes too."""
    rng, rollout, chosen, rejected, weight = batch(5, T, R, P, "mixed")
    lp = (-rng.exponential(1.0, T) * 10.0 ** rng.integers(-6, 3, T)).astype(np.float32)
    weight = (weight * 10.0 ** rng.integers(-20, 3, P)).astype(np.float32)
    a = run_terms(lp, None, rollout, R, chosen, rejected, weight, how_of())
    t, p = rng.permutation(T), rng.permutation(P)
    b = run_terms(lp[t], None, rollout[t], R, chosen[p], rejected[p], weight[p], how_of())
    assert np.array_equal(a[1][p], b[1])
    big = lambda x: np.abs(x) * 2.0 ** -47   # noqa: E731 - a wave's own sums are rounded in 64 bits before they are added up
    near(a[2], b[2], U * np.abs(a[2]) + big(a[2]).max())
    c = run_terms(lp, None, rollout, R, chosen, rejected, weight, how_of())
    for x, y in zip(a[:4], c[:4]):
        assert np.array_equal(x, y)


def test_terms_of_the_largest_call(gh):
    """As many tokens, rollouts and pairs as a call takes, against the same sums by the tensor library in 64 bits."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    T, R, P = (1 << 25) - 1, (1 << 22) - 1, (1 << 22) - 1
    g = torch.Generator(device="cuda").manual_seed(1)
    rollout = torch.randint(-1, R, (T,), generator=g, device="cuda", dtype=torch.int32)
    lp = -torch.rand(T, generator=g, device="cuda")
    c, j = (torch.randint(0, R, (P,), generator=g, device="cuda", dtype=torch.int32) for _ in range(2))
    loss, m, s, d = (torch.zeros(n, device="cuda") for n in (1, P, R, R))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS, T=T, R=R, Q=P), dtype=torch.uint8, device="cuda")
    how = how_of(smoothing=0.0, margin=0.0, average=1)
    aero.aero_preference_loss(lp, T, None, rollout, R, c, j, None, P, params_of(how), loss, m, s, d, ws, err)
    there = rollout >= 0
    count = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, rollout[there].long(), torch.ones_like(lp[there]).double()).clamp(min=1)
    ratio = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, rollout[there].long(), lp[there].double()) / count
    x = how["beta"] * (ratio[c.long()] - ratio[j.long()])
    share = -how["beta"] / P * torch.sigmoid(-x)
    slope = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, c.long(), share).index_add_(0, j.long(), -share) / count
    assert err.item() == 0
    assert bool(((s.double() - ratio).abs() <= 4 * U * ratio.abs()).all())
    assert bool(((m.double() - x).abs() <= 8 * U * how["beta"]).all())
    # a share is rounded to 32 bits, and so is 1 / P; every one is 0.3 / P at most, and a rollout has 20 of them at most
    assert bool(((d.double() - slope).abs() <= 20 * 4 * U * how["beta"] / P + 2 * U * slope.abs()).all())
    want = torch.nn.functional.softplus(-x).mean()
    assert abs(loss.item() - want.item()) <= 8 * U * want.item()


# ------------------------------------------------------------------------------------------------ from logits
def run_rows(z, T, V, ld, dtype, y, ref, rollout, R, chosen, rejected, weight, how, scale=1.0, inplace=False, want_dz=True, off=0):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    P = len(chosen)
    loss, err = torch.full((1,), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    m, s, lp = (torch.full((n,), 7.0, device="cuda") for n in (P, R, T))
    dz = None if not want_dz else z if inplace else sevens(T * ld, dtype, off)
    ws = torch.full((aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=T, V=V, R=R, Q=P),), 0x5a, dtype=torch.uint8, device="cuda")
    aero.aero_preference_loss_bwd(z, T, V, ld, on(y, np.int32), on(ref, np.float32) if ref is not None else None, on(rollout), R, on(chosen),
                                  on(rejected), on(weight) if weight is not None else None, P, params_of(how), scale, loss, m, s, lp, dz, ws, err)
    torch.cuda.synchronize()
    host = lambda t: None if t is None else wide(t)   # noqa: E731
    return host(loss), host(m), host(s), host(lp), None if dz is None else host(dz).reshape(T, ld), int(err.item())


def check_rows(seed, T, V, R, P, dtype, ld=None, off=0, off_d=None, shape="packed", ref=True, weights=True, inplace=False, change=None, err=0,
               scale=None, sigma=3.0, distances=False, **kw):
    rng, rollout, chosen, rejected, weight = batch(seed, T, R, P, shape)
    values = rng.normal(0, sigma, size=(T, V)).astype(np.float32)
    y = rng.integers(0, V, T).astype(np.int32)
    if change:
        change(values, y, rollout)
    z, host = stored(values, dtype, ld, off)
    ld = ld or V
    how = how_of(**kw)
    scale = scale or (4.0 * P if dtype in ("f16", "f8") else 1.0)
    rf = rng.normal(-6, 1, T).astype(np.float32) if ref else None
    weight = weight if weights else None
    with np.errstate(all="ignore"):
        want = orc.preference_rows(host, V, y, None if rf is None else rf.astype(np.float64), rollout, R, chosen, rejected, weight, grad_scale=scale, **how)
    w_loss, w_m, w_s, w_d, w_lp, w_dz, q = want
    part = (rollout >= 0) & (rollout < R) & (y >= 0) & (y < V) & ((host > orc.MASKED).any(axis=1) | np.isnan(host).any(axis=1))
    d = np.where(part, w_lp - (0 if rf is None else rf.astype(np.float64)), 0.0)
    count, size = np.zeros(R), np.zeros(R)
    np.add.at(count, rollout[part], 1)
    np.add.at(size, rollout[part], np.abs(d[part]))
    finite = np.abs(host[np.isfinite(host) & (np.abs(host) < 1.2e9)])
    e, own, lost = row(V, float(finite.max()) if finite.size else 0.0), 0.0, 0.0
    if distances:
        # an argument is rounded near the offset, which is a whole number within 3 of the row's largest (or half a unit of 32 bits there)
        half = 2.0 ** (np.frexp(1.4427 * np.abs(host).max())[1] - 25)
        far = np.where(q > 0, host.max(axis=1, keepdims=True) - host, 0.0) * 1.4427 + 3 + half
        # exponentials below 2^-126 are 0, in a sum that is at least its largest, 2^-(1 + half): at -1e9 (half a unit is 64) a logit 64 below the largest, e^-64 = 2^-92.3
        # of the sum, has an argument down to -157
        lost = 2.0 ** (-125 + half)
        own = U * far
        e = row(V, 0.0) + float((q * own).sum(axis=1).max())
    t_s, t_m, t_d, t_loss = bounds((w_loss, w_m, w_s, w_d), count, size, chosen, rejected, weight, how, e)
    loss, m, s, lp, dz, bits = run_rows(z, T, V, ld, dtype, y, rf, rollout, R, chosen, rejected, weight, how, scale, inplace,
                                        off=off if off_d is None else off_d)
    assert bits == err
    near(lp, w_lp, e + U * np.abs(w_lp))
    near(s, w_s, t_s)
    near(m, w_m, t_m)
    near(loss, [w_loss], t_loss)
    hot = np.zeros((T, V))
    hot[np.nonzero(part)[0], y[part]] = 1.0
    slope = np.where(part, w_d[np.clip(rollout, 0, max(R - 1, 0))] if R else 0.0, 0.0)
    t_slope = np.where(part, t_d[np.clip(rollout, 0, max(R - 1, 0))] if R else 0.0, 0.0)
    with np.errstate(all="ignore"):
        tol = scale * (t_slope[:, None] * (hot + q) + np.abs(slope)[:, None] * ((2 * e + own) * q + lost + 4 * U * (hot + q)))
        tol = tol * (1 + HALF_ULP[dtype]) + HALF_ULP[dtype] * np.abs(w_dz) + HALF_LEAST[dtype]
    if dtype == "f8":
        w_dz = np.clip(w_dz, -448, 448)
    left = rollout == -2
    assert (dz[left, :V] == (host[left] if inplace else 7.0)).all() or np.isnan(host[left]).any()
    near(dz[~left, :V], w_dz[~left], tol[~left])
    if not inplace:
        assert (dz[:, V:] == 7.0).all()
    return dz


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "f8"])
@pytest.mark.parametrize("T,V,R,P,ld,off", [
    (1, 1, 1, 1, 1, 0), (2, 1, 2, 1, 3, 1), (5, 7, 2, 3, 9, 0), (6, 64, 4, 2, 64, 0), (40, 1000, 6, 5, 1003, 3), (30, 1024, 8, 12, 1024, 0), (9, 2049, 4, 3, 2053, 1),
    (20, 4097, 5, 5, 4100, 0), (300, 130, 300, 40, 130, 1), (7, 10007, 3, 2, 10007, 5), (4, 50257, 2, 2, 50257, 0), (3, 65537, 2, 1, 65600, 0), (3, 151936, 2, 2, 151936, 0)])
def test_rows(gh, dtype, T, V, R, P, ld, off):
    check_rows([T, V], T, V, R, P, dtype, ld, off)


@pytest.mark.parametrize("T,R,P", [(4096, 256, 40), (4097, 256, 40), (4096, 257, 40), (4100, 5, 4097)])
def test_rows_where_the_forms_of_their_sums_meet(gh, T, R, P):
    check_rows([T, R], T, 65, R, P, "f32", shape="packed")
    check_rows([T, R, 1], T, 65, R, P, "bf16", ld=70, shape="turns")


@pytest.mark.parametrize("kind", ["logistic", "hinge", "square"])
@pytest.mark.parametrize("average", [0, 1])
@pytest.mark.parametrize("ref", [True, False])
def test_rows_of_every_loss(gh, kind, average, ref):
    check_rows(11, 60, 515, 7, 9, "bf16", ref=ref, kind=kind, average=average, weights=average == 0)
    check_rows(12, 60, 515, 300, 150, "f32", ref=ref, kind=kind, average=average, shape="mixed")


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f8"])
def test_rows_in_place_and_apart(gh, dtype):
    """In place; and into a buffer whose offset from 16 bytes is another one than the logits'."""
    check_rows(21, 50, 777, 6, 8, dtype, ld=780, inplace=True)
    check_rows(22, 12, 40000, 6, 8, dtype, inplace=True)
    check_rows(23, 50, 777, 6, 8, dtype, ld=777, off=0, off_d=1)
    check_rows(24, 8, 20001, 4, 4, dtype, ld=20001, off=3, off_d=2)


@pytest.mark.parametrize("R,P", [(6, 5), (280, 50)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_take_no_part(gh, dtype, R, P):
    """Padding, rows to be left alone, missing and bad ids, rows without an unmasked logit."""
    def change(z, y, rollout):
        rollout[3], rollout[4], rollout[5] = -2, -1, -9
        y[6], y[7] = -1, -3
        z[8] = -np.inf
        z[9] = -1e10
        z[10] = np.finfo(np.float32).min if dtype == "f32" else -3e38
        rollout[8:11] = 1
    check_rows(31, 40, 300, R, P, dtype, change=change)
    check_rows(31, 40, 300, R, P, dtype, change=change, inplace=True)

    def bad(z, y, rollout):
        change(z, y, rollout)
        y[12], rollout[12] = 300, 1
        rollout[13] = R
    check_rows(32, 40, 300, R, P, dtype, change=bad, err=2 | 4)


@pytest.mark.parametrize("R,P", [(6, 5), (280, 80)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_with_masked_logits(gh, dtype, R, P):
    low = {"bf16": -3.3e38, "f16": -np.inf, "f32": float(np.finfo(np.float32).min)}[dtype]

    def change(z, y, rollout):
        rng = np.random.default_rng(7)
        for t in range(len(z)):
            masked = rng.random(z.shape[1]) < rng.choice([0.1, 0.5, 0.99])
            masked[y[t]] = False
            z[t, masked] = rng.choice([-np.inf, low, -1e10 if dtype != "f16" else -np.inf])
    check_rows(41, 30, 1100, R, P, dtype, change=change)


@pytest.mark.parametrize("R", [4, 260])
def test_a_masked_sampled_token(gh, R):
    """Its log-prob is -inf, its rollout's ratio too; the pair's gradient is the limit's and stays finite (but for a pair of that rollout with itself,
    whose margin is -inf + inf)."""
    def change(z, y, rollout):
        rollout[:] = np.arange(len(rollout)) % 4
        z[5, y[5]] = -np.inf
    _, _, chosen, rejected, _ = batch(51, 24, R, 6)
    itself = bool(((chosen == 1) & (rejected == 1)).any())
    dz = check_rows(51, 24, 200, R, 6, "f32", change=change, smoothing=0.0)
    assert np.isfinite(dz[np.arange(24) % 4 != 1]).all() and (itself or np.isfinite(dz).all())


@pytest.mark.parametrize("value", [np.nan, np.inf, 2e9])
def test_a_row_with_a_bad_logit(gh, value):
    def change(z, y, rollout):
        rollout[:] = np.arange(len(rollout)) % 6
        z[3, 17] = value
    dz = check_rows(61, 30, 200, 6, 8, "f32", change=change)
    assert np.isnan(dz[3]).all()


@pytest.mark.parametrize("size", [1e3, 1e6, 1e8])
def test_rows_of_large_logits(gh, size):
    def change(z, y, rollout):
        z += size
    check_rows(71, 20, 300, 4, 4, "f32", change=change)


FAR = {"f32": [1e3, 1e5, 2.0 ** 23, 1e8, 1e9], "bf16": [1e3, 1e5, 1e8, 1e9], "f16": [1e3, 6e4]}


@pytest.mark.parametrize("dtype,size", [(d, sign * x) for d, sizes in FAR.items() for x in sizes for sign in (1, -1)])
def test_rows_far_from_0(gh, dtype, size):
    """All of a row's logits far from 0, in steps of their type's unit there (or of an eighth); a log-prob is as exact as near 0, and the probabilities are those of
    the distances from the largest logit.  Two rows are the same number throughout."""
    digits = {"f32": 24, "bf16": 8, "f16": 11}[dtype]
    unit = max(2.0 ** (np.frexp(size)[1] - digits), 0.125)

    def change(z, y, rollout):
        z[:] = size + unit * np.round(z / min(unit, 3.0))
        z[[3, 7]] = size
    check_rows(72, 24, 300, 4, 4, dtype, change=change, distances=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [-1e9, 1e9])
@pytest.mark.parametrize("V", [300, 20000])
def test_a_row_far_from_0_among_others(gh, dtype, size, V):
    """A uniform row, whatever its number: log-prob -ln V, in a rollout of ordinary rows."""
    def change(z, y, rollout):
        rollout[:] = np.arange(len(rollout)) % 4
        z[5] = size
    dz = check_rows(73, 20, V, 4, 4, dtype, change=change, distances=True)
    assert np.isfinite(dz).all() and (dz[5] != 0).all()


def test_rollout_far_off_the_reference(gh):
    """Margins of thousands: the logistic form saturates, its loss is the margin."""
    def change(z, y, rollout):
        z *= 30
    check_rows(81, 60, 400, 4, 6, "f32", change=change, beta=5.0)


def test_loss_alone_and_outputs_left_out(gh):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    rng, rollout, chosen, rejected, weight = batch(91, 40, 6, 5)
    z, host = stored(rng.normal(0, 3, (40, 600)).astype(np.float32), "bf16")
    y = rng.integers(0, 600, 40).astype(np.int32)
    full = run_rows(z, 40, 600, 600, "bf16", y, None, rollout, 6, chosen, rejected, weight, how_of())
    less = run_rows(z, 40, 600, 600, "bf16", y, None, rollout, 6, chosen, rejected, weight, how_of(), want_dz=False)
    for a, b in zip(full[:4], less[:4]):
        assert np.array_equal(a, b)
    loss = torch.zeros(1, device="cuda")
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=40, V=600, R=6, Q=5), dtype=torch.uint8, device="cuda")
    aero.aero_preference_loss_bwd(z, 40, 600, 600, on(y), None, on(rollout), 6, on(chosen), on(rejected), on(weight), 5, params_of(how_of()), 1.0, loss,
                                  None, None, None, None, ws)
    assert loss.item() == full[0][0]


def test_no_rows_no_rollouts_no_pairs(gh):
    for T, R, P in ((0, 3, 2), (4, 0, 0), (4, 3, 0)):
        rng, rollout, chosen, rejected, weight = batch(T, T, R, P)
        z, _ = stored(np.zeros((T, 50), np.float32), "bf16")
        loss, m, s, lp, dz, err = run_rows(z, T, 50, 50, "bf16", np.zeros(T, np.int32), None, rollout, R, chosen, rejected, weight, how_of())
        assert err == 0 and (dz == 0).all()
        want = orc.preference(np.zeros(T), None, np.full(T, -1), R, chosen, rejected, weight, **how_of())[0] if P else 0.0
        near(loss, [want], 1e-6)


@pytest.mark.parametrize("T,R,P", [(0, 256, 0), (0, 300, 0), (0, 256, 40), (0, 300, 40), (0, 4097, 5000), (3, 300, 40)])
@pytest.mark.parametrize("want_dz", [True, False])
def test_calls_stay_in_their_workspace(gh, T, R, P, want_dz):
    """A workspace of exactly the size that is asked for, with or without rows: what stands behind it stays, and the outputs are those of rollouts without tokens."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    _, rollout, chosen, rejected, weight = batch(T + R, T, R, P)
    V, behind = 50, 1 << 16
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    loss, m, s = (torch.full((n,), 7.0, device="cuda") for n in (1, P, R))
    size = aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=T, V=V, R=R, Q=P)
    ws = torch.full((size + behind,), 0x5a, dtype=torch.uint8, device="cuda")
    how = how_of()
    aero.aero_preference_loss_bwd(z, T, V, V, on(np.zeros(T, np.int32)), None, on(rollout), R, on(chosen), on(rejected), on(weight), P, params_of(how), 1.0, loss,
                                  m, s, torch.zeros(T, device="cuda"), torch.empty_like(z) if want_dz else None, ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0x5a).all()
    want = orc.preference(np.full(T, -np.log(V)), None, rollout, R, chosen, rejected, weight, **how)
    e = T * (row(V, 0) + 4 * U)   # of a log ratio; margins are beta < 1/2 times two of them, the loss's slope is 1 at most
    near(wide(s), want[2], e)
    near(wide(m), want[1], e)
    near(wide(loss), [want[0]], weight.sum() * e + 8 * U * abs(want[0]))


def test_offsets_beyond_32_bits(gh):
    """More than 2^32 logits: the last rows' gradient is right."""
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    V, T = 151936, 28300
    assert T * V > 1 << 32
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    y = torch.arange(T, device="cuda", dtype=torch.int32)
    z[-1, 5] = 12.0
    rollout = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    rollout[0], rollout[-2], rollout[-1] = 0, 1, 1
    loss, lp = torch.zeros(1, device="cuda"), torch.zeros(T, device="cuda")
    one = lambda k: torch.tensor([k], dtype=torch.int32, device="cuda")   # noqa: E731
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=T, V=V, R=2, Q=1), dtype=torch.uint8, device="cuda")
    aero.aero_preference_loss_bwd(z, T, V, V, y, None, rollout, 2, one(0), one(1), None, 1, params_of(how_of(beta=0.5, smoothing=0.0, margin=0.0)), 1.0,
                                  loss, None, None, lp, z, ws)
    lse = [np.log(V), np.log(V), np.log(V - 1 + np.exp(12.0))]
    x = 0.5 * (-lse[0] + lse[1] + lse[2])
    g = -0.5 / (1 + np.exp(x))
    got = z[[0, T - 2, T - 1]].double().cpu().numpy()
    for k, t in enumerate((0, T - 2, T - 1)):
        row_z = np.zeros(V)
        if k == 2:
            row_z[5] = 12.0
        want = -np.exp(row_z - lse[k])
        want[t] += 1.0
        want *= g if k == 0 else -g
        assert np.abs(got[k] - want).max() <= 2.0 ** -8 * np.abs(want).max() and np.abs(got[k] / want - 1).max() < 2.0 ** -8 + 1e-4
    assert not z[1:T - 2].any()


@pytest.mark.parametrize("T,R,P", [(200, 8, 10), (17000, 300, 200)])
def test_captured_replayed_and_on_another_stream(gh, T, R, P):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    V = 256
    rng, rollout, chosen, rejected, weight = batch(101, T, R, P)
    z, _ = stored(rng.normal(0, 3, (T, V)).astype(np.float32), "bf16")
    args = [on(rng.integers(0, V, T).astype(np.int32)), on(rng.normal(-6, 1, T).astype(np.float32)), on(rollout), R, on(chosen), on(rejected), on(weight), P]
    out = [torch.zeros(n, device="cuda") for n in (1, P, R, T)] + [torch.zeros_like(z)]
    terms = [torch.zeros(n, device="cuda") for n in (1, P, R, R)]
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=T, V=V, R=R, Q=P), dtype=torch.uint8, device="cuda")

    def call():
        aero.aero_preference_loss_bwd(z, T, V, V, *args, params_of(how_of()), 1.0, *out, ws)
        aero.aero_preference_loss(out[3], T, args[1], *args[2:], params_of(how_of()), *terms, ws)
    call()
    torch.cuda.synchronize()
    eager = [t.clone() for t in out + terms]
    near(wide(terms[0]), wide(out[0]), 1e-5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in out + terms:
            t.fill_(7)
        ws.fill_(0x33)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip(out + terms, eager):
            assert torch.equal(t, e)
    side = torch.cuda.Stream()
    for t in out + terms:
        t.fill_(7)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    for t, e in zip(out + terms, eager):
        assert torch.equal(t, e)


def test_binding_refuses(gh):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    rng, rollout, chosen, rejected, weight = batch(1, 8, 4, 3)
    z, _ = stored(np.zeros((8, 32), np.float32), "bf16")
    ws = torch.empty(aero.aero_workspace_bytes(binding.OP_PREFERENCE_LOSS_BWD, T=8, V=32, R=4, Q=3), dtype=torch.uint8, device="cuda")
    loss = torch.zeros(1, device="cuda")
    good = dict(z=z, y=on(np.zeros(8, np.int32)), r=on(rollout), c=on(chosen), j=on(rejected), w=on(weight), p=params_of(how_of()), l=loss, d=torch.empty_like(z))

    def call(**more):
        a = dict(good, **more)
        aero.aero_preference_loss_bwd(a["z"], 8, 32, 32, a["y"], None, a["r"], 4, a["c"], a["j"], a["w"], 3, a["p"], 1.0, a["l"], None, None, None, a["d"], ws)
    call()
    for more in (dict(y=good["y"].long()), dict(r=good["r"].cpu()), dict(c=good["c"].long()), dict(w=good["w"].double()), dict(l=None), dict(d=z.float()),
                 dict(z=z.double()), dict(p=aero.PreferenceParams(beta=0.0)), dict(z=torch.zeros((64, 8), dtype=torch.bfloat16, device="cuda").t())):
        with pytest.raises(aero.AeroError):
            call(**more)
