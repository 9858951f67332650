"""The calls around a drafter against the float64 checker: a teacher's lists, distillation and its gradient, verification of
drafted tokens, embedding rows and their gradient.

Tolerances.  A row's exponentials are exp2 of fma(z, log2 e, c): the argument carries the rounding of numbers of the size of
|z| + |offset| (2^-24 relative, so about 2^-23 max|z| in the logarithm), a thread adds up to V / 64 of them one after the other, the
rest is a tree: rel(V, z) below bounds the relative error of a row's sum and of a probability.  Sums of lists
are formed in 64 bits.  Results round to their storage type by half a unit in the last place, and near its smallest
numbers by half the smallest one.
"""
import numpy as np
import pytest
import torch

from oracle import drafter_oracle as orc

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f8": 2.0 ** -4}
HALF_LEAST = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25, "f8": 2.0 ** -10}


@pytest.fixture(scope="module")
def gh():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gpu_helpers
    return gpu_helpers


def rel(V, zmax):
    return 2.0 ** -24 * (V / 64 + 8 * zmax + 64)


def wide(t):
    return t.cpu().float().double().numpy()


def stored(values, dtype, ld=None, off=0):
    """[T, V] values in the storage type with pitch ld, NaN behind column V, `off` elements behind a 256-byte boundary; and the
    values as they are stored."""
    T, V = values.shape
    ld = ld or V
    host = torch.full((T, ld), float("nan"))
    host[:, :V] = torch.from_numpy(np.asarray(values, np.float32))
    host = host.to(TORCH[dtype])
    flat = torch.zeros(T * ld + off, dtype=torch.float32).to(TORCH[dtype])
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[flat.element_size()]
    flat.view(raw)[off:] = host.reshape(-1).view(raw)
    dev = flat.view(raw).to("cuda").view(TORCH[dtype])[off:]
    return dev, wide(host)[:, :V]


def sevens(T, ld, dtype, off=0):
    host = torch.full((T * ld + off,), 7.0).to(TORCH[dtype])
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[host.element_size()]
    return host.view(raw).to("cuda").view(TORCH[dtype])[off:]


def normal(seed, T, V, sigma=3.0):
    return np.random.default_rng(seed).normal(0, sigma, size=(T, V)).astype(np.float32)


def workspace(op, **sizes):
    import paper_2602_14338_amd as aero
    from paper_2602_14338_amd import binding
    return torch.full((aero.aero_workspace_bytes(getattr(binding, op), **sizes),), 0x5a, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ lists
def run_top(z, T, V, ld, K, active=None, want_lse=True):
    import paper_2602_14338_amd as aero
    index = torch.full((T, K), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((T, K), 7.0, device="cuda")
    lse = torch.full((T,), 7.0, device="cuda") if want_lse else None
    act = torch.from_numpy(active).to("cuda") if active is not None else None
    aero.aero_topk_logprob(z, T, V, ld, act, K, index, lp, lse, workspace("OP_TOPK_LOGPROB", T=T, V=V, H=K))
    torch.cuda.synchronize()
    return index.cpu().numpy(), lp.cpu().numpy().astype(np.float64), None if lse is None else lse.cpu().numpy().astype(np.float64)


def check_top(values, dtype, K, ld=None, off=0, active=None):
    T, V = values.shape
    z, host = stored(values, dtype, ld, off)
    index, lp, lse = run_top(z, T, V, ld or V, K, active)
    want_i, want_lp, want_lse = orc.top(host, V, K, active)
    assert np.array_equal(index, want_i)
    finite = np.abs(host[np.isfinite(host) & (host > orc.MASKED)])
    zmax = float(finite.max()) if finite.size else 0.0
    for got, want in ((lp, want_lp), (lse, want_lse)):
        nan, inf = np.isnan(want), np.isinf(want)
        assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[inf], want[inf])
        ok = ~nan & ~inf
        assert (np.abs(got[ok] - want[ok]) <= rel(V, zmax) + 2.0 ** -23 * np.abs(want[ok])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "f8"])
@pytest.mark.parametrize("T,V,K,ld,off", [
    (1, 1, 1, 1, 0), (3, 7, 4, 9, 0), (2, 5, 9, 5, 1), (5, 64, 64, 64, 0), (4, 1000, 1, 1000, 3), (6, 1024, 16, 1024, 0),
    (3, 2047, 256, 2047, 0), (3, 2049, 64, 2053, 1), (2, 4096, 130, 4096, 0), (2, 10007, 100, 10007, 5), (3, 50257, 50, 50257, 0),
    (2, 65537, 256, 65600, 0), (2, 151936, 64, 151936, 0), (1, 262144, 128, 262144, 0)])
def test_top(gh, dtype, T, V, K, ld, off):
    check_top(normal([T, V, K], T, V), dtype, K, ld, off)


@pytest.mark.parametrize("dtype,V,K", [
    ("bf16", 2047, 128), ("bf16", 2049, 129), ("bf16", 4095, 256), ("bf16", 4098, 256), ("bf16", 4097, 17), ("bf16", 8193, 128), ("bf16", 8210, 129),
    ("bf16", 16385, 100), ("bf16", 16400, 1), ("bf16", 32770, 64), ("bf16", 32790, 128), ("f32", 1023, 128), ("f32", 2051, 100), ("f32", 4099, 129),
    ("f32", 8197, 60), ("f8", 4096, 128), ("f8", 8193, 200), ("f8", 16385, 128), ("f8", 33000, 7)])
def test_top_where_its_forms_meet(gh, dtype, V, K):
    """Lengths around what a workgroup holds in registers, with few rows and with more than two per compute unit."""
    check_top(normal([V, K, 3], 3, V), dtype, K)
    check_top(normal([V, K, 4], 521, V), dtype, K, ld=V + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f8"])
@pytest.mark.parametrize("V", [300, 4000, 40000])
def test_top_of_rows_without_order(gh, dtype, V):
    """Equal logits, logits that rise or fall with the id, few distinct ones, large ones at the end, signed zeros."""
    rng = np.random.default_rng(V)
    z = normal(V, 9, V)
    z[0] = 0.0
    z[1] = np.sort(z[1])
    z[2] = -np.sort(-z[2])
    z[3] = rng.integers(0, 3, size=V)
    z[4, -200:] += 30.0
    z[5] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    z[6] = np.where(rng.random(V) < 0.05, 4.0, -4.0)
    z[7] = 448.0
    z[8, : V // 2] = 200.0
    for K in (1, 50, 256):
        check_top(z, dtype, K)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_top_of_masked_rows(gh, dtype):
    V, K = 3001, 40
    z = normal(4, 10, V)
    lowest = float(torch.finfo(TORCH[dtype]).min)
    z[0] = -np.inf
    z[1, 7:] = -np.inf
    z[2, : V - 3] = -np.inf
    z[3, 1::2] = lowest
    z[4, 100:] = lowest
    if dtype != "f16":
        z[5] = lowest
    z[6, 1234] = np.nan
    z[7, 2000] = np.inf
    active = np.ones(10, np.uint8)
    active[8] = 0
    check_top(z, dtype, K, active=active)
    check_top(z[:, :39], dtype, K, active=active)


def test_top_without_lse_and_of_no_rows(gh):
    import paper_2602_14338_amd as aero
    values = normal(5, 3, 500)
    z, host = stored(values, "bf16")
    index, lp, _ = run_top(z, 3, 500, 500, 5, want_lse=False)
    assert np.array_equal(index, orc.top(host, 500, 5)[0])
    aero.aero_topk_logprob(z, 0, 500, 500, None, 5, torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda"), None,
                           workspace("OP_TOPK_LOGPROB", T=0, V=500, H=5))


@pytest.mark.parametrize("T", [2, 63, 64, 200, 257, 600])
def test_top_of_any_number_of_rows(gh, T):
    """Rows are split over workgroups where there are few."""
    check_top(normal(T, T, 33000 if T <= 64 else 9000), "bf16", 64)


# ------------------------------------------------------------------------------------------------ distillation
def make_lists(seed, host, K, spread=0.5):
    """Lists of a teacher near the student."""
    rng = np.random.default_rng([seed, 5])
    near = host + rng.normal(0, spread, size=host.shape)
    index, lp, _ = orc.top(near, host.shape[1], K)
    return index.astype(np.int32), np.where(np.isfinite(lp), lp, -1.0).astype(np.float32)


def run_distill(z, T, V, ld, index, lp, w, tail, scale, dz, row_loss=True):
    import paper_2602_14338_amd as aero
    loss, rows = torch.full((1,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda") if row_loss else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    up = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).to("cuda")
    aero.aero_distill_loss_bwd(z, T, V, ld, up(index, np.int32), up(lp, np.float32), index.shape[1], up(w, np.float32), tail, scale, loss,
                               rows, dz, workspace("OP_DISTILL_LOSS_BWD", T=T, V=V), err)
    torch.cuda.synchronize()
    return loss.item(), None if rows is None else rows.cpu().numpy().astype(np.float64), int(err.item())


def distill_bounds(ref, host, w, dtype, scale):
    V = host.shape[1]
    zmax = float(np.abs(host[np.isfinite(host) & (host > orc.MASKED)]).max())
    r = rel(V, zmax)
    total, rest_p, rest_q = ref["masses"].T
    row = 4 * r * (total + rest_p) + 2.0 ** -22 * np.abs(ref["row_loss"])
    g = np.abs(scale * np.asarray(w, np.float64))[:, None]
    share = np.where(rest_q[:, None] > 0, ref["q"] / np.maximum(rest_q[:, None], 1e-300), 0.0)
    size = total[:, None] * ref["q"] + ref["p"] + np.where(ref["p"] > 0, 0.0, rest_p[:, None] * share)
    grad = g * size * (4 * r + 2.0 ** -22) + HALF_ULP[dtype] * np.abs(ref["dlogits"]) + HALF_LEAST[dtype]
    return row, grad


def check_distill(values, dtype, K, tail, ld=None, off=0, off_d=None, scale=1.0, w=None, lists=None, inplace=False, seed=0):
    T, V = values.shape
    ld = ld or V
    z, host = stored(values, dtype, ld, off)
    index, lp = lists if lists is not None else make_lists(seed, np.where(np.isfinite(host), host, -1e6), K)
    if w is None:
        w = np.random.default_rng([seed, 6]).uniform(0.2, 1.0, size=T).astype(np.float32)
        w[::5] = 0.0
        if T == 1:
            w[0] = 0.7
    ref = orc.distill(host, V, index, lp, w, tail, scale)
    dz = z if inplace else sevens(T, ld, dtype, off if off_d is None else off_d)
    loss, rows, err = run_distill(z, T, V, ld, index, lp, w, tail, scale, dz)
    assert err == (8 if ref["bad"].any() else 0)
    got = wide(dz).reshape(T, ld)
    if not inplace:
        assert (got[:, V:] == 7.0).all()
    got = got[:, :V]
    row_bound, grad_bound = distill_bounds(ref, host, w, dtype, scale)
    limit = 448.0 if dtype == "f8" else np.inf
    want = np.clip(ref["dlogits"], -limit, limit)
    inf = np.isinf(ref["row_loss"])
    assert np.array_equal(rows[inf], ref["row_loss"][inf])
    assert (np.abs(rows - ref["row_loss"])[~inf] <= row_bound[~inf]).all()
    if not inf.any():
        w64 = np.asarray(w, np.float64)
        assert abs(loss - ref["loss"]) <= (np.abs(w64) * row_bound).sum() + 2.0 ** -22 * (np.abs(w64 * ref["row_loss"])).sum()
    assert (np.abs(got - want) <= grad_bound).all()
    quiet = (np.asarray(w) == 0) | ref["bad"]
    assert not got[quiet].any() and not np.signbit(got[quiet]).any()
    return loss, rows, got


SCALE = {"f32": 1.0, "bf16": 1.0, "f16": 4096.0, "f8": 512.0}


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "f8"])
@pytest.mark.parametrize("T,V,K,ld,off", [
    (1, 1, 1, 1, 0), (6, 7, 4, 9, 0), (6, 64, 64, 64, 1), (11, 1000, 3, 1000, 3), (9, 1024, 16, 1024, 0), (6, 2049, 256, 2053, 1),
    (7, 4103, 50, 4103, 0), (3, 17000, 128, 17000, 0), (3, 50257, 50, 50257, 0), (2, 70000, 64, 70016, 7), (2, 151936, 64, 151936, 0),
    (2, 200003, 20, 200003, 0)])
def test_distill(gh, dtype, tail, T, V, K, ld, off):
    check_distill(normal([T, V, K, 1], T, V), dtype, K, tail, ld, off, scale=SCALE[dtype], seed=V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [700, 3001, 20001, 50257])
def test_distill_in_place_and_at_other_offsets(gh, dtype, V):
    z = normal(V, 7, V)
    a = check_distill(z, dtype, 30, 1, seed=V)
    b = check_distill(z, dtype, 30, 1, seed=V, inplace=True)
    assert np.array_equal(a[1], b[1]) and np.array_equal(a[2], b[2])
    check_distill(z, dtype, 30, 1, seed=V, off=1, off_d=2)       # element by element
    check_distill(z, dtype, 30, 0, seed=V, off=3, off_d=0)


@pytest.mark.parametrize("V", [40, 999, 30011])
def test_distill_of_a_teacher_that_is_the_student(gh, V):
    """The lists come from the rows themselves (and from the library's own call): with the bucket nothing is left to learn."""
    T, K = 6, 24
    z, host = stored(normal(V, T, V), "f32")
    index, lp, _ = run_top(z, T, V, V, K)
    dz = sevens(T, V, "f32")
    w = np.ones(T, np.float32)
    loss, rows, err = run_distill(z, T, V, V, index, lp.astype(np.float32), w, 1, 1.0, dz)
    assert err == 0 and np.abs(rows).max() <= 8 * rel(V, 20.0)
    assert np.abs(wide(dz)).max() <= 8 * rel(V, 20.0)


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_of_a_sure_student(gh, tail):
    """Nearly no mass outside the list: the others' sum is formed by itself, not as what the list leaves of 1."""
    T, V, K = 4, 5000, 8
    z = normal(3, T, V, 1.0)
    index = np.stack([np.random.default_rng(t).permutation(V)[:K] for t in range(T)]).astype(np.int32)
    for t, up in enumerate((20.0, 40.0, 90.0, 200.0)):
        z[t, index[t]] += up
    lp = np.log(np.random.default_rng(1).dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32)
    check_distill(z, "f32", K, tail, w=np.ones(T, np.float32), lists=(index, lp))


@pytest.mark.parametrize("V", [64, 3000, 20000])
@pytest.mark.parametrize("tail", [0, 1])
def test_distill_of_masked_rows_and_odd_lists(gh, tail, V):
    T, K = 12, 20
    z = normal(V, T, V)
    index, lp = make_lists(V, z.astype(np.float64), K)
    w = np.ones(T, np.float32)
    lowest = float(np.finfo(np.float32).min)
    z[0] = -np.inf                       # an empty row
    z[1] = lowest
    keep = np.zeros(V, bool)
    keep[index[2]] = True
    z[2, ~keep] = -np.inf                # nothing but the list
    z[3, ~keep] = lowest
    z[4, index[4, 3]] = -np.inf          # teacher probability on a masked logit
    index[5] = -1                        # no list
    index[6, 1:] = -1                    # one entry
    index[7, 2] = V                      # not an id
    index[8, 4] = index[8, 9]            # twice
    lp[9, 5:] = -np.inf                  # listed with probability 0
    lp[10] = -np.inf
    lp[11] = np.log(1.0 / K) + 1e-3      # sums to more than 1
    check_distill(z, "f32", K, tail, w=w, lists=(index, lp))


def test_distill_propagates_nan_rows(gh):
    T, V, K = 4, 900, 5
    z = normal(1, T, V)
    index, lp = make_lists(1, z.astype(np.float64), K)
    z[1, 13] = np.nan
    z[2, index[2, 0]] = np.inf
    z[3, index[3, 1]] = np.nan
    d, _ = stored(z, "f32")
    dz = sevens(T, V, "f32")
    loss, rows, _ = run_distill(d, T, V, V, index, lp, np.ones(T, np.float32), 1, 1.0, dz)
    got = wide(dz).reshape(T, V)
    assert np.isnan(loss) and np.isfinite(rows[0]) and np.isnan(rows[1:]).all()
    assert np.isfinite(got[0]).all() and np.isnan(got[1:]).all()


@pytest.mark.parametrize("tail", [0, 1])
def test_distill_gradient_by_differences_of_its_loss(gh, tail):
    """Central differences of the call's own row losses (fp32): h = 1/64 leaves h^2/6 of a third derivative below 1 and
    2 x 2^-22 / 2h of rounding."""
    V, K, h = 37, 6, 1.0 / 64
    base = np.round(normal(2, 1, V, 1.0) * 256) / 256
    index, lp = make_lists(2, base.astype(np.float64), K)
    both = np.concatenate([np.repeat(base, V, 0) + h * np.eye(V), np.repeat(base, V, 0) - h * np.eye(V), base]).astype(np.float32)
    T = 2 * V + 1
    z, _ = stored(both, "f32")
    dz = sevens(T, V, "f32")
    _, rows, _ = run_distill(z, T, V, V, np.repeat(index, T, 0), np.repeat(lp, T, 0), np.ones(T, np.float32), tail, 1.0, dz)
    diff = (rows[:V] - rows[V:2 * V]) / (2 * h)
    assert np.abs(diff - wide(dz).reshape(T, V)[-1]).max() <= h * h / 6 + 2.0 ** -22 / h * (1 + np.abs(rows).max())


def test_distill_without_gradient_or_rows(gh):
    T, V, K = 9, 6000, 12
    z, host = stored(normal(8, T, V), "bf16")
    index, lp = make_lists(8, host, K)
    w = np.random.default_rng(8).uniform(size=T).astype(np.float32)
    dz = sevens(T, V, "bf16")
    full = run_distill(z, T, V, V, index, lp, w, 1, 1.0, dz)
    alone = run_distill(z, T, V, V, index, lp, w, 1, 1.0, None, row_loss=False)
    assert full[0] == alone[0]
    empty = run_distill(z, 0, V, V, index[:0], lp[:0], w[:0], 1, 1.0, dz)
    assert empty[0] == 0.0


def test_distill_weights_of_either_sign_and_many_rows(gh):
    T, V, K = 700, 257, 9
    w = np.random.default_rng(3).normal(size=T).astype(np.float32)
    check_distill(normal(3, T, V), "bf16", K, 1, ld=260, w=w)


# ------------------------------------------------------------------------------------------------ verification
def draft_case(seed, B, G, V, dtype, probs, ld=None, miss=0.7):
    """Random rows, drafted tokens from the drafter, random numbers; decisions that fp32 and fp64 could take differently are
    moved apart."""
    rng = np.random.default_rng([seed, B, G, V])
    zt = rng.normal(0, 2.0, size=(B * (G + 1), V)).astype(np.float32)
    zd = np.concatenate([zt.reshape(B, G + 1, V)[b, :G] for b in range(B)] or [np.zeros((0, V))]).astype(np.float32)
    zd = zd + rng.normal(0, miss, size=zd.shape).astype(np.float32)
    tokens = np.zeros((B, G), np.int32)
    for b in range(B):
        for i in range(G):
            if probs or rng.random() < 0.5:
                p = np.exp(orc.log_softmax(zd[b * G + i]))
                tokens[b, i] = rng.choice(V, p=p / p.sum())
            else:
                tokens[b, i] = np.argmax(zt[b * (G + 1) + i])
                zt[b * (G + 1) + i, tokens[b, i]] += 4.0
    t_dev, t_host = stored(zt, dtype, ld)
    d_dev, d_host = stored(zd, dtype, ld) if probs and G else (None, None)
    u = rng.random((B, G)).astype(np.float32)
    noise = np.maximum(rng.exponential(size=(B, V)), 1e-6).astype(np.float32)
    t_host = t_host.reshape(B, G + 1, V)
    d_host = d_host.reshape(B, G, V) if d_host is not None else None
    return dict(t=t_dev, d=d_dev, th=t_host, dh=d_host, tokens=tokens, u=u, noise=noise)


def part_decisions(case, V, count):
    for _ in range(20):
        ref = orc.verify(case["th"], case["dh"], V, case["tokens"], count, case["u"], case["noise"])
        if ref["margin"] > 1e-4:
            return ref
        for b in range(len(case["u"])):
            one = orc.verify(case["th"][b:b + 1], None if case["dh"] is None else case["dh"][b:b + 1], V, case["tokens"][b:b + 1],
                             None if count is None else count[b:b + 1], case["u"][b:b + 1], case["noise"][b:b + 1])
            if one["margin"] <= 1e-4:
                case["u"][b] *= np.float32(0.97)
                j = one["tokens"][0, one["accepted"][0]]
                case["noise"][b, j] *= np.float32(0.9)
    raise AssertionError("decisions too close")


def run_verify(case, B, G, V, ld, count, want_logprob=True):
    import paper_2602_14338_amd as aero
    up = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).to("cuda")
    accepted = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    out = torch.full((B, G + 1), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((B, G + 1), 7.0, device="cuda") if want_logprob else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    aero.aero_verify_draft(case["t"], case["d"], B, G, V, ld, up(case["tokens"], np.int32) if G else None,
                           None if count is None else up(count, np.int32), up(case["u"], np.float32) if G else None,
                           up(case["noise"], np.float32), accepted, out, lp, workspace("OP_VERIFY_DRAFT", T=B * (G + 1), V=V, Q=B), err)
    torch.cuda.synchronize()
    return accepted.cpu().numpy(), out.cpu().numpy(), None if lp is None else lp.cpu().numpy().astype(np.float64), int(err.item())


def check_verify(case, B, G, V, ld, count, err=0):
    ref = part_decisions(case, V, count)
    accepted, out, lp, got_err = run_verify(case, B, G, V, ld, count)
    assert np.array_equal(accepted, ref["accepted"]) and np.array_equal(out, ref["tokens"]) and got_err == err
    assert (np.abs(lp - ref["logprob"]) <= rel(V, 16.0) + 2.0 ** -23 * np.abs(ref["logprob"])).all()
    return ref


@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "f8"])
@pytest.mark.parametrize("B,G,V,ld", [(1, 1, 2, 2), (1, 0, 700, 700), (3, 4, 7, 9), (5, 3, 1000, 1003), (70, 2, 300, 304), (4, 63, 150, 150),
                                      (2, 5, 50257, 50257), (9, 4, 8192, 8192), (1, 2, 151936, 151936)])
def test_verify(gh, dtype, probs, B, G, V, ld):
    case = draft_case(1, B, G, V, dtype, probs, ld)
    ref = check_verify(case, B, G, V, ld, None)
    if B == 70:
        assert len(set(ref["accepted"].tolist())) == G + 1     # every place of the first refusal, and none


@pytest.mark.parametrize("probs", [True, False])
def test_verify_ragged_idle_and_bad_sequences(gh, probs):
    B, G, V = 40, 5, 999
    case = draft_case(2, B, G, V, "bf16", probs)
    count = np.random.default_rng(2).integers(0, G + 1, size=B).astype(np.int32)
    count[3] = -1
    count[4] = G + 1
    case["tokens"][5, 1] = -4
    case["tokens"][6, 0] = V
    count[5] = count[6] = G
    ref = part_decisions(case, V, count)
    check_verify(case, B, G, V, V, count, err=2 | 16)
    assert (ref["tokens"][3] == -1).all() and (ref["tokens"][4] == -1).all()


def test_verify_of_a_drafter_that_is_the_policy(gh):
    """The same rows on both sides: everything is accepted, and with all uniform numbers 0 in any case."""
    B, G, V = 6, 4, 3000
    case = draft_case(3, B, G, V, "f32", True, miss=0.0)
    case["u"][:] = np.minimum(case["u"], 0.999)
    accepted, out, _, _ = run_verify(case, B, G, V, V, None)
    assert (accepted == G).all() and np.array_equal(out[:, :G], case["tokens"])


def test_verify_of_masked_rows(gh):
    """Rows cut to a few logits, empty rows and rows with NaN, on either side."""
    B, G, V = 9, 2, 400
    case = draft_case(4, B, G, V, "f32", True)
    zt, zd = case["th"].copy(), case["dh"].copy()
    zt[0, 0, 10:] = -np.inf
    zt[1, 0] = -np.inf                    # an empty target row: nothing accepted, nothing drawn
    zt[2, 0, 5] = np.nan
    zt[3, 0, ::2] = np.finfo(np.float32).min
    zd[4, 0] = -np.inf                    # an empty draft row: refused, drawn from p
    zd[5, 0, 3] = np.nan
    zd[6, 0, 10:] = -np.inf
    case["tokens"][6, 0] = 50             # the drafter gives it nothing, the policy something: accepted
    zt[7, 0, :] = -np.inf
    zt[7, 0, 9] = 1.0                     # one choice, not the drafted token
    case["tokens"][7, 0] = 8
    zt[8, 1] = -np.inf
    case["u"][8, 0] = 0.0
    case["t"], case["th"] = stored(zt.reshape(-1, V), "f32")[0], zt.astype(np.float64)
    case["d"], case["dh"] = stored(zd.reshape(-1, V), "f32")[0], zd.astype(np.float64)
    ref = check_verify(case, B, G, V, V, None)
    assert ref["tokens"][1, 0] == -1 and ref["accepted"][6] >= 1 and ref["tokens"][7, 0] == 9 and ref["tokens"][8, 1] == -1


def test_verify_without_logprob_and_of_no_sequences(gh):
    import paper_2602_14338_amd as aero
    case = draft_case(6, 3, 2, 500, "bf16", True)
    ref = part_decisions(case, 500, None)
    accepted, out, _, _ = run_verify(case, 3, 2, 500, 500, None, want_logprob=False)
    assert np.array_equal(out, ref["tokens"]) and np.array_equal(accepted, ref["accepted"])
    e = torch.empty(0, device="cuda")
    i = torch.empty(0, dtype=torch.int32, device="cuda")
    aero.aero_verify_draft(case["t"], case["d"], 0, 2, 500, 500, i, None, e, e, i, i, e, workspace("OP_VERIFY_DRAFT", T=0, V=500, Q=0))


# ------------------------------------------------------------------------------------------------ embedding
def token_ids(seed, T, V):
    """Ids whose frequency falls as 1 / rank, some padding."""
    rng = np.random.default_rng([seed, T, V])
    rank = np.minimum((V ** rng.random(T)).astype(np.int64), V) - 1
    ids = rng.permutation(V)[np.clip(rank, 0, V - 1)]
    ids[rng.random(T) < 0.1] = -1
    return ids.astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,V,H,ld,off", [(1, 1, 1, 1, 0), (5, 7, 3, 5, 1), (33, 100, 64, 64, 0), (40, 1000, 257, 257, 0), (17, 500, 128, 272, 0),
                                          (300, 5000, 1536, 1536, 0), (3, 20, 5000, 5000, 3)])
def test_embedding(gh, dtype, T, V, H, ld, off):
    import paper_2602_14338_amd as aero
    table, host = stored(normal([T, V, H], V, H, 0.05), dtype)
    ids = token_ids(1, T, V)
    if T > 4:
        ids[3] = V
    out = sevens(T, ld, dtype, off)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    aero.aero_embedding_fwd(table, V, H, torch.from_numpy(ids).to("cuda"), T, float(np.sqrt(H)), out, ld, err)
    torch.cuda.synchronize()
    got = wide(out).reshape(T, ld)
    want = orc.embedding(host, ids, float(np.float32(np.sqrt(H))))
    assert int(err.item()) == (2 if T > 4 else 0) and (got[:, H:] == 7.0).all()
    assert (np.abs(got[:, :H] - want) <= (HALF_ULP[dtype] + 2.0 ** -24) * np.abs(want) + HALF_LEAST[dtype]).all()
    assert not got[(ids < 0) | (ids >= V), :H].any()


def run_embed_bwd(dout, T, H, ld, ids, V, scale, grad, accumulate):
    import paper_2602_14338_amd as aero
    table = sevens(V, H, grad)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    aero.aero_embedding_bwd(dout, T, H, ld, torch.from_numpy(ids).to("cuda"), V, scale, table, workspace("OP_EMBEDDING_BWD", T=T, V=V, H=H),
                            accumulate, err)
    torch.cuda.synchronize()
    return table, int(err.item())


def check_embed_bwd(T, V, H, ld, dtype, grad, accumulate, ids, off=0, err=0):
    dout, host = stored(normal([T, V, H], T, H, 1.0), dtype, ld, off)
    table, got_err = run_embed_bwd(dout, T, H, ld, ids, V, 0.75, grad, accumulate)
    want, size = orc.embedding_grad(host, ids, V, 0.75)
    n = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    base = 7.0 if accumulate else 0.0
    bound = 2.0 ** -24 * (n + 2) * (size + base) + HALF_ULP[grad] * np.abs(base + want) + HALF_LEAST[grad]
    got = wide(table).reshape(V, H)
    assert got_err == err and (np.abs(got - (base + want)) <= bound).all()
    assert (got[n[:, 0] == 0] == base).all()
    again, _ = run_embed_bwd(dout, T, H, ld, ids, V, 0.75, grad, accumulate)
    raw = {2: torch.int16, 4: torch.int32}[again.element_size()]
    assert torch.equal(table.view(raw), again.view(raw))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,grad", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("T,V,H,ld,off", [(1, 1, 1, 1, 0), (7, 3, 5, 9, 1), (64, 1000, 64, 64, 0), (700, 300, 257, 257, 0), (999, 5000, 72, 80, 0),
                                          (3000, 2000, 512, 512, 0), (40, 300, 1537, 1540, 0)])
def test_embedding_gradient(gh, T, V, H, ld, off, dtype, grad, accumulate):
    check_embed_bwd(T, V, H, ld, dtype, grad, accumulate, token_ids(2, T, V), off)


@pytest.mark.parametrize("ids_of", ["one", "padding", "two", "all", "bad", "runs"])
def test_embedding_gradient_of_uneven_tokens(gh, ids_of):
    """One id for thousands of tokens, none at all, every id once, ids outside the table, runs that end at the pieces' ends."""
    T, V, H = 9000, 3000, 40
    t = np.arange(T)
    ids = {"one": np.full(T, 1234), "padding": np.full(T, -1), "two": np.where(t % 3 == 0, 5, 5 + 256), "all": t % V,
           "bad": np.where(t % 2 == 0, V + t, t % 100), "runs": np.repeat(np.arange(T // 32 + 1), 32)[:T]}[ids_of].astype(np.int32)
    for accumulate in (False, True):
        check_embed_bwd(T, V, H, H, "bf16", "f32", accumulate, ids, err=2 if ids_of == "bad" else 0)


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,H,off", [(1, 1, 1, 1), (9, 700, 3, 3), (30, 400, 24, 1), (64, 300, 257, 5), (5, 1000, 8, 0), (300, 40, 1001, 2)])
def test_embedding_gradient_within_its_table(gh, T, V, H, off, grad):
    """A table at any element of a buffer: the same bits as elsewhere, and nothing outside it is written."""
    import paper_2602_14338_amd as aero
    dout, _ = stored(normal([T, V, H], T, H, 1.0), "bf16")
    ids = token_ids(4, T, V)
    want, _ = run_embed_bwd(dout, T, H, H, ids, V, 0.75, grad, False)
    buf = sevens(1, off + V * H + 64, grad).reshape(-1)
    table = buf[off:off + V * H].reshape(V, H)
    aero.aero_embedding_bwd(dout, T, H, H, torch.from_numpy(ids).to("cuda"), V, 0.75, table, workspace("OP_EMBEDDING_BWD", T=T, V=V, H=H))
    torch.cuda.synchronize()
    raw = {2: torch.int16, 4: torch.int32}[table.element_size()]
    assert torch.equal(table.view(raw), want.reshape(V, H).view(raw))
    assert bool((buf[:off] == 7.0).all()) and bool((buf[off + V * H:] == 7.0).all())


@pytest.mark.parametrize("H", [1, 3, 40, 1001])
@pytest.mark.parametrize("T", [2, 64, 65, 256, 257, 512, 513])
def test_embedding_gradient_of_few_tokens(gh, T, H):
    """Around as many tokens as need no sort: ids that meet across the waves of a workgroup, all the same, none, outside the table."""
    V = 700
    t = np.arange(T)
    for kind, ids in enumerate((np.full(T, 699), t % 2 * 64, t * 5 % V, np.where(t % 3 == 0, V + t, t % 7), np.full(T, -1), t // 2)):
        check_embed_bwd(T, V, H, H, "bf16", "f32" if kind % 2 else "bf16", kind % 3 == 0, ids.astype(np.int32), err=2 if kind == 3 else 0)


def test_embedding_gradient_of_large_tables(gh):
    """More ids than 256 workgroups count, and lengths around a workgroup's step."""
    for T, V in ((4096, 300000), (4097, 262145), (8191, 151936)):
        check_embed_bwd(T, V, 8, 8, "bf16", "f32", False, token_ids(3, T, V))


@pytest.mark.parametrize("T", [40, 300])
def test_embedding_gradient_of_a_table_past_32_bits(gh, T):
    """Elements and bytes past 2^32, and more zeros than one launch writes; rows looked up from it at the same places."""
    import paper_2602_14338_amd as aero
    V, H = 1 << 24, 513
    ids = np.random.default_rng(5).integers(0, V, T).astype(np.int32)
    ids[:4] = (0, V - 1, V - 2, V // 2)
    dout, host = stored(normal([T, H], T, H, 1.0), "f32")
    table = torch.full((V, H), 7.0, device="cuda")
    dev = torch.from_numpy(ids).to("cuda")
    aero.aero_embedding_bwd(dout, T, H, H, dev, V, 0.5, table, workspace("OP_EMBEDDING_BWD", T=T, V=V, H=H))
    out = torch.empty((T, H), device="cuda")
    aero.aero_embedding_fwd(table, V, H, dev, T, 2.0, out, H)
    torch.cuda.synchronize()
    assert len(set(ids.tolist())) == T and np.array_equal(wide(out).reshape(T, H), host.reshape(T, H))
    total = sum(int(table[v:v + (1 << 20)].count_nonzero()) for v in range(0, V, 1 << 20))
    assert total == np.count_nonzero(host)


def test_embedding_gradient_without_tokens(gh):
    import paper_2602_14338_amd as aero
    table = sevens(50, 24, "f32")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    aero.aero_embedding_bwd(torch.empty(0, dtype=torch.bfloat16, device="cuda"), 0, 24, 24, none, 50, 1.0, table,
                            workspace("OP_EMBEDDING_BWD", T=0, V=50, H=24))
    assert not wide(table).any()


# ------------------------------------------------------------------------------------------------ all of them
def test_calls_in_a_graph_and_on_another_stream(gh):
    """Recorded once and replayed with other work between; then on a stream of the caller's.  The same bits each time."""
    import paper_2602_14338_amd as aero
    T, V, K, H, B, G = 300, 5003, 32, 96, 12, 3
    z, host = stored(normal(1, T, V), "bf16")
    teacher, _ = stored(normal(2, T, V), "bf16")
    case = draft_case(9, B, G, V, "bf16", True)
    up = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).to("cuda")
    tokens, u, noise = up(case["tokens"], np.int32), up(case["u"], np.float32), up(case["noise"], np.float32)
    w, ids = torch.full((T,), 1.0 / T, device="cuda"), up(token_ids(4, T, V), np.int32)
    table = torch.from_numpy(normal(3, V, H, 0.02)).to("cuda").bfloat16()
    bufs = {}

    def call():
        aero.aero_topk_logprob(teacher, T, V, V, None, K, bufs["index"], bufs["lp"], bufs["lse"], bufs["ws1"])
        aero.aero_distill_loss_bwd(z, T, V, V, bufs["index"], bufs["lp"], K, w, 1, 1.0, bufs["loss"], bufs["rows"], bufs["dz"], bufs["ws2"])
        aero.aero_verify_draft(case["t"], case["d"], B, G, V, V, tokens, None, u, noise, bufs["accepted"], bufs["out"], bufs["olp"], bufs["ws3"])
        aero.aero_embedding_fwd(table, V, H, ids, T, 2.0, bufs["emb"], H)
        aero.aero_embedding_bwd(bufs["emb"], T, H, H, ids, V, 2.0, bufs["demb"], bufs["ws4"])

    def fresh():
        f = lambda *s: torch.full(s, 7.0, device="cuda")
        i = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")
        bufs.update(index=i(T, K), lp=f(T, K), lse=f(T), loss=f(1), rows=f(T), dz=sevens(T, V, "bf16"), accepted=i(B), out=i(B, G + 1),
                    olp=f(B, G + 1), emb=sevens(T, H, "bf16"), demb=f(V, H), ws1=workspace("OP_TOPK_LOGPROB", T=T, V=V, H=K),
                    ws2=workspace("OP_DISTILL_LOSS_BWD", T=T, V=V), ws3=workspace("OP_VERIFY_DRAFT", T=B * (G + 1), V=V, Q=B),
                    ws4=workspace("OP_EMBEDDING_BWD", T=T, V=V, H=H))

    outs = ["index", "lp", "lse", "loss", "rows", "dz", "accepted", "out", "olp", "emb", "demb"]
    raw = lambda t: t.view({2: torch.int16, 4: torch.int32}[t.element_size()])
    fresh()
    call()
    torch.cuda.synchronize()
    want = {k: raw(bufs[k]).clone() for k in outs}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        for k in outs:
            raw(bufs[k]).fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        for k in outs:
            assert torch.equal(raw(bufs[k]), want[k]), k
        junk = torch.randn(1 << 22, device="cuda").sum().item()
        assert junk == junk
    fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    for k in outs:
        assert torch.equal(raw(bufs[k]), want[k]), k


def test_refusals(gh):
    import paper_2602_14338_amd as aero
    f = lambda *s: torch.zeros(s, device="cuda")
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    z, zh = f(4, 16), f(4, 16).half()

    def refused(match, fn, *args, **kw):
        with pytest.raises(aero.AeroError, match=match):
            fn(*args, **kw)

    top = aero.aero_topk_logprob
    refused("capacity", top, z, 4, 16, 16, None, 257, i(4, 257), f(4, 257), None, ws)
    refused("size", top, z, 4, 16, 15, None, 4, i(4, 4), f(4, 4), None, ws)
    refused("size", top, z, 4, 0, 16, None, 4, i(4, 4), f(4, 4), None, ws)
    refused("size", top, z, -1, 16, 16, None, 4, i(4, 4), f(4, 4), None, ws)
    refused("size", top, z, 4, 16, 16, None, 0, i(4, 4), f(4, 4), None, ws)
    refused("NULL", top, z, 4, 16, 16, None, 4, None, f(4, 4), None, ws)
    refused("workspace", top, z, 4, 16, 16, None, 4, i(4, 4), f(4, 4), None, None)
    refused("workspace", top, z, 4, 16, 16, None, 4, i(4, 4), f(4, 4), None, ws[:64])
    refused("workspace", top, z, 4, 16, 16, None, 4, i(4, 4), f(4, 4), None, ws[16:])
    refused("dtype", top, z.double(), 4, 16, 16, None, 4, i(4, 4), f(4, 4), None, ws)
    refused("dtype", top, z, 4, 16, 16, None, 4, f(4, 4), f(4, 4), None, ws)
    refused("GPU", top, z.cpu(), 4, 16, 16, None, 4, i(4, 4), f(4, 4), None, ws)
    refused("contiguous", top, z[:, ::2], 4, 8, 8, None, 4, i(4, 4), f(4, 4), None, ws)

    dis = aero.aero_distill_loss_bwd
    refused("capacity", dis, z, 4, 16, 16, i(4, 300), f(4, 300), 300, f(4), 0, 1.0, f(1), None, None, ws)
    refused("size", dis, z, 4, 16, 15, i(4, 3), f(4, 3), 3, f(4), 0, 1.0, f(1), None, None, ws)
    refused("size", dis, z, 4, 16, 16, i(4, 3), f(4, 3), 3, f(4), 2, 1.0, f(1), None, None, ws)
    refused("size", dis, z, 4, 16, 16, i(4, 3), f(4, 3), 3, f(4), 0, float("nan"), f(1), None, None, ws)
    refused("NULL", dis, z, 4, 16, 16, i(4, 3), f(4, 3), 3, f(4), 0, 1.0, None, None, None, ws)
    refused("NULL", dis, z, 4, 16, 16, i(4, 3), None, 3, f(4), 0, 1.0, f(1), None, None, ws)
    refused("dlogits", dis, z, 4, 16, 16, i(4, 3), f(4, 3), 3, f(4), 0, 1.0, f(1), None, zh, ws)
    refused("workspace", dis, z, 4, 16, 16, i(4, 3), f(4, 3), 3, f(4), 0, 1.0, f(1), None, None, ws[:100])

    ver = aero.aero_verify_draft
    big = f(70, 16)
    args = (i(1, 3), None, f(1, 3), f(1, 16), i(1), i(1, 4), f(1, 4))
    refused("capacity", ver, big, None, 1, 64, 16, 16, i(1, 64), None, f(1, 64), f(1, 16), i(1), i(1, 65), None, ws)
    refused("size", ver, z, None, 1, 3, 16, 15, *args, ws)
    refused("size", ver, z, None, 1, -1, 16, 16, *args, ws)
    refused("draft_logits", ver, z, zh, 1, 3, 16, 16, *args, ws)
    refused("NULL", ver, z, None, 1, 3, 16, 16, None, *args[1:], ws)
    refused("workspace", ver, z, None, 1, 3, 16, 16, *args, ws[:100])

    fwd, bwd = aero.aero_embedding_fwd, aero.aero_embedding_bwd
    refused("size", fwd, z, 4, 16, i(2), 2, 1.0, f(2, 16), 15)
    refused("size", fwd, z, 4, 0, i(2), 2, 1.0, f(2, 16), 16)
    refused("out", fwd, z, 4, 16, i(2), 2, 1.0, zh, 16)
    refused("NULL", fwd, z, 4, 16, None, 2, 1.0, f(2, 16), 16)
    refused("dtype", fwd, z.to(torch.float8_e4m3fn), 4, 16, i(2), 2, 1.0, z.to(torch.float8_e4m3fn), 16)
    refused("size", bwd, z, 4, 16, 15, i(4), 9, 1.0, f(9, 16), ws)
    refused("dtype", bwd, z, 4, 16, 16, i(4), 9, 1.0, f(9, 16).half(), ws)
    refused("NULL", bwd, z, 4, 16, 16, None, 9, 1.0, f(9, 16), ws)
    refused("workspace", bwd, z, 4, 16, 16, i(4), 9, 1.0, f(9, 16), ws[:100])


@pytest.mark.parametrize("dtype,V,ld,K,tail", [("bf16", 66001, 66001, 40, 1), ("f32", 33003, 33004, 70, 0), ("f8", 140001, 140003, 20, 1)])
def test_distill_of_more_long_rows_than_compute_units(gh, dtype, V, ld, K, tail):
    """Several rows per workgroup of the streaming kernel, each at another offset from 16 bytes, with rows of weight 0, bad lists and
    empty rows among them; checked on some of them."""
    import paper_2602_14338_amd as aero
    T = 600
    rng = np.random.default_rng(V)
    base = normal([V, 3], 40, V)
    pick = rng.integers(0, 40, size=T)
    shift = rng.integers(1, V, size=T)
    z = np.stack([np.roll(base[p], s) for p, s in zip(pick, shift)])
    if dtype != "f8":   # which has no infinities
        z[7] = -np.inf
    dev, host = stored(z, dtype, ld, 3)
    index = np.zeros((T, K), np.int32)
    lp = np.zeros((T, K), np.float32)
    lists = [make_lists(k, host[np.flatnonzero(pick == k)[:1]], K) if (pick == k).any() else None for k in range(40)]
    for t in range(T):
        first = np.flatnonzero(pick == pick[t])[0]
        index[t] = (lists[pick[t]][0][0] - shift[first] + shift[t]) % V
        lp[t] = lists[pick[t]][1][0]
    index[7] = np.arange(K)
    index[11, 3] = index[11, 5]
    index[300, 0] = V
    index[400, : K // 2] = -1
    w = rng.uniform(0.2, 1.0, size=T).astype(np.float32)
    w[rng.random(T) < 0.2] = 0.0
    w[[7, 11, 300, 400]] = 0.5
    some = np.unique(np.concatenate([[0, 7, 11, 299, 300, 301, 400, 599], rng.integers(0, T, size=24)]))
    ref = orc.distill(host[some], V, index[some], lp[some], w[some], tail, SCALE[dtype])
    dz = sevens(T, ld, dtype, 3)
    loss, rows, err = run_distill(dev, T, V, ld, index, lp, w, tail, SCALE[dtype], dz)
    assert err == 8 and abs(loss - (rows * w).sum()) <= 2.0 ** -20 * (np.abs(rows * w)).sum()
    got = wide(dz.view(T, ld)[torch.from_numpy(some).to("cuda")] if dtype != "f8" else
               dz.view(torch.uint8).view(T, ld)[torch.from_numpy(some).to("cuda")].view(torch.float8_e4m3fn))
    assert (got[:, V:] == 7.0).all()
    row_bound, grad_bound = distill_bounds(ref, host[some], w[some], dtype, SCALE[dtype])
    assert (np.abs(rows[some] - ref["row_loss"]) <= row_bound).all()
    assert (np.abs(got[:, :V] - ref["dlogits"]) <= grad_bound).all()
    assert not rows[w == 0].any()
    again = sevens(T, ld, dtype, 3)
    run_distill(dev, T, V, ld, index, lp, w, tail, SCALE[dtype], again)
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[again.element_size()]
    assert torch.equal(dz.view(raw), again.view(raw))


@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("dtype,V,ld", [("bf16", 300, 301), ("f32", 997, 997)])
def test_verify_of_many_sequences(gh, dtype, V, ld, probs):
    """Enough positions for the way that decides them one by one, with ragged counts, idle and bad sequences."""
    B, G = 420, 3
    case = draft_case(11, B, G, V, dtype, probs, ld)
    count = np.random.default_rng(3).integers(0, G + 1, size=B).astype(np.int32)
    count[:200] = G
    count[201], count[202] = -1, G + 5
    case["tokens"][7, 1], case["tokens"][8, 0] = -1, V + 3
    zt = case["th"].copy()
    zt[20, 0] = -np.inf
    zt[21, 1] = np.nan
    if dtype == "f32":
        case["t"], case["th"] = stored(zt.reshape(-1, V), dtype, ld)[0], zt
    ref = check_verify(case, B, G, V, ld, count, err=2 | 16)
    assert len(set(ref["accepted"].tolist())) == G + 1
    check_verify(draft_case(12, 1100, 0, 40, dtype, probs), 1100, 0, 40, 40, None)      # nothing drafted, one slice


@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("dtype,B,G,V", [("bf16", 40, 5, 20001), ("f32", 260, 3, 12001), ("bf16", 260, 3, 23001), ("f32", 9, 2, 9001)])
def test_verify_of_longer_rows(gh, dtype, B, G, V, probs):
    """Rows too long for one launch, of few sequences and of many: ragged counts, idle and bad sequences, masked, empty and NaN rows."""
    case = draft_case(13, B, G, V, dtype, probs)
    count = np.random.default_rng(13).integers(0, G + 1, size=B).astype(np.int32)
    count[3], count[4], count[5:9] = -1, G + 1, G
    case["tokens"][5, 1] = -4
    case["tokens"][6, 0] = V
    zt = np.asarray(case["th"], np.float32).reshape(B, G + 1, V).copy()
    zt[7, 0, ::3] = -np.inf
    zt[8, 0] = -np.inf
    zt[0, 0, V - 1] = np.nan
    zt[1, 0, :V - 2] = np.finfo(np.float32).min if dtype == "f32" else -3.0e38
    case["t"], host = stored(zt.reshape(-1, V), dtype)
    case["th"] = host.reshape(B, G + 1, V)
    if probs:
        zd = np.asarray(case["dh"], np.float32).reshape(B, G, V).copy()
        zd[2, 0] = -np.inf
        case["d"], host = stored(zd.reshape(-1, V), dtype)
        case["dh"] = host.reshape(B, G, V)
    ref = check_verify(case, B, G, V, V, count, err=2 | 16)
    assert ref["tokens"][0, 0] == -1 and ref["tokens"][8, 0] == -1 and ref["tokens"][1, 0] >= V - 2


def test_verify_of_equal_rows_that_are_refused(gh):
    """Where the residual vanishes the token is drawn from p: the drafter's rows are the policy's and the drafted token is masked in both,
    so that it is refused; with one slice per sequence and with several."""
    for B, V in ((3, 20000), (300, 600)):
        case = draft_case(13, B, 1, V, "f32", True, miss=0.0)
        z = case["th"].copy()
        z[:, 0, 5] = -np.inf
        case["t"], case["th"] = stored(z.reshape(-1, V), "f32")[0], z
        zd = z[:, :1].copy()
        case["d"], case["dh"] = stored(zd.reshape(-1, V), "f32")[0], zd
        case["tokens"][:] = 5
        ref = check_verify(case, B, 1, V, V, None)
        assert not ref["accepted"].any() and (ref["tokens"][:, 0] >= 0).all() and (ref["tokens"][:, 0] != 5).all()


@pytest.mark.parametrize("dtype,V,off_d", [("bf16", 90001, None), ("f32", 41003, None), ("f32", 100003, None), ("bf16", 9001, 1)])
def test_distill_of_few_long_rows(gh, dtype, V, off_d):
    """Rows that are split over workgroups: with and without a gradient, in place, with quiet rows among them."""
    T, K = 7, 60
    z = normal([V, 8], T, V)
    host = torch.from_numpy(z).to(TORCH[dtype]).float().double().numpy()
    index, lp = make_lists(V, host, K)
    index[4, 7] = index[4, 50]
    index[5] = -1
    for tail in (0, 1):
        a = check_distill(z, dtype, K, tail, off=3, off_d=off_d if off_d is None else off_d, lists=(index, lp))
        if off_d is None:
            b = check_distill(z, dtype, K, tail, off=3, lists=(index, lp), inplace=True)
            assert np.array_equal(a[1], b[1]) and np.array_equal(a[2], b[2])
        d, _ = stored(z, dtype, V, 3)
        w = np.random.default_rng([0, 6]).uniform(0.2, 1.0, size=T).astype(np.float32)
        w[::5] = 0.0
        alone = run_distill(d, T, V, V, index, lp, w, tail, 1.0, None)
        assert np.allclose(alone[1], a[1], rtol=0, atol=4 * rel(V, 16.0))
