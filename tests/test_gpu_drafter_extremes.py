"""The calls around a drafter on logits that masks and other callers write: finite masks, logits far from 0, probabilities that vanish.
Helpers, checks and tolerances are those of test_gpu_drafter."""
import numpy as np
import pytest
import torch

from oracle import drafter_oracle as orc
from test_gpu_drafter import (TORCH, check_distill, check_top, check_verify, distill_bounds, draft_case, gh, make_lists, normal,  # noqa: F401
                              rel, run_distill, run_top, sevens, stored, wide)

pytestmark = pytest.mark.gpu

LOWEST = {"f32": float(torch.finfo(torch.float32).min), "bf16": float(torch.finfo(torch.bfloat16).min)}

# sequences, drafted tokens and logits for which verification takes one launch, decides by sequence, and decides by position
FORMS = [(12, 2, 500), (12, 2, 7001), (16, 63, 1100)]


def parts(case, B, G, V):
    zt = np.asarray(case["th"], np.float32).reshape(B, G + 1, V).copy()
    return zt, None if case["dh"] is None else np.asarray(case["dh"], np.float32).reshape(B, G, V).copy()


def put(case, zt, zd, dtype):
    V = zt.shape[2]
    case["t"], host = stored(zt.reshape(-1, V), dtype)
    case["th"] = host.reshape(zt.shape)
    if zd is not None:
        case["d"], host = stored(zd.reshape(-1, V), dtype)
        case["dh"] = host.reshape(zd.shape)


@pytest.mark.parametrize("uniform", [1e-30, 0.25])
@pytest.mark.parametrize("mask", ["lowest", -1e30, -np.inf])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,G,V", FORMS)
def test_verify_decides_on_masks(gh, B, G, V, dtype, probs, mask, uniform):   # noqa: F811
    """A masked token has probability 0 whatever it is masked with: it is refused where the policy's row masks it (u 0 < 0 is false), also
    where the drafter's does so, and accepted where only the drafter's does; an empty row of the policy accepts nothing."""
    mask = LOWEST[dtype] if mask == "lowest" else mask
    case = draft_case(21, B, G, V, dtype, probs)
    zt, zd = parts(case, B, G, V)
    x = case["tokens"][:, 0]
    for b in range(B):
        zt[b, 0, x[b]] += 2.0   # sequences of their own otherwise
    for b in range(6):
        zt[b, 0, x[b]] = mask
    zt[1, 0] = mask                                     # an empty row
    zt[2, 0] = np.where(np.arange(V) % 3 == 0, -np.inf, np.where(np.arange(V) % 3 == 1, -1e30, LOWEST[dtype]))
    zt[6, 0] = mask
    zt[6, 0, (x[6] + 1) % V] = -3.0                      # one choice, not the drafted token
    if probs:
        zd[0, 0, x[0]] = mask                           # masked in both rows, with the same and with other numbers
        zd[3, 0, x[3]] = -np.inf
        zd[4, 0, x[4]] = LOWEST[dtype]
        zd[5, 0, x[5]] = -1e30
        zd[7, 0, x[7]] = mask                           # by the drafter alone
        zd[8, 0] = mask                                 # an empty row of the drafter's
        zd[9, 0] = mask
        zt[9, 0] = mask
    put(case, zt, zd, dtype)
    case["u"][:10, 0] = uniform
    ref = check_verify(case, B, G, V, V, None)
    assert not ref["accepted"][:7].any() and (ref["tokens"][1:3, 0] == -1).all() and ref["tokens"][6, 0] == (x[6] + 1) % V
    if probs:
        assert ref["accepted"][7] > 0 and ref["accepted"][8] == 0 and ref["tokens"][8, 0] >= 0 and ref["tokens"][9, 0] == -1


@pytest.mark.parametrize("B,G,V", FORMS)
def test_verify_of_ratios_past_32_bits(gh, B, G, V):   # noqa: F811
    """p / q beyond what a 32-bit exponential holds, either way, and a ratio whose logarithm 32 bits round by more than 1."""
    case = draft_case(22, B, G, V, "f32", True)
    zt, zd = parts(case, B, G, V)
    x = case["tokens"][:, 0]
    u = case["u"]
    u[:8, 0] = 0.999
    zd[0, 0, x[0]] = -1e9                               # a mask that is an ordinary logit: q = 0 nearly, accepted
    zd[1, 0, x[1]] = -1e9
    zt[1, 0] -= np.float32(2.5) + np.log(np.exp(zt[1, 0].astype(np.float64)).sum()).astype(np.float32)
    zd[2, 0, x[2]] = -3e8
    zd[3, 0, x[3]] = -200.0                             # e^200
    zt[4, 0, x[4]] = -1e9                               # p = 0 nearly, refused
    zt[5, 0, x[5]] = zt[5, 0].max() - 120.0             # p > 0, which a number of 0 is below
    u[5, 0] = 0.0
    zt[6, 0, x[6]] = zd[6, 0, x[6]] - 110.0             # e^-110 of about 1.7e-48: the smallest 32-bit number is above it,
    u[6, 0] = 2.0 ** -149
    zt[7, 0, x[7]] = zd[7, 0, x[7]] - 95.0              # and below e^-95
    u[7, 0] = 2.0 ** -149
    put(case, zt, zd, "f32")
    ref = check_verify(case, B, G, V, V, None)
    assert (ref["accepted"][[0, 1, 2, 3, 5, 7]] > 0).all() and not ref["accepted"][[4, 6]].any()
    bare = dict(case, d=None, dh=None)                  # without the drafter's rows: p itself
    ref = check_verify(bare, B, G, V, V, None)
    assert ref["accepted"][5] > 0 and not ref["accepted"][4]


@pytest.mark.parametrize("V", [200, 5000, 40003])
def test_distill_of_lists_that_leave_little(gh, V):   # noqa: F811
    """A teacher whose list leaves 1e-9 to 1e-7 of its probability, and a student that leaves less outside it: the others' gradient is that small
    difference alone, to the accuracy of everything else."""
    T, K = 6, 12
    rng = np.random.default_rng(V)
    z = normal([V, 6], T, V, 1.0)
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    for t in range(T):
        z[t, index[t]] += 60.0
    lists = []
    while len(lists) < T:
        lp = np.log(rng.dirichlet(np.ones(K))).astype(np.float32)
        if 1e-9 < 1.0 - np.exp(lp.astype(np.float64)).sum() < 1e-7:
            lists.append(lp)
    check_distill(z, "f32", K, 1, w=np.ones(T, np.float32), lists=(index, np.stack(lists)))


# ------------------------------------------------------------------------------------------------ logits far from 0
MASKS = [-1.2e9, -5e9, -1e10, -1e20, -1e30]
N_MASKED = 8


def masked_rows(seed, V, mask):
    """Rows cut by a finite mask: the first half, all but the last few, every other logit, everything, all but one, the first vectors
    of every thread, the end, none."""
    z = normal([seed, V], N_MASKED, V)
    z[0, : V // 2] = mask
    z[1, : V - 7] = mask
    z[2, ::2] = mask
    z[3] = mask
    z[4, np.arange(V) != V // 3] = mask
    z[5, : min(V - 5, 16384)] = mask
    z[6, V // 5:] = mask
    return z


def check_top_near(values, dtype, K):
    """Rows whose logits are all far from 0 and next to each other: an exponential's argument is up to 64 in size, so that a probability is
    off by 2^-18."""
    T, V = values.shape
    z, host = stored(values, dtype)
    index, lp, lse = run_top(z, T, V, V, K)
    want_i, want_lp, want_lse = orc.top(host, V, K)
    assert np.array_equal(index, want_i)
    there = want_i >= 0
    assert (np.abs(lp - want_lp)[there] <= rel(V, 16.0) + 2.0 ** -18 + 2.0 ** -23 * np.abs(want_lp[there])).all()
    assert (lp[~there] == -np.inf).all() and (np.abs(lse - want_lse) <= 2.0 ** -23 * np.abs(want_lse)).all()


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,copies", [(130, 1), (3001, 1), (3001, 70), (40003, 1), (40003, 70), (151936, 1)])
def test_top_of_rows_with_finite_masks(gh, dtype, mask, V, copies):   # noqa: F811
    z = np.repeat(masked_rows(1, V, mask), copies, 0)
    if dtype == "bf16" and mask == -1.2e9:
        mask_is = float(torch.tensor(mask).bfloat16())
        assert mask_is > orc.MASKED   # not at the limit in this type: an ordinary logit
    for K in (5, 200) if copies == 1 else (20,):
        check_top(z, dtype, K)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 5003, 40003])
def test_top_of_rows_far_from_zero(gh, dtype, V):   # noqa: F811
    """Whole rows at one large number or a few next to it, of either sign; and the first logits that are too large."""
    z = np.zeros((10, V), np.float32)
    pick = np.random.default_rng(V).integers(0, 3, size=(10, V)).astype(np.float32)
    for t, (at, step) in enumerate([(-1e9, 0), (1e9, 0), (-1e9, 64), (1e9, 64), (-1.19e9, 128), (1.19e9, 128), (-2.0 ** 24, 1), (2.0 ** 27, 8), (-3e7, 2),
                                    (5e5, 0.25)]):
        z[t] = np.float32(at) + np.float32(step) * pick[t]
    check_top_near(z, dtype, 30)
    large = normal([V, 2], 6, V)
    for t, at in enumerate([1.2e9, 5e9, 1e10, 1e20, 3e38]):
        large[t, V - 1 - 7 * t] = at
    large[5] = 1e10
    if dtype == "bf16":
        large[0, V - 1] = 1.25e9
    check_top(large, dtype, 30)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype,V,copies", [("f32", 130, 1), ("bf16", 3001, 1), ("f32", 40003, 1), ("bf16", 90001, 1), ("bf16", 66001, 17)])
def test_distill_of_rows_with_finite_masks(gh, dtype, V, copies, tail, mask):   # noqa: F811
    """Lists of unmasked ids and, in two rows, one masked id, which makes their losses infinite."""
    z = masked_rows(2, V, mask)
    host = torch.from_numpy(z).to(TORCH[dtype]).float().double().numpy()
    index, lp = make_lists(V, host, 12, spread=0.2)
    index, lp, z = (np.repeat(x, copies, 0) for x in (index, lp, z))
    w = np.random.default_rng(V).uniform(0.2, 1.0, size=len(z)).astype(np.float32)
    check_distill(z, dtype, 12, tail, w=w, lists=(index, lp))
    index[[0, 2 * copies], 3] = 0
    index[[0, 2 * copies], 4:] = -1
    check_distill(z, dtype, 12, tail, w=w, lists=(index, lp), inplace=True)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("V,copies", [(300, 1), (5003, 1), (40003, 1), (33003, 40)])
def test_distill_of_rows_far_from_zero(gh, V, copies, tail):   # noqa: F811
    """A loss and a gradient do not change when a number is added to a row, which is exact here; then rows with a logit that is too large."""
    rng = np.random.default_rng([V, tail])
    pick = rng.integers(0, 3, size=(4, V)).astype(np.float32)
    z = np.stack([np.float32(at) + np.float32(step) * pick[t]
                  for t, (at, step) in enumerate([(-1e9, 0), (1e9, 0), (-2.0 ** 23, 1), (2.0 ** 22, 0.5)])])
    z = np.repeat(z, copies, 0)
    T, K = len(z), 9
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    lp = np.log(rng.dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32)
    w = rng.uniform(0.2, 1.0, size=T).astype(np.float32)
    dev, host = stored(z, "f32")
    near = host - host.max(1, keepdims=True)
    ref = orc.distill(near, V, index, lp, w, tail, 1.0)
    dz = sevens(T, V, "f32")
    _, rows, err = run_distill(dev, T, V, V, index, lp, w, tail, 1.0, dz)
    row_bound, grad_bound = distill_bounds(ref, near, w, "f32", 1.0)
    far = 4 * 2.0 ** -18 * np.abs(w)[:, None] * (ref["masses"][:, :1] + ref["masses"][:, 1:2]) * np.ones(V)   # of an argument up to 64, as in the lists
    assert err == 0 and (np.abs(rows - ref["row_loss"]) <= row_bound + 4 * 2.0 ** -18 + 2.0 ** -22 * np.abs(ref["row_loss"])).all()
    assert (np.abs(wide(dz).reshape(T, V) - ref["dlogits"]) <= grad_bound + far).all()

    large = np.repeat(normal([V, 5], 4, V), copies, 0)
    index, lp = make_lists(V, large.astype(np.float64), K)
    large[0, 7] = 1.2e9
    large[1, index[1, 2]] = 1e10
    large[2] = 3e38
    dev, _ = stored(large, "f32")
    dz = sevens(T, V, "f32")
    loss, rows, _ = run_distill(dev, T, V, V, index, lp, np.ones(T, np.float32), tail, 1.0, dz)
    got = wide(dz).reshape(T, V)
    assert np.isnan(loss) and np.isnan(rows[:3]).all() and np.isfinite(rows[3:]).all()
    assert np.isnan(got[:3]).all() and np.isfinite(got[3:]).all()


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("V", [3000, 40003, 100003])
def test_distill_of_offsets_off_either_way(gh, V, tail, sign):   # noqa: F811
    """Offsets that are 60 above the others' exponents and 60 below the listed ones': each sum keeps what its offset leaves, 2^60 and 2^-60 a logit, and
    the others' share of the whole is 0, not the infinite ratio of those times 0."""
    k = float(np.float32(1.4426950408889634))
    far = (np.float32(1.1e9) + 128 * np.arange(4000)).astype(np.float32) * np.float32(sign)
    residual = far.astype(np.float64) * k - np.rint((far.astype(np.float64) * k).astype(np.float32).astype(np.float64))
    others = far[residual > 60].min()
    listed = far[(residual < -60) & (far > others)].min()
    T, K = 3, 5
    rng = np.random.default_rng(V)
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    lp = np.log(rng.dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32)
    z = np.full((T, V), others, np.float32)
    for t in range(T):
        z[t, index[t]] = listed
    dev, host = stored(z, "f32")
    ref = orc.distill(host - float(listed), V, index, lp, np.ones(T), tail, 1.0)
    dz = sevens(T, V, "f32")
    _, rows, _ = run_distill(dev, T, V, V, index, lp, np.ones(T, np.float32), tail, 1.0, dz)
    total, rest_p, _ = ref["masses"].T
    share = np.full((T, V), 1.0 / (V - K))
    np.put_along_axis(share, index, 0.0, 1)
    size = total[:, None] * ref["q"] + ref["p"] + rest_p[:, None] * share
    assert (np.abs(rows - ref["row_loss"]) <= 4 * 2.0 ** -18 + 2.0 ** -22 * np.abs(ref["row_loss"])).all()
    assert (np.abs(wide(dz).reshape(T, V) - ref["dlogits"]) <= 4 * 2.0 ** -18 * size + 2.0 ** -126).all()


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("B,G,V", FORMS)
def test_verify_of_rows_with_finite_masks(gh, B, G, V, probs, mask):   # noqa: F811
    """The policy's and the drafter's rows cut alike or otherwise; a masked row; rows of large numbers."""
    case = draft_case(23, B, G, V, "f32", probs)
    zt, zd = parts(case, B, G, V)
    x = case["tokens"][:, 0]
    for b in range(4):
        cut = np.zeros(V, bool)
        cut[[slice(0, V // 2), slice(0, V - 7), slice(0, None, 2), slice(V // 5, None)][b]] = True
        cut[x[b]] = b % 2
        zt[b, 0, cut] = mask
        if probs and b < 3:
            zd[b, 0, cut] = mask
    zt[4, 0] = mask
    zt[5, 0] = np.where(np.arange(V) % 2 == 0, np.float32(-1e9), np.float32(-1e9 - 64))
    zt[6, 0, V - 1] = 1e10
    if probs:
        zd[7, 0] = mask
        zd[8, 0, 1] = 1.2e9
        zd[9, 0] = zt[9, 0] = np.where(np.arange(V) % 2 == 0, np.float32(1e9), np.float32(-1e9))
    put(case, zt, zd, "f32")
    ref = check_verify(case, B, G, V, V, None)
    assert ref["tokens"][4, 0] == -1 and ref["tokens"][6, 0] == -1 and ref["tokens"][5, 0] >= 0


@pytest.mark.parametrize("B,G,V", [(5, 1, 600), (5, 1, 20001), (300, 1, 600)])
def test_no_masked_token_is_drawn(gh, B, G, V):   # noqa: F811
    """Next to the limit a masked logit's exponential may be 2^-120 for 0: where the drafter's row leaves nothing of the others, the token comes from
    p all the same."""
    case = draft_case(24, B, G, V, "f32", True)
    zt, zd = parts(case, B, G, V)
    masked = np.arange(V) % 50 != 3
    zt[:, 0] = np.where(masked, np.float32(-1.2e9), np.float32(-1.2e9 + 128))
    zd[:, 0] = np.where(masked, np.float32(-3e38), np.float32(-1.2e9 + 128))
    case["tokens"][:] = 0
    case["u"][:] = 0.5
    put(case, zt, zd, "f32")
    ref = check_verify(case, B, G, V, V, None)
    assert not ref["accepted"].any() and (ref["tokens"][:, 0] % 50 == 3).all()


# ------------------------------------------------------------------------------------------------ many sequences
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("B,G,V", [(1030, 1, 13001), (1030, 1, 5000), (420, 2, 24001)])
def test_verify_of_many_sequences_of_longer_rows(gh, B, G, V, probs):   # noqa: F811
    """On both sides of the lengths up to which a workgroup takes a whole sequence, where there are more sequences than compute units."""
    case = draft_case(25, B, G, V, "bf16", probs)
    count = np.full(B, G, np.int32)
    count[5], count[6], count[7] = -1, 0, G + 1
    check_verify(case, B, G, V, V, count, err=16)


@pytest.mark.parametrize("B,G,V", [(1100, 0, 700), (1100, 0, 3001), (600, 0, 2001), (1100, 1, 3001), (1100, 1, 6001), (300, 2, 9001)])
def test_verify_of_many_sequences_of_few_rows(gh, B, G, V):   # noqa: F811
    """Few rows a sequence, which leave most of a workgroup's waves idle: on both sides of where one launch ends."""
    for dtype, probs in (("bf16", True), ("f32", False)):
        count = None
        if G:
            count = np.full(B, G, np.int32)
            count[3], count[4] = -1, 0
        check_verify(draft_case(26, B, G, V, dtype, probs), B, G, V, V, count)
