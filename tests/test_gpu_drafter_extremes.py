"""The calls around a drafter on logits that masks and other callers write: finite masks, logits far from 0, probabilities that vanish.
Helpers, checks and tolerances are those of test_gpu_drafter."""
import numpy as np
import pytest
import torch

from test_gpu_drafter import check_distill, check_verify, draft_case, gh, normal, stored  # noqa: F401

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
