"""The checker of the loss on pairs and of the AdamW step against differences and properties, the pairs of a step's groups, and what the
calls refuse (no GPU: a call that is refused launches nothing)."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from oracle import training_oracle as orc


def library():
    from paper_2602_14338_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build()
    return binding


# ------------------------------------------------------------------------------------------------ preference loss
@pytest.mark.parametrize("kind", [orc.LOGISTIC, orc.HINGE, orc.SQUARE])
@pytest.mark.parametrize("average", [0, 1])
def test_slope_against_differences(kind, average):
    rng = np.random.default_rng(kind * 2 + average)
    rollout = np.array([0, 0, 1, 2, 2, 2, -1, 3, 5, 5])
    lp, ref = -rng.exponential(size=10), -rng.exponential(size=10)
    chosen, rejected, w = [0, 2, 0, 4], [1, 1, 3, 5], rng.uniform(0.5, 1, 4)
    how = dict(kind=kind, average=average, beta=0.7, smoothing=0.2, margin=0.3)
    _, _, _, slope, count = orc.preference(lp, ref, rollout, 6, chosen, rejected, w, **how)
    assert count[4] == 0 and slope[4] != 0.0 or kind == orc.HINGE
    h = 1e-5
    for t in range(10):
        up, down = lp.copy(), lp.copy()
        up[t] += h
        down[t] -= h
        got = (orc.preference(up, ref, rollout, 6, chosen, rejected, w, **how)[0] -
               orc.preference(down, ref, rollout, 6, chosen, rejected, w, **how)[0]) / (2 * h)
        assert abs(got - (slope[rollout[t]] if rollout[t] >= 0 else 0.0)) < 1e-8


def test_gradient_rows_against_differences():
    rng = np.random.default_rng(3)
    z = rng.normal(0, 2, size=(6, 5))
    z[1, 3] = -np.inf
    y, rollout = np.array([0, 4, 2, 1, 3, 0]), np.array([0, 0, 1, 1, -1, 2])
    ref = -rng.exponential(size=6)
    args = (5, y, ref, rollout, 3, [0, 2], [1, 1], None)
    how = dict(grad_scale=1.0, beta=0.9, smoothing=0.1)
    dz = orc.preference_rows(z, *args, **how)[5]
    h = 1e-5
    for t in range(6):
        for j in range(5):
            up, down = z.copy(), z.copy()
            up[t, j] += h
            down[t, j] -= h
            got = (orc.preference_rows(up, *args, **how)[0] - orc.preference_rows(down, *args, **how)[0]) / (2 * h)
            assert abs(got - dz[t, j]) < 1e-8


def test_pairs_of_groups():
    from paper_2602_14338_amd.preference import pairs_of_groups
    rewards = np.array([1, 0, 0, 1, 1, 0, 0, 1, 0], np.float32)
    kept, offsets = np.array([0, 1, 3, 5, 6, 7], np.int32), np.array([0, 4, 4, 6], np.int32)
    c, j = pairs_of_groups(rewards, kept, offsets)
    assert c.dtype == j.dtype == np.int32 and c.tolist() == [0, 3, 7] and j.tolist() == [1, 5, 6]
    c, j = pairs_of_groups(rewards, kept, offsets, every=True)
    assert sorted(zip(c.tolist(), j.tolist())) == [(0, 1), (0, 5), (3, 1), (3, 5), (7, 6)]
    c, j = pairs_of_groups(rewards, kept, np.array([0], np.int32))
    assert c.size == j.size == 0


# ------------------------------------------------------------------------------------------------ moments in 8 bits
def test_every_code_stands_for_itself():
    for first in (True, False):
        codes = np.arange(-127, 128) if first else np.arange(256)
        codes = np.concatenate([codes, np.zeros(256 - len(codes), int)])
        scale = np.array([orc.F(0.37)])
        x = orc.values_of(codes, scale, first)
        again = orc.scale_of(x, orc.TOP1 if first else orc.TOP2)
        assert abs(float(again[0]) / 0.37 - 1) < 2.0 ** -22
        assert np.array_equal(orc.codes_of(x, again, np.full(256, 0.5), first), codes)


@pytest.mark.parametrize("first", [True, False])
def test_nearest_code(first):
    rng = np.random.default_rng(5)
    x = (rng.normal(size=256) if first else rng.exponential(size=256) ** 4).astype(orc.F)
    scale = orc.scale_of(x, orc.TOP1 if first else orc.TOP2)
    codes = orc.codes_of(x, scale, np.full(256, 0.5), first)
    every = np.arange(-127, 128) if first else np.arange(1, 256)
    values = orc.values_of(every, np.repeat(scale, len(every)), first).astype(np.float64)
    best = np.abs(values[None, :] - x[:, None].astype(np.float64)).min(axis=1)
    got = np.abs(orc.values_of(codes, scale, first).astype(np.float64) - x)
    assert (got <= best + 2.0 ** -21 * np.abs(x)).all()   # but for numbers as far from either by their roundings


@pytest.mark.parametrize("first", [True, False])
def test_random_rounding_keeps_the_mean(first):
    """A moment between two codes a and b is stored as either, its mean over n steps within 5 standard deviations, (b - a) / (2 sqrt n) at most,
    and 2^-17 (b - a) for the 16 bits."""
    x = np.full(256, 0.0123, orc.F)
    x[0] = 1.0
    scale = orc.scale_of(x, orc.TOP1 if first else orc.TOP2)
    total, n = np.zeros(256), 400
    for step in range(n):
        h = orc.random_bits(0x123456789, step, 3, 256)
        u = (((h & 0xffff) if first else (h >> 16)).astype(np.float64) + 0.5) / 65536
        total += orc.values_of(orc.codes_of(x, scale, u, first), scale, first)
    mean = total[1:].mean() / n
    lo = orc.codes_of(x, scale, np.full(256, 1 - 2.0 ** -17), first)[1]
    a, b = (float(orc.values_of(np.array([c]), scale, first)[0]) for c in (lo, lo + 1))
    assert a < 0.0123 < b and abs(mean - float(x[1])) <= (b - a) * (5 / (2 * math.sqrt(n * 255)) + 2.0 ** -17)


def test_random_bits_look_random():
    """Each of the 32 bits, and its agreement with that of another step, tensor, seed or neighbour, within 5 standard deviations of evenness; so too the 16
    high bits of the odd multiple (a parameter's), and their agreement with each half of the number (the moments')."""
    n = 1 << 16
    even = lambda bits: abs(int((bits & 1).sum()) - n / 2) < 5 * math.sqrt(n) / 2   # noqa: E731
    a = orc.random_bits(1, 0, 0, n)
    others = (orc.random_bits(1, 1, 0, n), orc.random_bits(1, 0, 1, n), orc.random_bits(2, 0, 0, n), orc.random_bits(1 + (1 << 32), 0, 0, n), np.roll(a, 1))
    for bit in range(32):
        assert even(a >> bit), bit
        for other in others:
            assert even((a ^ other) >> bit), bit
    high = (a * 0x9E3779B1 & 0xffffffff) >> 16
    for bit in range(16):
        assert even(high >> bit) and even((high ^ a) >> bit) and even((high ^ (a >> 16)) >> bit), bit


def test_second_moment_is_never_lost():
    x = np.zeros(256, orc.F)
    x[0], x[1] = 1.0, 1e-20
    codes = orc.codes_of(x, orc.scale_of(x, orc.TOP2), np.full(256, 0.5), False)
    assert codes[0] == 255 and codes[1] == 1 and (codes[2:] == 0).all()


# ------------------------------------------------------------------------------------------------ refusals
FAKE = 0x1000000   # an aligned address that is never followed


def entry(b, **more):
    x = dict(param=FAKE, grad=FAKE, master=None, exp_avg=FAKE, exp_avg_sq=FAKE, exp_avg_scale=None, exp_avg_sq_scale=None, n=1000,
             param_dtype=b.AERO_F32, grad_dtype=b.AERO_F32, decay=1.0)
    x.update(more)
    return b._TensorC(**x)


def image_of(b, *entries, short=0):
    rows = (b._TensorC * max(len(entries), 1))(*entries)
    size = b._lib.aero_tensor_table_bytes(rows, len(entries))
    raw = np.zeros(size + 16, np.uint8)
    at = (raw.ctypes.data + 15) & ~15
    return b._lib.aero_tensor_table(rows, len(entries), at, size - short), at, raw


def test_table_takes_what_it_should():
    b = library()
    good = [dict(), dict(n=0), dict(n=1), dict(n=(1 << 32) - 1), dict(param=None, exp_avg=None, exp_avg_sq=None), dict(grad_dtype=b.AERO_BF16),
            dict(param_dtype=b.AERO_BF16), dict(param_dtype=b.AERO_BF16, master=FAKE), dict(param_dtype=b.AERO_F16, master=FAKE, grad_dtype=b.AERO_F16),
            dict(exp_avg_scale=FAKE, exp_avg_sq_scale=FAKE), dict(exp_avg_scale=FAKE, exp_avg_sq_scale=FAKE, exp_avg=FAKE + 1, exp_avg_sq=FAKE + 3),
            dict(param_dtype=b.AERO_BF16, param=FAKE + 2), dict(decay=0.0)]
    for e in good:
        assert image_of(b, entry(b, **e))[0] == 0, e
    assert image_of(b)[0] == 0
    assert image_of(b, *(entry(b, **e) for e in good))[0] == 0


def test_table_refusals():
    b = library()
    NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
    bad = [(dict(grad=None), NULL), (dict(exp_avg=None), NULL), (dict(exp_avg_sq=None), NULL), (dict(exp_avg_scale=FAKE), NULL),
           (dict(exp_avg_sq_scale=FAKE), NULL), (dict(n=-1), SHAPE), (dict(n=1 << 32), SHAPE), (dict(decay=math.nan), SHAPE),
           (dict(decay=math.inf), SHAPE), (dict(grad_dtype=b.AERO_F8E4M3), DTYPE), (dict(param_dtype=b.AERO_F8E4M3), DTYPE),
           (dict(param_dtype=b.AERO_F16), DTYPE), (dict(master=FAKE), DTYPE), (dict(grad=FAKE + 2), ALIGN), (dict(param=FAKE + 1), ALIGN),
           (dict(param_dtype=b.AERO_BF16, master=FAKE + 2), ALIGN), (dict(exp_avg=FAKE + 2), ALIGN),
           (dict(exp_avg_scale=FAKE + 1, exp_avg_sq_scale=FAKE), ALIGN)]
    for e, status in bad:
        assert image_of(b, entry(b), entry(b, **e))[0] == status, e
    assert image_of(b, entry(b), short=1)[0] == WORKSPACE
    assert b._lib.aero_tensor_table(None, 1, FAKE, 100) == NULL
    rows = (b._TensorC * 1)(entry(b))
    assert b._lib.aero_tensor_table(rows, 1, None, 10 ** 6) == NULL
    assert b._lib.aero_tensor_table(rows, -1, FAKE, 100) == SHAPE and b._lib.aero_tensor_table(rows, 1 << 20, FAKE, 100) == SHAPE


def test_step_and_norm_refusals():
    b = library()
    NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
    st, image, keep = image_of(b, entry(b))
    assert st == 0
    step = lambda **k: b._lib.aero_adamw_step(image, FAKE, C.byref(b.AdamWParams(**k).to_c()), FAKE, None, None, None)   # noqa: E731
    for k in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=math.nan),
              dict(eps=math.inf), dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(weight_decay=math.nan)):
        assert step(**k) == SHAPE, k
    good = C.byref(b.AdamWParams().to_c())
    junk = np.zeros(4096, np.uint8)
    call = b._lib.aero_adamw_step
    assert call(junk.ctypes.data, FAKE, good, FAKE, None, None, None) == SHAPE        # no image
    assert call(image, FAKE + 8, good, FAKE, None, None, None) == ALIGN
    for a in ((None, FAKE, good, FAKE), (image, None, good, FAKE), (image, FAKE, None, FAKE), (image, FAKE, good, None)):
        assert call(*a, None, None, None) == NULL
    norm = b._lib.aero_grad_norm
    size = b._lib.aero_workspace_bytes(b.OP_GRAD_NORM, 0, 0, 0, 0, 0)
    assert norm(image, FAKE, math.nan, 1.0, FAKE, FAKE, FAKE, size, None) == SHAPE
    assert norm(image, FAKE, math.inf, 1.0, FAKE, FAKE, FAKE, size, None) == SHAPE
    assert norm(image, FAKE, 1.0, math.nan, FAKE, FAKE, FAKE, size, None) == SHAPE
    assert norm(image, FAKE, 1.0, 1.0, FAKE, FAKE, None, size, None) == WORKSPACE
    assert norm(image, FAKE, 1.0, 1.0, FAKE, FAKE, FAKE, size - 1, None) == WORKSPACE
    assert norm(image, FAKE, 1.0, 1.0, FAKE, FAKE, FAKE + 16, size, None) == WORKSPACE
    assert norm(None, FAKE, 1.0, 1.0, FAKE, FAKE, FAKE, size, None) == NULL and norm(image, None, 1.0, 1.0, FAKE, FAKE, FAKE, size, None) == NULL
    moments = b._lib.aero_adamw_moments
    assert moments(image, FAKE, b.AERO_F16, FAKE, FAKE, None) == DTYPE and moments(image, FAKE, b.AERO_F32, FAKE, None, None) == NULL
    assert moments(image, FAKE, b.AERO_F32, FAKE + 2, FAKE, None) == ALIGN


def test_preference_refusals():
    b = library()
    NULL, SHAPE, DTYPE, WORKSPACE = 1, 2, 3, 5
    good = dict(logprob=FAKE, T=10, ref=None, rollout=FAKE, R=4, chosen=FAKE, rejected=FAKE, weight=None, P=2, params={}, loss=FAKE, ws=FAKE, short=0)

    def terms(**more):
        a = dict(good, **more)
        params = C.byref(b.PreferenceParams(**a["params"]).to_c()) if a["params"] is not None else None
        size = b._lib.aero_workspace_bytes(b.OP_PREFERENCE_LOSS, a["T"], 0, 0, a["R"], a["P"]) - a["short"]
        return b._lib.aero_preference_loss(a["logprob"], a["T"], a["ref"], a["rollout"], a["R"], a["chosen"], a["rejected"], a["weight"], a["P"], params,
                                           a["loss"], None, None, None, None, a["ws"], size, None)

    def rows(**more):
        a = {**good, "V": 100, "ld": 100, "dtype": b.AERO_BF16, "targets": FAKE, **more}
        params = C.byref(b.PreferenceParams(**a["params"]).to_c()) if a["params"] is not None else None
        size = b._lib.aero_workspace_bytes(b.OP_PREFERENCE_LOSS_BWD, a["T"], a["V"], 0, a["R"], a["P"]) - a["short"]
        return b._lib.aero_preference_loss_bwd(a["logprob"], a["dtype"], a["T"], a["V"], a["ld"], a["targets"], a["ref"], a["rollout"], a["R"], a["chosen"],
                                               a["rejected"], a["weight"], a["P"], params, 1.0, a["loss"], None, None, None, FAKE, None, a["ws"], size, None)

    both = [(dict(T=-1), SHAPE), (dict(T=1 << 25), SHAPE), (dict(R=-1), SHAPE), (dict(R=1 << 22), SHAPE), (dict(P=-1), SHAPE), (dict(P=1 << 22), SHAPE),
            (dict(params=dict(kind=3)), SHAPE), (dict(params=dict(kind=-1)), SHAPE), (dict(params=dict(average=2)), SHAPE),
            (dict(params=dict(beta=0.0)), SHAPE), (dict(params=dict(beta=-1.0)), SHAPE), (dict(params=dict(beta=math.nan)), SHAPE),
            (dict(params=dict(beta=math.inf)), SHAPE), (dict(params=dict(margin=math.nan)), SHAPE), (dict(params=dict(margin=math.inf)), SHAPE),
            (dict(params=dict(smoothing=-0.1)), SHAPE), (dict(params=dict(smoothing=0.6)), SHAPE), (dict(params=dict(smoothing=math.nan)), SHAPE),
            (dict(params=None), NULL), (dict(loss=None), NULL), (dict(logprob=None), NULL), (dict(rollout=None), NULL), (dict(chosen=None), NULL),
            (dict(rejected=None), NULL), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 16), WORKSPACE), (dict(short=1), WORKSPACE)]
    for more, status in both:
        assert terms(**more) == status, more
        assert rows(**more) == status, more
    for more, status in ((dict(T=1 << 22), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1, ld=1 << 25), SHAPE), (dict(V=101), SHAPE), (dict(dtype=4), DTYPE),
                         (dict(targets=None), NULL)):
        assert rows(**more) == status, more


def test_constants_match_the_header(tmp_path):
    import subprocess
    b = library()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {"AERO_OP_PREFERENCE_LOSS": b.OP_PREFERENCE_LOSS, "AERO_OP_PREFERENCE_LOSS_BWD": b.OP_PREFERENCE_LOSS_BWD, "AERO_OP_GRAD_NORM": b.OP_GRAD_NORM,
             "AERO_PAIR_LOGISTIC": b.AERO_PAIR_LOGISTIC, "AERO_PAIR_HINGE": b.AERO_PAIR_HINGE, "AERO_PAIR_SQUARE": b.AERO_PAIR_SQUARE,
             "AERO_MOMENT_BLOCK": b.AERO_MOMENT_BLOCK, "sizeof(aero_preference_params)": C.sizeof(b._PreferenceParamsC),
             "sizeof(aero_adamw_params)": C.sizeof(b._AdamWParamsC), "sizeof(aero_tensor)": C.sizeof(b._TensorC)}
    src, exe = tmp_path / "c.c", tmp_path / "c"
    src.write_text('#include "aero.h"\n#include <stdio.h>\nint main(void) {\n' + "".join(f'  printf("%ld\\n", (long)({n}));\n' for n in names) + "  return 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == list(names.values())


def test_an_eps_whose_reciprocal_is_infinite_is_refused():
    b = library()
    st, image, keep = image_of(b, entry(b))
    assert st == 0
    for eps in (1e-40, 2.0 ** -128, 2.0 ** -127, float(np.nextafter(np.float32(2.0 ** -126), np.float32(0)))):
        params = C.byref(b.AdamWParams(eps=eps).to_c())
        assert b._lib.aero_adamw_step(image, FAKE, params, FAKE, None, None, None) == 2, eps
