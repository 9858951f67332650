"""The drafter that learns from the policy and drafts for it (paper_2602_14338_amd/drafter.py), and the native step of the
binding's calls that it makes.
"""
import numpy as np
import pytest
import torch

from oracle import drafter_oracle as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -8   # bf16: half a unit in the last place


@pytest.fixture(scope="module")
def gh():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gpu_helpers
    return gpu_helpers


def wide(t):
    return t.cpu().float().double().numpy()


def device(x):
    return torch.from_numpy(x).to("cuda")


class _Int(int):
    pass


@pytest.mark.parametrize("entry", ["topk", "distill", "verify", "embed_fwd", "embed_bwd"])
def test_native_step(gh, monkeypatch, entry):
    """Plain arguments go through the native step; what is not plain it leaves alone, with NotImplemented.  Either way the
    results, or the error, are those of the general way.  Every size has a value of its own, so that two that change places show."""
    b = gh.aero.binding
    rng = np.random.default_rng(6)
    T, V, H, K, ld, B, G = 33, 300, 24, 5, 311, 6, 3
    rows = lambda *s: device(rng.normal(0, 2, size=s).astype(np.float32)).bfloat16()   # noqa: E731
    new = lambda *s, dtype=torch.float32: torch.full(s, 7, dtype=dtype, device="cuda")   # noqa: E731
    ints = lambda lo, hi, *s: device(rng.integers(lo, hi, size=s).astype(np.int32))   # noqa: E731
    ws = torch.empty(max(gh.aero.aero_workspace_bytes(op, T=T, V=V, H=H, Q=B)
                         for op in (b.OP_TOPK_LOGPROB, b.OP_DISTILL_LOSS_BWD, b.OP_VERIFY_DRAFT, b.OP_EMBEDDING_BWD)),
                     dtype=torch.uint8, device="cuda")
    z, zt, zd, table, dout = rows(T, ld), rows(B, G + 1, ld), rows(B, G, ld), rows(V, H), rows(T, 31)
    active = device(rng.integers(0, 2, size=T).astype(np.uint8))
    lists = device(np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32))
    lists_lp = device(np.log(rng.dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32))
    weight = device(rng.random(T).astype(np.float32))
    ids, toks, count = ints(-1, V, T), ints(0, V, B, G), ints(0, G + 1, B)
    uniform, noise = device(rng.random((B, G)).astype(np.float32)), device(rng.exponential(size=(B, V)).astype(np.float32))

    def call(**kw):
        g = lambda k, v: kw.get(k, v)   # noqa: E731
        err = new(1, dtype=torch.int32) * 0
        if entry == "topk":
            out = [new(T, K, dtype=torch.int32), new(T, K), new(T)]
            b.aero_topk_logprob(g("z", z), g("T", T), g("V", V), ld, g("active", active), K, *out, g("ws", ws))
        elif entry == "distill":
            out = [new(1), new(T), new(T, ld, dtype=g("dz", torch.bfloat16))]
            b.aero_distill_loss_bwd(g("z", z), g("T", T), g("V", V), ld, lists, lists_lp, K, g("weight", weight), g("tail", 1), g("scale", 1.5),
                                    *out, g("ws", ws), err)
        elif entry == "verify":
            out = [new(B, dtype=torch.int32), new(B, G + 1, dtype=torch.int32), new(B, G + 1)]
            b.aero_verify_draft(zt, g("zd", zd), g("T", B), G, g("V", V), ld, toks, g("count", count), uniform, g("noise", noise), *out, g("ws", ws), err)
        elif entry == "embed_fwd":
            out = [new(T, 29, dtype=g("out", torch.bfloat16))]
            b.aero_embedding_fwd(g("z", table), g("V", V), H, g("ids", ids), g("T", T), g("scale", 0.5), *out, 29, err)
        else:
            out = [new(V, H, dtype=g("dtable", torch.float32))]
            b.aero_embedding_bwd(g("z", dout), g("T", T), H, 31, g("ids", ids), g("V", V), g("scale", 0.5), *out, g("ws", ws),
                                 g("accumulate", False), err)
        return out + [err]

    answers, general = [], []
    step = getattr(b._m, entry)

    def watched(*a):
        answers.append(NotImplemented if general else step(*a))
        return answers[-1]
    monkeypatch.setattr(b._m, entry, watched)

    def outcome(kw):
        try:
            return call(**kw)
        except Exception as e:   # noqa: BLE001
            return type(e), str(e)

    plain = [dict(), dict(T=-1), dict(V=0)] + {
        "topk": [dict(active=None), dict(ws=None)], "distill": [dict(tail=0), dict(scale=2), dict(ws=None)],
        "verify": [dict(count=None), dict(zd=None), dict(ws=None)], "embed_fwd": [dict(scale=2)],
        "embed_bwd": [dict(accumulate=True), dict(dtable=torch.bfloat16), dict(ws=None)]}[entry]
    other = [dict(T=_Int(T if entry != "verify" else B)), dict(T=2.0), dict(V=2 ** 40)] + {
        "topk": [dict(z=z.double()), dict(z=z.cpu()), dict(active=active.int()), dict(z=z.t().contiguous().t())],
        "distill": [dict(z=z.double()), dict(dz=torch.float32), dict(weight=weight.double()), dict(scale="x"), dict(tail=1.0)],
        "verify": [dict(zd=zd.float()), dict(noise=noise.double()), dict(count=count.long())],
        "embed_fwd": [dict(out=torch.float32), dict(ids=ids.long()), dict(z=table.double())],
        "embed_bwd": [dict(dtable=torch.float64), dict(ids=ids.cpu()), dict(accumulate=1)]}[entry]
    for kw in plain + other:
        answers.clear()
        got = outcome(kw)
        assert len(answers) == 1 and (type(answers[0]) is int if any(kw is p for p in plain) else answers[0] is NotImplemented), (kw, answers)
        general.append(True)
        want = outcome(kw)
        general.clear()
        if isinstance(want, tuple):
            assert got == want, kw
        else:
            assert isinstance(got, list) and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, want)), kw
            assert not (got[0] == 7).all(), kw


def test_teacher_lists(gh):
    from paper_2602_14338_amd import drafter as d
    rng = np.random.default_rng(1)
    z = rng.normal(0, 2, size=(9, 250)).astype(np.float32)
    active = (np.arange(9) != 4).astype(np.uint8)
    lists = d.teacher_lists(device(z), 241, 12, device(active))
    index, lp, lse = orc.top(z, 241, 12, active)
    assert np.array_equal(lists.index.cpu().numpy(), index)
    assert np.abs(wide(lists.logprob) - lp).max() <= 1e-5 and np.abs(wide(lists.lse) - lse).max() <= 1e-5


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_gradient_of_the_tied_table(gh, tail, grad):
    """Against automatic differentiation in 64 bits of the loss as a function of the table: L = w (P lse(z) - sum p z + const), or with
    the others as one event.

    The drafter's chain rounds z to bf16 (an error of U |z|, so a factor e^(2 U max|z|) in every probability), dz, dx and the head's part
    of the gradient once each, and the sum once."""
    from paper_2602_14338_amd import drafter as d
    rng = np.random.default_rng([7, tail])
    T, V, H, K = 150, 700, 32, 6
    table = device(rng.normal(0, 0.3, size=(V, H)).astype(np.float32)).bfloat16()
    ids = rng.integers(0, V // 3, size=T).astype(np.int32)
    ids[[3, 77]] = -1
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    lp = np.log(rng.dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32)
    weight = rng.random(T).astype(np.float32)
    weight[5] = 0
    drafter = d.Drafter(table, scale=2.0)   # a power of two: the rows looked up are exact
    dtable = torch.empty((V, H), dtype=grad, device="cuda")
    loss = drafter.loss_bwd(device(ids), d.TeacherLists(device(index), device(lp), None), device(weight), dtable, tail)
    alone = drafter.loss_bwd(device(ids), d.TeacherLists(device(index), device(lp), None), device(weight), None, tail)
    assert drafter.err.item() == 0 and torch.equal(loss, alone)

    E = table.cpu().double().requires_grad_()
    there = torch.from_numpy(ids >= 0)
    x = torch.where(there[:, None], 2.0 * E[torch.from_numpy(np.maximum(ids, 0)).long()], 0.0)
    z = x @ E.t()
    z.retain_grad()
    x.retain_grad()
    logq = torch.log_softmax(z, 1)
    p = torch.from_numpy(lp).double().exp()
    at = torch.from_numpy(index).long()
    w = torch.from_numpy(weight).double()
    if tail == 0:
        p = p / p.sum(1, keepdim=True)
        rows = (p * (p.log() - logq.gather(1, at))).sum(1)
    else:
        rest = 1.0 - p.sum(1)
        rows = (p * (p.log() - logq.gather(1, at))).sum(1) + rest * (rest.log() - torch.log1p(-logq.gather(1, at).exp().sum(1)))
    total = (w * rows).sum()
    total.backward()

    zmax = float(z.detach().abs().max())
    growth = np.expm1(2 * 1.01 * U * zmax)   # of a probability or a share of the rest
    q = logq.detach().exp()
    size = w[:, None] * (q * (2.0 if tail else 1.0)).scatter_add(1, at, p)   # |P q| + |p_r share| + |p|
    dz_err = growth * size + U * z.grad.abs()
    xs, Es = x.detach().abs(), E.detach().abs()
    head = dz_err.t() @ xs + 3 * U * (z.grad.abs().t() @ xs)
    dx_err = dz_err @ Es + 2 * U * (z.grad.abs() @ Es)
    lookup = torch.zeros(V, H, dtype=torch.float64).index_add(0, torch.from_numpy(ids[ids >= 0]).long(), 2.0 * dx_err[there])
    bound = head + lookup + 2 * U * E.grad.abs() + 1e-9
    assert ((dtable.cpu().double() - E.grad).abs() <= bound).all()
    assert abs(float(loss) - float(total.detach())) <= float((w * 2 * 1.01 * U * zmax * 2).sum())
    # neither part of the gradient alone is within the bound
    head_part = z.grad.t() @ x.detach()
    assert ((E.grad - head_part).abs() > bound).any() and (head_part.abs() > bound).any()


def test_tokens_are_the_policy_s(gh):
    """Counts of the first and of the second token of 40000 sequences against the policy's probabilities: chi-square with 11 degrees of
    freedom (45 and more: one in 200000)."""
    from paper_2602_14338_amd import drafter as d
    rng = np.random.default_rng(3)
    B, V, G = 40000, 12, 2
    target = rng.normal(0, 1.0, size=(G + 1, V)).astype(np.float32)
    table = device(rng.normal(0, 0.8, size=(V, 16)).astype(np.float32)).bfloat16()
    drafter = d.Drafter(table)
    gen = torch.Generator(device="cuda").manual_seed(11)
    last = torch.full((B,), 3, dtype=torch.int32, device="cuda")
    policy = lambda ids: device(target).bfloat16().expand(B, G + 1, V).contiguous()   # noqa: E731
    accepted, tokens, logprob, rows, drafted = d.generate(drafter, policy, last, G, gen)
    torch.cuda.synchronize()
    assert drafter.err.item() == 0 and rows.shape == (B, G + 1, V) and drafted.shape == (B, G)
    n, tok, lp = accepted.cpu().numpy(), tokens.cpu().numpy(), wide(logprob)
    logp = np.stack([orc.log_softmax(r) for r in wide(rows)[0]])
    assert 0.05 < (n == 0).mean() < 0.95 and (n == G).any()
    for i in range(G + 1):
        there = n >= i
        assert (tok[~there, i] == -1).all() and (tok[there, i] >= 0).all()
        assert np.abs(lp[there, i] - logp[i][tok[there, i]]).max() <= 1e-5 and not lp[~there, i].any()
        if i < 2:
            expected = there.sum() * np.exp(logp[i])
            assert ((np.bincount(tok[there, i], minlength=V) - expected) ** 2 / expected).sum() < 45
    kept = np.arange(G)[None] < n[:, None]
    assert (tok[:, :G][kept] == drafted.cpu().numpy()[kept]).all()


def test_drafted_tokens_are_the_drafter_s(gh):
    """A proposed token has the probability that verification reckons with; rows with padding columns are no different."""
    from paper_2602_14338_amd import drafter as d
    rng = np.random.default_rng(4)
    B, V = 30000, 10
    drafter = d.Drafter(device(rng.normal(0, 0.8, size=(V, 8)).astype(np.float32)).bfloat16())
    gen = torch.Generator(device="cuda").manual_seed(12)
    last = torch.full((B,), 7, dtype=torch.int32, device="cuda")
    tokens, rows = drafter.propose(last, 1, gen)
    p = np.exp(orc.log_softmax(wide(rows)[0, 0]))
    count = np.bincount(tokens.cpu().numpy()[:, 0], minlength=V)
    assert ((count - B * p) ** 2 / (B * p)).sum() < 42   # 9 degrees of freedom
    policy = lambda ids: torch.nn.functional.pad(drafter.logits(ids.reshape(-1)).view(B, 2, V), (0, 6), value=float("nan"))   # noqa: E731
    accepted, out, _, _, _ = d.generate(drafter, policy, last, 1, gen)
    assert (accepted == 1).all() and (out >= 0).all() and (out < V).all() and drafter.err.item() == 0


def test_example(gh, monkeypatch, capsys):
    """The drafter learns: from nothing kept to most of what it proposes."""
    from paper_2602_14338_amd import drafter as d
    monkeypatch.setattr("sys.argv", ["drafter", "--vocab", "1000", "--sequences", "64", "--turns", "120"])
    d.main()
    lines = capsys.readouterr().out.strip().splitlines()
    first, final = ([float(x.split()[-1 if "divergence" in x else 0]) for x in lines[i].split(", ")] for i in (0, -1))
    assert final[0] < 0.2 * first[0] and first[1] < 1.0 and final[1] > 2.0


def test_head_gradient_is_summed_in_32_bits(gh):
    """An fp32 table gradient is the head's product and the lookup's sums of the rounded dz and dx in 32 bits, which the same calls give here: sums of T
    products, n tokens of an id, and the addition."""
    from paper_2602_14338_amd import drafter as d
    rng = np.random.default_rng(8)
    T, V, H, K, scale = 300, 900, 48, 7, 2.0
    table = device(rng.normal(0, 0.3, size=(V, H)).astype(np.float32)).bfloat16()
    ids = rng.integers(0, V, size=T).astype(np.int32)
    index = np.stack([rng.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    lp = np.log(rng.dirichlet(np.ones(K + 1), size=T)[:, :K]).astype(np.float32)
    teacher = d.TeacherLists(device(index), device(lp), None)
    weight = device(rng.random(T).astype(np.float32))
    drafter = d.Drafter(table, scale)
    dtable = torch.full((V, H), 7.0, device="cuda")
    drafter.loss_bwd(device(ids), teacher, weight, dtable)
    x = drafter.hidden(device(ids))
    dz = x @ table.t()
    gh.aero.aero_distill_loss_bwd(dz, T, V, V, teacher.index, teacher.logprob, K, weight, 1, 1.0, torch.empty(1, device="cuda"), None, dz,
                                  torch.empty(gh.aero.aero_workspace_bytes(gh.aero.binding.OP_DISTILL_LOSS_BWD, T=T, V=V), dtype=torch.uint8, device="cuda"))
    dx = dz @ table
    z64, x64 = wide(dz), wide(x)
    lookup, size = orc.embedding_grad(wide(dx), ids, V, scale)
    n = np.bincount(ids, minlength=V)[:, None]
    head, head_size = z64.T @ x64, np.abs(z64.T) @ np.abs(x64)
    bound = 2.0 ** -24 * ((T + 2) * head_size + (n + 2) * size + 2 * np.abs(head + lookup)) + 2.0 ** -126
    assert (np.abs(wide(dtable) - head - lookup) <= bound).all()
