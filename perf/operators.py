"""The work that keeping a drafter close to the policy, and drafting with it, has this library do, as timed and
checked cases.

Five kinds, one per public call:

  topk       the K largest logits of each of the policy's rows, as ids and log-probs (a teacher's lists)
  distill    divergence of a drafter's rows from such lists, and its gradient with respect to the drafter's logits
  verify     drafted tokens against the policy's rows: how many are accepted, the token drawn after them, log-probs
  embed_fwd  the drafter's input rows, looked up and scaled
  embed_bwd  their gradient with respect to the table, by sorted tokens

With ``own`` false a pass is elementary tensor operations in 32 bits, with it true the library's calls.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2, "f8": 1}
_CHUNK = 1 << 27   # logits handled at a time outside the timed pass
_SIGMA = 3.0       # spread of a row's logits
_MISS = 0.5        # spread of the drafter's logits around the policy's: four of five drafted tokens are accepted
_ACCEPT = 0.8
_COPIED = 0.7      # what the policy gives a token copied from another rollout


def listed():
    return [
        # lists at one position of each of 64 sequences under way: the smallest call, a fraction of the CUs
        dict(name="topk_positions", kind="topk", dtype="bf16", T=64, V=151936, ld=151936, K=64),
        # lists of a micro-batch of rollout tokens
        dict(name="topk_rollouts", kind="topk", dtype="bf16", T=4096, V=151936, ld=151936, K=64),
        # a small drafter in single precision: 4 queries x 8 rollouts x 64 tokens
        dict(name="distill_f32_small", kind="distill", dtype="f32", T=2048, V=1024, ld=1024, K=16, tail=0),
        # an odd vocabulary whose rows are not 16-byte aligned, a few hundred tokens
        dict(name="distill_odd_vocab", kind="distill", dtype="bf16", T=500, V=50257, ld=50257, K=50, tail=1),
        # half precision with a 32K vocabulary, lists renormalised
        dict(name="distill_f16_32k", kind="distill", dtype="f16", T=8192, V=32000, ld=32000, K=32, tail=0),
        # the training micro-batch: 8K packed tokens against the whole vocabulary, the rest of it in one bucket
        dict(name="distill_rollouts", kind="distill", dtype="bf16", T=8192, V=151936, ld=151936, K=64, tail=1),
        # one query's group of 8 rollouts being generated, 4 tokens drafted each: latency counts
        dict(name="verify_group", kind="verify", dtype="bf16", B=8, G=4, V=151936, ld=151936, ragged=0, probs=1),
        # 128 rollouts being generated, up to 5 drafted tokens, some sequences with fewer or none
        dict(name="verify_batch", kind="verify", dtype="bf16", B=128, G=5, V=151936, ld=151936, ragged=1, probs=1),
        # tokens copied from the rollouts of the same query: a drafter that has no probabilities
        dict(name="verify_copied", kind="verify", dtype="bf16", B=256, G=3, V=151936, ld=151936, ragged=0, probs=0),
        # input rows of a packed micro-batch
        dict(name="embed_fwd_16k", kind="embed_fwd", dtype="bf16", T=16384, V=151936, H=1536),
        # gradient of a few hundred tokens with respect to the whole table
        dict(name="embed_bwd_small", kind="embed_bwd", dtype="bf16", T=600, V=151936, H=1536, grad="bf16"),
        # gradient of 32K packed tokens, most of a smaller table's rows among them
        dict(name="embed_bwd_32k", kind="embed_bwd", dtype="bf16", T=32768, V=32000, H=3584, grad="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["topk", "topk", "distill", "distill", "distill", "verify", "verify", "embed_fwd", "embed_bwd", "embed_bwd"])
    V = _log_int(rng, 1000, 152064) if rng.random() < 0.6 else rng.choice([1024, 32000, 50257, 151936, 152064])
    if kind.startswith("embed"):
        H = 8 * _log_int(rng, 8, 448) if rng.random() < 0.7 else _log_int(rng, 64, 3584)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        T = _log_int(rng, 1, 32768 if dtype != "f32" else 16384)
        case = dict(kind=kind, dtype=dtype, T=T, V=V, H=H)
        if kind == "embed_bwd":
            case["grad"] = rng.choice(["f32", "bf16"])
        return case
    ld = V if rng.random() < 0.5 else (V + 63) // 64 * 64
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"] + (["f8"] if kind != "distill" else []))
    if kind == "verify":
        G = rng.randint(1, 8)
        probs = int(rng.random() < 0.7)
        return dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, max(1, min(256, 900 // G))), G=G, V=V, ld=ld,
                    ragged=rng.randint(0, 1), probs=probs)
    room = 620000000 if kind == "topk" else 600000000
    case = dict(kind=kind, dtype=dtype, T=_log_int(rng, 1, min(8192, room // V)), V=V, ld=ld, K=_log_int(rng, 1, 128))
    if kind == "distill":
        case["tail"] = rng.randint(0, 1)
    return case


# ---------------------------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 16 + stream)
    return g


def _chunks(T, V):
    step = max(1, _CHUNK // V)
    return [(a, min(T, a + step)) for a in range(0, T, step)]


def _rows(case, T, gen, around=None, spread=_SIGMA):
    """[T, ld] logits: normal, or normal around other rows; what lies behind column V is never read."""
    V, ld, dtype = case["V"], case["ld"], _TORCH[case["dtype"]]
    out = torch.empty((T, ld), dtype=dtype, device="cuda")
    for a, b in _chunks(T, V):
        z = torch.randn((b - a, ld), generator=gen, device="cuda") * spread
        if around is not None:
            z += around[a:b].float()
        out[a:b] = z.to(dtype)
    return out


def _key(z):
    """Whole numbers in the order of (logit, lowest id first): -0 and 0 are the same logit."""
    bits = (z + 0.0).view(torch.int32).to(torch.int64)
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return (bits << 24) + (z.shape[1] - 1 - torch.arange(z.shape[1], device=z.device))


def _top(z, K):
    """Ids of the K largest of each row of 32-bit logits, the lowest id first where logits are equal."""
    key = torch.topk(_key(z), K, dim=1, sorted=True).values
    return z.shape[1] - 1 - (key & 0xffffff)


def _grad_scale(case):
    """Gradients of half precision are lifted into its range; a token's weight is about 1 / T."""
    return 2.0 ** math.floor(math.log2(256 * case["T"])) if case["dtype"] == "f16" else 1.0


def prepare(case, seed):
    kind, dtype = case["kind"], _TORCH[case["dtype"]]
    V = case["V"]
    st = dict(case=case)
    if kind in ("embed_fwd", "embed_bwd"):
        T, H = case["T"], case["H"]
        # frequencies fall with the rank as 1 / rank: one token in 16 is the commonest; one position in 20 is padding
        g = _gen(seed, 0)
        rank = torch.exp(torch.rand(T, generator=g, device="cuda") * math.log(V)).long().clamp_(1, V) - 1
        ids = torch.randperm(V, generator=g, device="cuda")[rank]
        pad = torch.rand(T, generator=g, device="cuda") < 0.05
        st["ids"] = torch.where(pad, -1, ids).to(torch.int32)
        st["scale"] = math.sqrt(H)
        if kind == "embed_fwd":
            st["table"] = (torch.randn((V, H), generator=_gen(seed, 1), device="cuda") * 0.02).to(dtype)
            if own:
                st["out"] = torch.empty((T, H), dtype=dtype, device="cuda")
        else:
            st["dout"] = (torch.randn((T, H), generator=_gen(seed, 1), device="cuda") * 1e-3).to(dtype)
            if own:
                from paper_2602_14338_amd import aero_workspace_bytes, binding
                st["dtable"] = torch.empty((V, H), dtype=_TORCH[case["grad"]], device="cuda")
                size = aero_workspace_bytes(binding.OP_EMBEDDING_BWD, T=T, V=V, H=H)
                st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return st
    if kind == "topk":
        T, K = case["T"], case["K"]
        st["logits"] = _rows(case, T, _gen(seed, 0))
        if own:
            st["index"] = torch.empty((T, K), dtype=torch.int32, device="cuda")
            st["logprob"] = torch.empty((T, K), device="cuda")
            st["lse"] = torch.empty(T, device="cuda")
            from paper_2602_14338_amd import aero_workspace_bytes, binding
            size = aero_workspace_bytes(binding.OP_TOPK_LOGPROB, T=T, V=V, H=K)
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return st
    if kind == "distill":
        T, K = case["T"], case["K"]
        teacher = _rows(case, T, _gen(seed, 0))
        index, logprob = [], []
        for a, b in _chunks(T, V):
            z = teacher[a:b, :V].float()
            top = _top(z, K)
            index.append(top.to(torch.int32))
            logprob.append(z.gather(1, top) - torch.logsumexp(z, dim=1, keepdim=True))
        st["index"], st["logprob"] = torch.cat(index), torch.cat(logprob)
        st["logits"] = _rows(case, T, _gen(seed, 1), teacher, _MISS)
        # one token in eight is padding; the others weigh the same
        keep = torch.rand(T, generator=_gen(seed, 2), device="cuda") >= 0.125
        st["weight"] = keep.float() / T
        if own:
            from paper_2602_14338_amd import aero_workspace_bytes, binding
            st["loss"], st["row_loss"] = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
            st["dlogits"] = torch.empty_like(st["logits"]) if case["ld"] == V else torch.zeros_like(st["logits"])
            size = aero_workspace_bytes(binding.OP_DISTILL_LOSS_BWD, T=T, V=V)
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return st
    # verify: B sequences, G positions of the drafter and one more of the policy; noise of the race that draws a token
    B, G = case["B"], case["G"]
    st["target"] = _rows(case, B * (G + 1), _gen(seed, 0)).view(B, G + 1, case["ld"])
    st["noise"] = torch.empty((B, V), device="cuda").exponential_(generator=_gen(seed, 3)).clamp_(min=1e-30)
    st["uniform"] = torch.rand((B, G), generator=_gen(seed, 4), device="cuda")
    around = st["target"][:, :G].reshape(B * G, case["ld"])
    draft = _rows(case, B * G, _gen(seed, 1), around, _MISS)
    tokens, g = [], _gen(seed, 2)
    for a, b in _chunks(B * G, V):
        z = draft[a:b, :V].float()
        race = torch.empty_like(z).exponential_(generator=g).clamp_(min=1e-30)
        tokens.append(torch.argmax(torch.exp(z - z.max(dim=1, keepdim=True).values) / race, dim=1))
    st["tokens"] = torch.cat(tokens).to(torch.int32).view(B, G)
    st["draft"] = draft.view(B, G, case["ld"]) if case["probs"] else None
    if not case["probs"]:
        lse = math.log(V) + _SIGMA ** 2 / 2   # of the other logits
        rows = torch.arange(B * G, device="cuda")
        st["target"][rows // G, rows % G, st["tokens"].reshape(-1).long()] = lse + math.log(_COPIED / (1 - _COPIED))
    st["count"] = torch.randint(0, G + 1, (B,), generator=_gen(seed, 5), device="cuda", dtype=torch.int32) if case["ragged"] \
        else torch.full((B,), G, dtype=torch.int32, device="cuda")
    if own:
        from paper_2602_14338_amd import aero_workspace_bytes, binding
        st["accepted"] = torch.empty(B, dtype=torch.int32, device="cuda")
        st["out"] = torch.empty((B, G + 1), dtype=torch.int32, device="cuda")
        st["out_logprob"] = torch.empty((B, G + 1), device="cuda")
        size = aero_workspace_bytes(binding.OP_VERIFY_DRAFT, T=B * (G + 1), V=V, Q=B)
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------- one pass
def run(st):
    return _run_own(st) if own else _PLAIN[st["case"]["kind"]](st)


def _run_own(st):
    import paper_2602_14338_amd as aero
    case = st["case"]
    kind, V = case["kind"], case["V"]
    if kind == "topk":
        aero.aero_topk_logprob(st["logits"], case["T"], V, case["ld"], None, case["K"], st["index"], st["logprob"], st["lse"],
                               st["workspace"])
        return st["index"], st["logprob"], st["lse"]
    if kind == "distill":
        aero.aero_distill_loss_bwd(st["logits"], case["T"], V, case["ld"], st["index"], st["logprob"], case["K"], st["weight"],
                                   case["tail"], _grad_scale(case), st["loss"], st["row_loss"], st["dlogits"], st["workspace"])
        return st["loss"], st["row_loss"], st["dlogits"][:, :V]
    if kind == "verify":
        aero.aero_verify_draft(st["target"], st["draft"], case["B"], case["G"], V, case["ld"], st["tokens"], st["count"],
                               st["uniform"], st["noise"], st["accepted"], st["out"], st["out_logprob"], st["workspace"])
        return st["accepted"], st["out"], st["out_logprob"]
    if kind == "embed_fwd":
        aero.aero_embedding_fwd(st["table"], V, case["H"], st["ids"], case["T"], st["scale"], st["out"], case["H"])
        return st["out"]
    aero.aero_embedding_bwd(st["dout"], case["T"], case["H"], case["H"], st["ids"], V, st["scale"], st["dtable"], st["workspace"])
    return st["dtable"]


def _plain_topk(st):
    case = st["case"]
    z = st["logits"][:, :case["V"]].float()
    top = _top(z, case["K"])
    m = z.max(dim=1, keepdim=True).values
    lse = m + torch.log(torch.exp(z - m).sum(dim=1, keepdim=True))
    return top.to(torch.int32), z.gather(1, top) - lse, lse[:, 0]


def _plain_distill(st):
    case = st["case"]
    z = st["logits"][:, :case["V"]].float()
    i, l, w = st["index"].long(), st["logprob"], st["weight"][:, None]
    m = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - m)
    s = e.sum(dim=1, keepdim=True)
    logq = z.gather(1, i) - m - torch.log(s)
    q = e / s
    p = torch.exp(l)
    if case["tail"]:
        rest_q = (e.scatter(1, i, 0.0).sum(dim=1, keepdim=True)) / s
        rest_p = (1.0 - p.sum(dim=1, keepdim=True)).clamp(min=0.0)
        row = (p * (l - logq)).sum(dim=1, keepdim=True) + torch.where(
            rest_p > 0, rest_p * (torch.log(rest_p) - torch.log(rest_q)), 0.0)
        total = p.sum(dim=1, keepdim=True) + rest_p
        dz = q * (total - rest_p / rest_q)
        dz.scatter_(1, i, total * q.gather(1, i) - p)
    else:
        total = p.sum(dim=1, keepdim=True)
        p = p / total
        row = (p * (l - torch.log(total) - logq)).sum(dim=1, keepdim=True)
        dz = q
        dz.scatter_add_(1, i, -p)
    row = torch.where(w != 0, row, 0.0)
    return (w * row).sum().reshape(1), row[:, 0], (dz * (w * _grad_scale(case))).to(st["logits"].dtype)


def _plain_verify(st):
    case = st["case"]
    B, G, V = case["B"], case["G"], case["V"]
    z = st["target"][:, :, :V].float()
    m = z.max(dim=2, keepdim=True).values
    lse = m + torch.log(torch.exp(z - m).sum(dim=2, keepdim=True))
    x = st["tokens"].long()[:, :, None]
    logp = (z - lse)
    own_p = torch.exp(logp[:, :G].gather(2, x))[:, :, 0]
    if st["draft"] is not None:
        q = torch.softmax(st["draft"][:, :, :V].float(), dim=2)
        own_q = q.gather(2, x)[:, :, 0]
    else:
        own_q = torch.ones_like(own_p)
    place = torch.arange(G + 1, device=z.device)[None, :]
    ok = (st["uniform"] * own_q < own_p) & (place[:, :G] < st["count"][:, None])
    n = torch.cumprod(ok.int(), dim=1).sum(dim=1)
    each = torch.arange(B, device=z.device)
    p = torch.exp(logp[each, n])
    refused = (n < st["count"])[:, None]
    at = n.clamp(max=G - 1)
    if st["draft"] is not None:
        less = q[each, at]
    else:
        less = torch.zeros_like(p).scatter_(1, x[each, at], torch.inf)
    left = torch.where(refused, (p - less).clamp(min=0.0), p)
    left = torch.where((left > 0).any(dim=1, keepdim=True), left, p)
    drawn = torch.argmax(left / st["noise"], dim=1)
    filled = torch.cat([st["tokens"].long(), torch.zeros((B, 1), dtype=torch.int64, device=z.device)], dim=1)
    tokens = torch.where(place < n[:, None], filled, torch.where(place == n[:, None], drawn[:, None], -1))
    lp = logp.gather(2, tokens.clamp(min=0)[:, :, None])[:, :, 0]
    return n.to(torch.int32), tokens.to(torch.int32), torch.where(tokens >= 0, lp, 0.0)


def _plain_embed_fwd(st):
    ids = st["ids"].long()
    rows = st["table"][ids.clamp(min=0)].float() * st["scale"]
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(st["table"].dtype)


def _plain_embed_bwd(st):
    case = st["case"]
    ids = st["ids"].long()
    rows = torch.where(ids[:, None] >= 0, st["dout"].float() * st["scale"], 0.0)
    total = torch.zeros((case["V"], case["H"]), device=rows.device)
    total.index_add_(0, ids.clamp(min=0), rows)
    return total.to(_TORCH[case["grad"]])


_PLAIN = {"topk": _plain_topk, "distill": _plain_distill, "verify": _plain_verify, "embed_fwd": _plain_embed_fwd,
          "embed_bwd": _plain_embed_bwd}


# ---------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind, V = case["kind"], case["V"]
    if kind == "embed_fwd":
        ids = st["ids"].long()
        out = torch.zeros((case["T"], case["H"]), dtype=torch.float64, device="cuda")
        there = ids >= 0
        out[there] = st["table"].double()[ids[there]] * st["scale"]
        return out
    if kind == "embed_bwd":
        ids = st["ids"].long()
        there = ids >= 0
        out = torch.zeros((V, case["H"]), dtype=torch.float64, device="cuda")
        out.index_put_((ids[there],), st["dout"].double()[there] * st["scale"], accumulate=True)
        return out
    if kind == "topk":
        T, K = case["T"], case["K"]
        lp, lse = torch.empty((T, K), dtype=torch.float64, device="cuda"), torch.empty(T, dtype=torch.float64, device="cuda")
        for a, b in _chunks(T, V):
            z = st["logits"][a:b, :V].double()
            lse[a:b] = torch.logsumexp(z, dim=1)
            lp[a:b] = torch.sort(z, dim=1, descending=True).values[:, :K] - lse[a:b, None]
        return None, lp, lse
    if kind == "distill":
        T = case["T"]
        row = torch.zeros(T, dtype=torch.float64, device="cuda")
        grad = torch.empty((T, V), dtype=torch.float64, device="cuda")
        for a, b in _chunks(T, V):
            i, w = st["index"][a:b].long(), st["weight"][a:b].double()
            logq = torch.log_softmax(st["logits"][a:b, :V].double(), dim=1)
            p = torch.exp(st["logprob"][a:b].double())
            listed_q = logq.gather(1, i)
            q = torch.exp(logq)
            if case["tail"]:
                rest_p = torch.clamp(1.0 - p.sum(1), min=0.0)
                rest_q = q.scatter(1, i, 0.0).sum(1)
                mass = p.sum(1) + rest_p
                value = (p * (torch.log(p) - listed_q)).sum(1) + torch.xlogy(rest_p, rest_p / rest_q)
                dz = q * (mass - rest_p / rest_q)[:, None]
            else:
                p = p / p.sum(1, keepdim=True)
                mass = torch.ones_like(w)
                value = (p * (torch.log(p) - listed_q)).sum(1)
                dz = q
            dz = dz.scatter(1, i, mass[:, None] * torch.exp(listed_q) - p)
            grad[a:b] = dz * (w * _grad_scale(case))[:, None]
            row[a:b] = torch.where(w != 0, value, 0.0)
        return (row * st["weight"].double()).sum().reshape(1), row, grad
    # verify: the log-probs of the tokens that come out follow from which tokens they are
    B, G = case["B"], case["G"]
    accepted = torch.zeros(B, dtype=torch.int32, device="cuda")
    tokens = torch.full((B, G + 1), -1, dtype=torch.int32, device="cuda")
    lp = torch.zeros((B, G + 1), dtype=torch.float64, device="cuda")
    counts, drafted, u = st["count"].tolist(), st["tokens"].tolist(), st["uniform"].double().tolist()
    for b in range(B):
        logp = torch.log_softmax(st["target"][b, :, :V].double(), dim=1)
        q = torch.softmax(st["draft"][b, :, :V].double(), dim=1) if st["draft"] is not None else None
        x = torch.tensor(drafted[b], device="cuda")[:, None]
        own_lp = logp[:G].gather(1, x)[:, 0]
        own_q = (q.gather(1, x)[:, 0] if q is not None else torch.ones_like(own_lp)).tolist()
        own_p = torch.exp(own_lp).tolist()
        n = 0
        while n < counts[b] and u[b][n] * own_q[n] < own_p[n]:
            n += 1
        left = torch.exp(logp[n])
        if n < counts[b]:
            if q is not None:
                left = torch.clamp(left - q[n], min=0.0)
            else:
                left[drafted[b][n]] = 0.0
        drawn = torch.argmax(left / st["noise"][b].double())
        accepted[b] = n
        tokens[b, :n] = st["tokens"][b, :n]
        tokens[b, n] = drawn
        lp[b, :n] = own_lp[:n]
        lp[b, n] = logp[n, drawn]
    return accepted, tokens, lp


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Bytes: each input read once, each output written once.  flops: an exponential, its product and its sum per logit
    and their like."""
    kind, V = case["kind"], case["V"]
    if kind == "embed_fwd":   # padding rows are not read
        e = _BYTES[case["dtype"]] * case["T"] * case["H"]
        return {"bytes": 0.95 * e + e + 4 * case["T"], "flops": case["T"] * case["H"]}
    if kind == "embed_bwd":
        e = _BYTES[case["dtype"]] * case["T"] * case["H"]
        return {"bytes": 0.95 * e + _BYTES[case["grad"]] * V * case["H"] + 4 * case["T"], "flops": 2 * case["T"] * case["H"]}
    e = _BYTES[case["dtype"]]
    if kind == "topk":
        T, K = case["T"], case["K"]
        return {"bytes": T * V * e + T * K * 8 + T * 4, "flops": 4 * T * V}
    if kind == "distill":   # rows without weight are only written
        T, K = case["T"], case["K"]
        return {"bytes": 0.875 * T * V * e + T * V * e + T * K * 8 + T * 8, "flops": 7 * 0.875 * T * V}
    # verify: the rows up to the first refusal, which the drafter's share of accepted tokens sets, and one row of noise
    B, G = case["B"], case["G"]
    counts = range(G + 1) if case["ragged"] else [G]
    accept = _ACCEPT if case["probs"] else _COPIED
    target = sum(sum(accept ** i for i in range(c + 1)) for c in counts) / len(counts)
    draft = sum(sum(accept ** i for i in range(c)) for c in counts) / len(counts) if case["probs"] else 0.0
    rows = B * (target + draft)
    return {"bytes": rows * V * e + B * V * 4 + B * (G + 1) * 16, "flops": 4 * rows * V + 8 * B * V}
