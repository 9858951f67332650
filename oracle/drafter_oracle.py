"""Float64 checker of the calls around a drafter: a teacher's lists, distillation, verification, embedding.  Plain loops over
rows, by the definitions; shares no code with the product.  Logits are widened float64 rows; a logit at or below -1.2e9 (-inf,
say) is masked, one at or above 1.2e9 makes its row NaN as +inf does."""
import numpy as np

MASKED, TOO_LARGE = -1.2e9, 1.2e9


def log_partition(z):
    """log sum exp over the unmasked logits; -inf without any, NaN with a NaN or too large one among them."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or (z >= TOO_LARGE).any():
        return np.nan
    z = z[z > MASKED]
    if z.size == 0:
        return -np.inf
    m = z.max()
    return m + np.log(np.exp(z - m).sum())


def log_softmax(z):
    z = np.asarray(z, np.float64)
    lse = log_partition(z)
    out = np.full(z.shape, -np.inf) if not np.isnan(lse) else np.full(z.shape, np.nan)
    if np.isfinite(lse):
        out[z > MASKED] = z[z > MASKED] - lse
    return out


def top(z, V, K, row_active=None):
    """index [T, K], logprob [T, K], lse [T]."""
    T = len(z)
    index, lp, lse = np.full((T, K), -1, np.int64), np.full((T, K), -np.inf), np.zeros(T)
    for t in range(T):
        if row_active is not None and not row_active[t]:
            lp[t] = 0.0
            continue
        row = np.asarray(z[t][:V], np.float64)
        lse[t] = log_partition(row)
        ids = [j for j in range(V) if row[j] > MASKED] if V <= 4096 else np.nonzero(row > MASKED)[0]
        ids = np.asarray(ids, np.int64)
        ids = ids[np.lexsort((ids, -row[ids]))][:K]
        index[t, :len(ids)] = ids
        lp[t, :len(ids)] = row[ids] - lse[t]
    return index, lp, lse


def distill(z, V, index, logprob, weight, tail, grad_scale):
    """row_loss [T], loss, dlogits [T, V], and for bounds: q [T, V], listed teacher mass by id [T, V], (P, p_r, q_r) [T, 3], bad [T]."""
    T = len(z)
    row_loss, dz = np.zeros(T), np.zeros((T, V))
    q_all, p_all, masses, bad = np.zeros((T, V)), np.zeros((T, V)), np.zeros((T, 3)), np.zeros(T, bool)
    for t in range(T):
        w = float(weight[t])
        if w == 0.0:
            continue
        ids = [int(i) for i in index[t] if i >= 0]
        lp = [float(l) for i, l in zip(index[t], logprob[t]) if i >= 0]
        if any(i >= V for i in ids) or len(set(ids)) != len(ids):
            bad[t] = True
            continue
        p = np.exp(np.asarray(lp, np.float64))
        row = np.asarray(z[t][:V], np.float64)
        if len(ids) == 0 or (not tail and p.sum() == 0.0) or np.isneginf(log_partition(row)):
            continue
        logq = log_softmax(row)
        q = np.exp(logq)
        lse, rest = log_partition(row), log_partition(np.delete(row, ids))
        rest_p = rest_lq = 0.0
        if tail:
            if not np.isneginf(rest):
                rest_p, rest_lq = max(0.0, 1.0 - p.sum()), rest - lse
        else:
            p = p / p.sum()
        total = p.sum() + rest_p
        for k, i in enumerate(ids):
            if p[k] > 0.0:
                row_loss[t] += p[k] * (np.log(p[k]) - logq[i])
        if rest_p > 0.0:
            row_loss[t] += rest_p * (np.log(rest_p) - rest_lq)
        d = total * q
        if rest_p > 0.0:
            others = np.ones(V, bool)
            others[ids] = False
            share = np.where(row[others] > MASKED, np.exp(row[others] - rest), 0.0)
            d[others] -= rest_p * share
        for k, i in enumerate(ids):
            d[i] -= p[k]
            p_all[t, i] = p[k]
        dz[t] = grad_scale * w * d
        q_all[t] = q
        masses[t] = total, rest_p, np.exp(rest_lq) if rest_p > 0.0 else 0.0
    return dict(row_loss=row_loss, loss=float((np.asarray(weight, np.float64) * row_loss).sum()), dlogits=dz, q=q_all, p=p_all, masses=masses,
                bad=bad)


def verify(target, draft, V, draft_tokens, draft_count, uniform, noise):
    """accepted [B], tokens [B, G+1], logprob [B, G+1]; margins: the least relative distance of any decision from
    the other way."""
    B, G = len(target), len(target[0]) - 1
    accepted, tokens, lps = np.zeros(B, np.int64), np.full((B, G + 1), -1, np.int64), np.zeros((B, G + 1))
    margin = np.inf
    for b in range(B):
        count = G if draft_count is None else int(draft_count[b])
        if count < 0 or count > G:
            continue
        for i in range(count):
            if not 0 <= draft_tokens[b][i] < V:
                count = i
                break
        n = 0
        while n < count:
            x = int(draft_tokens[b][n])
            lp = log_softmax(target[b][n][:V])[x]
            lq = log_softmax(draft[b][n][:V])[x] if draft is not None else 0.0
            p, q = np.exp(lp), np.exp(lq)
            usable = np.isfinite(log_partition(draft[b][n][:V])) if draft is not None else True
            if usable and np.isfinite(p):
                margin = min(margin, abs(float(uniform[b][n]) * q - p) / max(p, 1e-300) if p > 0 or q > 0 else np.inf)
            lu = np.log(float(uniform[b][n])) if uniform[b][n] > 0 else -np.inf
            if usable and lu + lq < lp:   # u q < p, also where 64 bits hold neither
                lps[b, n] = lp
                tokens[b, n] = x
                n += 1
            else:
                break
        accepted[b] = n
        row = np.asarray(target[b][n][:V], np.float64)
        if not np.isfinite(log_partition(row)):
            continue
        p = np.exp(log_softmax(row))
        r = p.copy()
        if n < count:
            if draft is None:
                r[int(draft_tokens[b][n])] = 0.0
            elif np.isfinite(log_partition(draft[b][n][:V])):
                r = np.maximum(0.0, p - np.exp(log_softmax(draft[b][n][:V])))
            if not (r > 0.0).any():
                r = p
        score = r / np.asarray(noise[b], np.float64)
        j = int(np.argmax(score))
        if V > 1:
            second = np.partition(score, V - 2)[V - 2]
            margin = min(margin, (score[j] - second) / score[j])
        tokens[b, n] = j
        lps[b, n] = log_softmax(row)[j]
    return dict(accepted=accepted, tokens=tokens, logprob=lps, margin=margin)


def embedding(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            out[t] = scale * np.asarray(table[i], np.float64)
    return out


def embedding_grad(dout, ids, V, scale):
    """dtable [V, H] and, for bounds, the sum of the summands' magnitudes."""
    d, mag = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < V:
            d[i] += scale * np.asarray(dout[t], np.float64)
            mag[i] += np.abs(scale * np.asarray(dout[t], np.float64))
    return d, mag
