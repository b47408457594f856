"""Plain 64-bit forms of the training-side operators, for the tests (no code shared with the
library): policy loss, token sort, gate gradient, SwiGLU with an 8-bit checkpoint."""
import math

import torch

GROUP = 128
TINY = 1e-30


def policy(logits, target, advantage, weight=None, logp_old=None, logp_ref=None, inv_temp=1.0,
           clip_low=0.2, clip_high=0.2, kl_coef=0.0, grad_scale=1.0):
    """loss [4], logp, entropy, grad and ``scale`` (size of each row's gradient terms)."""
    T, V = logits.shape
    z = logits.double() * float(inv_temp)
    w = torch.full((T,), 1.0 / T, dtype=torch.float64) if weight is None else weight.double().cpu()
    loss = [0.0] * 4
    logp, ent = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    grad = torch.zeros(T, V, dtype=torch.float64, device=z.device)
    scale = torch.zeros(T, dtype=torch.float64)
    for t in range(T):
        a, wt = int(target[t]), float(w[t])
        if wt == 0.0 or not 0 <= a < V:
            continue
        if bool((z[t] == -math.inf).all()):
            logp[t] = -math.inf
            continue
        x = z[t] - z[t].max()  # (a row at the type's lowest value is far below its own lse's last bit)
        lp = x - torch.logsumexp(x, 0)
        p = lp.exp()
        logp[t] = lp[a]
        ent[t] = -(p * torch.where(p > 0, lp, 0.0)).sum()
        A = float(advantage[t])
        old = float(logp[t]) if logp_old is None else float(logp_old[t])
        r = math.exp(float(logp[t]) - old)
        lo, hi = 1.0 - clip_low, 1.0 + clip_high
        kept = min(r * A, min(max(r, lo), hi) * A)
        shut = (A > 0 and r > hi) or (A < 0 and r < lo)
        c = 0.0 if shut else -r * A
        kl = 0.0
        if logp_ref is not None:
            gap = float(logp_ref[t]) - float(logp[t])
            kl = math.expm1(gap) - gap
            c -= kl_coef * math.expm1(gap)
        loss[1] -= wt * kept
        loss[2] += wt * kl
        loss[3] += wt * shut
        grad[t] = -p
        grad[t, a] += 1.0
        grad[t] *= grad_scale * inv_temp * wt * c
        scale[t] = abs(wt * inv_temp * grad_scale) * (r * (1 + abs(A)) + (
            0.0 if logp_ref is None else kl_coef * (1 + math.exp(gap))))
    loss[0] = loss[1] + kl_coef * loss[2]
    return dict(loss=torch.tensor(loss, dtype=torch.float64), logp=logp, entropy=ent, grad=grad,
                scale=scale)


def plan(idx, N):
    """offsets, perm, inv of the stable sort by expert (lists; -1 as in the library)."""
    T, k = len(idx), len(idx[0]) if len(idx) else 0
    slots = []
    for t in range(T):
        for s in range(k):
            e = idx[t][s]
            if 0 <= e < N and e not in idx[t][:s]:
                slots.append((e, t * k + s))
    slots.sort()  # by expert, then slot
    perm = [f for _, f in slots] + [-1] * (T * k - len(slots))
    inv = [-1] * (T * k)
    for r, (_, f) in enumerate(slots):
        inv[f] = r
    offsets = [sum(1 for e, _ in slots if e < x) for x in range(N + 1)]
    return offsets, perm, inv


def rows_of(x, inv, T, k):
    """The row of each slot [T, k, d] in 64 bits; zero for an invalid slot."""
    at = inv.reshape(T, k).long()
    got = x.double()[at.clamp(min=0)]
    return torch.where((at >= 0)[..., None], got, 0.0)


def gates_backward(probs, idx, dgates, norm):
    T, N = probs.shape
    k = idx.shape[1]
    rho = probs.double()
    out = torch.zeros(T, N, dtype=torch.float64)
    for t in range(T):
        row = idx[t].tolist()
        ok = [s for s in range(k) if 0 <= row[s] < N and row[s] not in row[:s]]
        if not ok:
            continue
        total = sum(float(rho[t, row[s]]) for s in ok) if norm else 1.0
        if total == 0.0:
            continue
        jac = torch.zeros(len(ok), N, dtype=torch.float64)  # d rho_s / d p_j
        for i, s in enumerate(ok):
            jac[i] = -rho[t, row[s]] * rho[t]
            jac[i, row[s]] += rho[t, row[s]]
        if norm:  # d (rho_s / S)
            g = torch.tensor([float(rho[t, row[s]]) for s in ok], dtype=torch.float64) / total
            jac = (jac - g[:, None] * jac.sum(0)) / total
        out[t] = dgates[t, ok].double() @ jac
    return out


def hold(x):
    """(q, scale) of fp32 rows [R, m] by the format's own 32-bit roundings (CPU, IEEE)."""
    x = x.float().cpu()
    R, m = x.shape
    G = -(-m // GROUP)
    q, scale = torch.zeros(R, m, dtype=torch.int8), torch.zeros(R, G)
    inv127 = torch.tensor(1 / 127, dtype=torch.float32)
    for g in range(G):
        v = x[:, g * GROUP:(g + 1) * GROUP]
        top = v.abs().amax(1)
        bad = ~torch.isfinite(v).all(1)
        live = (top >= TINY) & ~bad
        f = torch.where(live, torch.full_like(top, 127.0) / top, torch.zeros_like(top))
        q[:, g * GROUP:(g + 1) * GROUP] = torch.where(
            live[:, None], torch.round(v * f[:, None]), torch.zeros_like(v)).to(torch.int8)
        scale[:, g] = torch.where(bad, torch.full_like(top, math.nan),
                                  torch.where(live, top * inv127, torch.zeros_like(top)))
    return q, scale


def held(q, scale):
    m = q.shape[1]
    return q.double() * scale.double()[:, torch.arange(m) // GROUP]


def swiglu(g, u):
    return g * torch.sigmoid(g) * u


def swiglu_backward(g, u, d):
    s = torch.sigmoid(g)
    return d * u * s * (1 + g * (1 - s)), d * g * s, g * s * u
