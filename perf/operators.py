"""Cases of the training-side operators: what they compute in plain form, and how a user calls them.

Operators (one pass each):
  policy      clipped policy loss with a KL term over a vocabulary, with or without the gradient
              of the logits
  sort        tokens sorted by expert: the plan (offsets, perm, inv) and the sorted rows
  unsort      expert rows back to token order, weighted by the gates
  unsort_grad gradient of that: expert rows and gates
  sort_grad   gradient of the sort: token rows
  act_step    SwiGLU activation that keeps its inputs in 8 bits, then its backward pass from them
  act_grad    that backward pass alone
  gates_grad  gradient of the replay gates w.r.t. the router logits

`own` False: plain torch operations in 32 bits; True: the framework's entry points.
"""
import math

import torch

own = False

_GROUP = 128  # elements that share a scale of the 8-bit checkpoint
_TINY = 1e-30  # groups whose largest magnitude is below this are held as zeros
_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp32": 4}
_binding = None


def _lib():
    global _binding
    if _binding is None:
        from paper_2606_00395_gb300 import binding
        _binding = binding
    return _binding


# ---- cases ------------------------------------------------------------------------------------

def _policy(T, V, dtype="bf16", grad=True, pad=0, beta=0.05, temp=1.0, masked=0.1, banned=0.0):
    return dict(kind="policy", T=T, V=V, dtype=dtype, grad=grad, pad=pad, beta=beta, temp=temp,
                masked=masked, banned=banned)


def _tokens(kind, T, d, N, k, dtype="bf16", zipf=0.0, masked=0.0):
    return dict(kind=kind, T=T, d=d, N=N, k=k, dtype=dtype, zipf=zipf, masked=masked)


def _act(kind, rows, m, dtype="bf16", fused=True):
    return dict(kind=kind, rows=rows, m=m, dtype=dtype, fused=fused)


def _gates(T, N, k, norm):
    return dict(kind="gates_grad", T=T, N=N, k=k, norm=norm)


def listed():
    return [
        # the log-probability, loss and gradient of a single token: latency
        dict(_policy(1, 32001, masked=0.0, beta=0.0), name="policy_one_token"),
        # a training micro-batch: loss and gradient over a large vocabulary
        dict(_policy(4096, 131072), name="policy_train"),
        # scoring pass (log-probabilities, entropy and loss, no gradient), padded vocabulary
        dict(_policy(2048, 65000, grad=False, pad=536, temp=0.8), name="policy_score"),
        # exact-fp32 logits, odd vocabulary (rows start at any element), banned entries at -inf
        dict(_policy(517, 50001, dtype="fp32", masked=0.3, banned=0.01), name="policy_fp32_odd"),
        # a decode-sized batch of the Qwen3-shaped layer: plan and rows, latency
        dict(_tokens("sort", 256, 2048, 128, 8), name="sort_small"),
        # long replay batch with skewed routes and some padding tokens
        dict(_tokens("sort", 32768, 2048, 128, 8, zipf=1.2, masked=0.05), name="sort_long"),
        # the Qwen3-shaped training batch: weighted rows back to tokens
        dict(_tokens("unsort", 4096, 2048, 128, 8), name="unsort_train"),
        # the DeepSeek-V3-shaped layer's backward: expert rows' and gates' gradients
        dict(_tokens("unsort_grad", 8192, 7168, 256, 8), name="unsort_grad_wide"),
        # a small fp32 layer with a ragged batch and an odd width
        dict(_tokens("sort_grad", 1001, 1023, 60, 4, dtype="fp32", masked=0.1), name="sort_grad_odd"),
        # activations of the Qwen3-shaped experts for a training batch, forward and backward
        dict(_act("act_step", 32768, 768), name="act_step_train"),
        # an odd fp32 layer's backward from the checkpoint, gate and up held apart
        dict(_act("act_grad", 1777, 1001, dtype="fp32", fused=False), name="act_grad_odd"),
        # the router's gradient of a training batch
        dict(_gates(4096, 128, 8, False), name="gates_grad_train"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: half the time one that models use, else any odd one."""
    if rng.random() < 0.5:
        return rng.choice([w for w in (64, 128, 256, 512, 768, 1024, 2048, 4096, 7168) if lo <= w <= hi])
    return min(hi - 1 + hi % 2, _log(rng, lo, hi) | 1)


def draw(rng):
    most = 2 * 4096 * 131072 * 2 * 1.001
    while True:
        kind = rng.choice(["policy", "policy", "sort", "unsort", "unsort_grad", "sort_grad", "act_step",
                           "act_grad", "gates_grad"])
        dtype = "bf16" if rng.random() < 0.7 else "fp32"
        if kind == "policy":
            V = _log(rng, 1000, 200000)
            case = _policy(_log(rng, 1, 8192), V, dtype, rng.random() < 0.7, rng.choice([0, 0, 1, -V % 64]),
                           rng.choice([0.0, 0.01, 0.05]), rng.choice([0.7, 1.0, 1.3]),
                           rng.choice([0.0, 0.1, 0.4]), rng.choice([0.0, 0.01]))
            if case["T"] * V > 4096 * 131072:
                continue
        elif kind.startswith("act"):
            case = _act(kind, _log(rng, 1, 262144), _width(rng, 64, 4096), dtype, rng.random() < 0.5)
        elif kind == "gates_grad":
            N = rng.choice([8, 60, 64, 128, 160, 256])
            case = _gates(_log(rng, 1, 65536), N, rng.randint(1, 8), rng.random() < 0.5)
        else:
            N = rng.choice([8, 60, 64, 128, 160, 256])
            case = _tokens(kind, _log(rng, 1, 32768), _width(rng, 64, 7168), N, rng.randint(1, 8), dtype,
                           rng.choice([0.0, 0.0, 1.2]), rng.choice([0.0, 0.05]))
        if work(case)["bytes"] <= most:
            return case


def work(case):
    c = case
    if c["kind"] == "policy":
        n, es = c["T"] * c["V"], _ES[c["dtype"]]
        live = n * (1.0 - c["masked"])  # tokens that do not count are not read
        return {"bytes": live * es + (n * es if c["grad"] else 0) + 4 * 6 * c["T"],
                "flops": live * (8 + (4 if c["grad"] else 0))}
    if c["kind"].startswith("act"):
        n, es = c["rows"] * c["m"], _ES[c["dtype"]]
        held = 2 * n + 8 * c["rows"] * -(-c["m"] // _GROUP)
        back = held + n * es + 3 * n * es  # checkpoint, d(act) read; d(gate), d(up), act written
        if c["kind"] == "act_grad":
            return {"bytes": back, "flops": 16 * n}
        return {"bytes": 3 * n * es + held + back, "flops": 32 * n}
    if c["kind"] == "gates_grad":
        return {"bytes": 8 * c["T"] * c["N"] + 8 * c["T"] * c["k"], "flops": 3 * c["T"] * c["N"]}
    es, T, k, d = _ES[c["dtype"]], c["T"], c["k"], c["d"]
    rows, toks = T * k * d * es, T * d * es
    live = rows * (1.0 - c["masked"])
    if c["kind"] == "sort":
        return {"bytes": toks + rows + 12 * T * k + 4 * c["N"], "flops": 0}
    if c["kind"] == "sort_grad":
        return {"bytes": live + toks + 4 * T * k, "flops": T * k * d}
    if c["kind"] == "unsort":
        return {"bytes": live + toks + 8 * T * k, "flops": 2 * T * k * d}
    return {"bytes": live + toks + rows + 12 * T * k, "flops": 3 * T * k * d}


# ---- inputs -----------------------------------------------------------------------------------

def _route(c, g):
    """k distinct experts per token, skewed by (e + 1)^-zipf (Gumbel top-k); a padding token's
    entries are -1."""
    u = torch.rand(c["T"], c["N"], generator=g, device="cuda").clamp_(1e-12, 1 - 1e-7)
    rank = torch.arange(1, c["N"] + 1, device="cuda").float().log()
    score = -torch.log(-torch.log(u)) - c.get("zipf", 0.0) * rank
    idx = score.topk(c["k"], dim=1).indices.int()
    if c.get("masked", 0.0):
        idx[torch.rand(c["T"], generator=g, device="cuda") < c["masked"]] = -1
    return idx.contiguous()


def _plan(idx, N):
    """offsets [N + 1], perm [T k] (-1 past the last valid slot) and inv [T k] (-1: invalid slot)
    of the stable sort of the flat slots by expert."""
    flat = idx.reshape(-1).long()
    ok = (flat >= 0) & (flat < N)
    key = torch.where(ok, flat, N)
    ranked, order = torch.sort(key, stable=True)
    at = torch.arange(flat.numel(), device=idx.device)
    offsets = torch.searchsorted(ranked, torch.arange(N + 1, device=idx.device)).int()
    perm = torch.where(at < offsets[N], order, -1).int()
    inv = torch.empty_like(order)
    inv[order] = at
    return offsets, perm, torch.where(ok, inv, -1).int()


def _groups(x):
    """[R, m] as [R, groups, _GROUP] with zeros past m."""
    R, m = x.shape
    G = -(-m // _GROUP)
    if G * _GROUP != m:
        x = torch.nn.functional.pad(x, (0, G * _GROUP - m))
    return x.reshape(R, G, _GROUP)


def _hold(x):
    """The 8-bit form of fp32 [R, m]: integers (as fp32, [R, m]) and scales [R, groups]."""
    v = _groups(x)
    top = v.abs().amax(-1)
    live = top >= _TINY
    r = torch.where(live, torch.div(torch.full_like(top, 127.0), top), 0.0)
    q = torch.round(v * r[..., None]).reshape(x.shape[0], -1)[:, :x.shape[1]]
    return q, torch.where(live, top * torch.full_like(top, 1 / 127), 0.0)


def _held(q, scale):
    """The values that integers [R, m] with scales [R, groups] stand for, in the scales' type."""
    m = q.shape[1]
    return (_groups(q.to(scale.dtype)) * scale[..., None]).reshape(q.shape[0], -1)[:, :m]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    s = {"case": c}

    def randn(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    def out(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    dt = _DT[c["dtype"]] if "dtype" in c else torch.float32
    if c["kind"] == "policy":
        T, V = c["T"], c["V"]
        ld = V + c["pad"]
        logits = torch.empty(T, ld, dtype=dt, device="cuda")
        target = torch.randint(0, V, (T,), generator=g, device="cuda")
        bonus = 12 * torch.rand(T, generator=g, device="cuda")  # sampled tokens are likely ones
        logp = torch.empty(T, device="cuda")
        step = max(1, (1 << 27) // ld)
        for a in range(0, T, step):
            b = min(T, a + step)
            z = randn(b - a, ld, std=2.0)
            if c["banned"]:
                z[torch.rand(b - a, ld, generator=g, device="cuda") < c["banned"]] = -math.inf
            at = torch.arange(b - a, device="cuda")
            z[at, target[a:b]] = bonus[a:b]
            logits[a:b] = z.to(dt)
            z = logits[a:b, :V].float() / c["temp"]
            logp[a:b] = z[at, target[a:b]] - torch.logsumexp(z, 1)
        # the behaviour policy is a few steps old; ratios right at a clip bound are left out, where
        # a last-bit difference of a log-probability switches a gradient on or off
        drift = randn(T, std=0.12)
        near = ((drift.exp() - 0.8).abs() < 2e-3) | ((drift.exp() - 1.28).abs() < 2e-3)
        drift = torch.where(near, 0.05, drift)
        live = (torch.rand(T, generator=g, device="cuda") >= c["masked"]).float()
        s.update(logits=logits, target=target.int(), logp_old=logp - drift,
                 logp_ref=logp + randn(T, std=0.2) if c["beta"] else None,
                 advantage=randn(T), weight=live / live.sum().clamp(min=1.0),
                 loss=out(4), logp=out(T), entropy=out(T),
                 grad=torch.zeros(T, ld, dtype=dt, device="cuda") if c["grad"] else None)
        return s
    if c["kind"].startswith("act"):
        R, m = c["rows"], c["m"]
        wide = torch.where(torch.rand(2 * m, generator=g, device="cuda") < 0.01, 10.0, 1.0)
        both = (randn(R, 2 * m) * wide).to(dt)  # a few channels are much larger than the rest
        if c["fused"]:
            s.update(gate=both[:, :m], up=both[:, m:])
            d = out(R, 2 * m, dtype=dt)
            s.update(dgate=d[:, :m], dup=d[:, m:])
        else:
            s.update(gate=both[:, :m].contiguous(), up=both[:, m:].contiguous(),
                     dgate=out(R, m, dtype=dt), dup=out(R, m, dtype=dt))
        s.update(dact=randn(R, m, std=0.01, dtype=dt), act=out(R, m, dtype=dt), again=out(R, m, dtype=dt))
        G = -(-m // _GROUP)
        s.update(q=out(R, 2, m, dtype=torch.int8), scale=out(R, 2, G))
        if c["kind"] == "act_grad":  # the checkpoint is at hand
            for i, x in enumerate((s.pop("gate"), s.pop("up"))):
                q, scale = _hold(x.float())
                s["q"][:, i] = q.to(torch.int8)
                s["scale"][:, i] = scale
        return s
    idx = _route(c, g)
    if c["kind"] == "gates_grad":
        T, N, k = c["T"], c["N"], c["k"]
        s.update(probs=torch.softmax(randn(T, N, std=1.5), 1), idx=idx, dgates=randn(T, k, std=0.1),
                 dlogits=out(T, N))
        return s
    T, d, N, k = c["T"], c["d"], c["N"], c["k"]
    if c["kind"] == "sort":
        s.update(idx=idx, h=randn(T, d, dtype=dt), x=out(T * k, d, dtype=dt),
                 offsets=out(N + 1, dtype=torch.int32), perm=out(T * k, dtype=torch.int32),
                 inv=out(T * k, dtype=torch.int32))
        return s
    offsets, perm, inv = _plan(idx, N)
    s.update(offsets=offsets, perm=perm, inv=inv)
    rows = randn(T * k, d, dtype=dt)
    rows[perm < 0] = math.nan  # nobody wrote the rows past the last valid slot
    if c["kind"] == "sort_grad":
        s.update(dx=rows, dh=out(T, d, dtype=dt))
        return s
    s.update(y=rows, gates=torch.softmax(randn(T, N), 1)[:, :k].contiguous())
    if c["kind"] == "unsort":
        s.update(out=out(T, d, dtype=dt))
    else:
        s.update(dout=randn(T, d, std=0.01, dtype=dt), dy=out(T * k, d, dtype=dt), dgates=out(T, k))
    return s


# ---- plain form -------------------------------------------------------------------------------

def _policy_plain(s):
    c = s["case"]
    z = s["logits"][:, :c["V"]].float() * (1.0 / c["temp"])
    a, w, adv = s["target"].long(), s["weight"], s["advantage"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    p = e / total
    live = w != 0
    entropy = torch.where(live, lse - torch.where(p > 0, p * z, 0.0).sum(1), 0.0)
    logp = torch.where(live, z.gather(1, a[:, None])[:, 0] - lse, 0.0)
    r = torch.exp(torch.where(live, logp - s["logp_old"], 0.0))
    part = -torch.minimum(r * adv, r.clamp(1 - 0.2, 1 + 0.28) * adv)
    shut = ((adv > 0) & (r > 1 + 0.28)) | ((adv < 0) & (r < 1 - 0.2))
    slope = torch.where(shut, 0.0, -r * adv)
    kl = torch.zeros_like(r)
    if c["beta"]:
        gap = torch.where(live, s["logp_ref"] - logp, 0.0)
        kl = torch.exp(gap) - gap - 1
        slope = slope + c["beta"] * (1 - torch.exp(gap))
    first, second = (w * part).sum(), (w * kl).sum()
    loss = torch.stack([first + c["beta"] * second, first, second, (w * shut).sum()])
    got = {"loss": loss, "logp": logp, "entropy": entropy}
    if c["grad"]:
        f = w * slope * (1.0 / c["temp"])
        grad = -p * f[:, None]
        grad[torch.arange(c["T"], device=z.device), a] += f
        got["grad"] = torch.where(live[:, None], grad, 0.0).to(s["logits"].dtype)
    return got


def _sort_plain(s):
    c = s["case"]
    offsets, perm, inv = _plan(s["idx"], c["N"])
    x = torch.where(perm[:, None] >= 0, s["h"][perm.clamp(min=0).long() // c["k"]], 0)
    return {"offsets": offsets, "perm": perm, "inv": inv, "x": x}


def _rows_of(x, inv, T, k):
    """The rows [T, k, d] of each token's slots, in 32 bits; zeros for an invalid slot."""
    at = inv.reshape(T, k, 1).long()
    return torch.where(at >= 0, x[at.clamp(min=0)[..., 0]].float(), 0.0)


def _tokens_plain(s):
    c = s["case"]
    T, k = c["T"], c["k"]
    if c["kind"] == "sort_grad":
        return {"dh": _rows_of(s["dx"], s["inv"], T, k).sum(1).to(s["dx"].dtype)}
    y = _rows_of(s["y"], s["inv"], T, k)
    if c["kind"] == "unsort":
        return {"out": (y * s["gates"][..., None]).sum(1).to(s["y"].dtype)}
    dout = s["dout"].float()
    dgates = (y * dout[:, None]).sum(2)
    slot = s["perm"].clamp(min=0).long()
    dy = s["gates"].reshape(-1)[slot][:, None] * dout[slot // k]
    return {"dy": torch.where(s["perm"][:, None] >= 0, dy, 0.0).to(s["y"].dtype), "dgates": dgates}


def _act_plain(s):
    c = s["case"]
    dt = s["dact"].dtype
    got = {}
    if c["kind"] == "act_step":
        gate, up = s["gate"].float(), s["up"].float()
        got["act"] = (gate / (1 + torch.exp(-gate)) * up).to(dt)
        (qg, sg), (qu, su) = _hold(gate), _hold(up)
        got["scale"] = torch.stack([sg, su], 1)
    else:
        qg, qu, sg, su = s["q"][:, 0], s["q"][:, 1], s["scale"][:, 0], s["scale"][:, 1]
    gate, up, d = _held(qg, sg), _held(qu, su), s["dact"].float()
    sig = 1 / (1 + torch.exp(-gate))
    got.update(again=(gate * sig * up).to(dt), dup=(d * gate * sig).to(dt),
               dgate=(d * up * sig * (1 + gate * (1 - sig))).to(dt))
    return got


def _gates_plain(s):
    c = s["case"]
    idx, dg, rho = s["idx"].long(), s["dgates"], s["probs"]
    sel = rho.gather(1, idx)
    if c["norm"]:
        total = sel.sum(1, keepdim=True)
        dg = (dg - (dg * sel / total).sum(1, keepdim=True)) / total
    dr = torch.zeros_like(rho).scatter_(1, idx, dg)
    return {"dlogits": rho * (dr - (dg * sel).sum(1, keepdim=True))}


# ---- the framework's calls ----------------------------------------------------------------------

def _own(s):
    B, c = _lib(), s["case"]
    kind = c["kind"]
    if "dims" not in s:
        if kind == "policy":
            s["dims"] = B.policy_dims(c["T"], c["V"], c["dtype"], ld_logits=c["V"] + c["pad"],
                                      ld_grad=c["V"] + c["pad"], inv_temp=1.0 / c["temp"],
                                      clip_low=0.2, clip_high=0.28, kl_coef=c["beta"])
            s["ws"] = B.alloc_policy_workspace(s["dims"])
        elif kind.startswith("act"):
            s["dims"] = B.act_dims(c["rows"], c["m"], c["dtype"], ld=s["dgate"].stride(0))
        elif kind == "gates_grad":
            s["dims"] = B.dims(c["T"], 64, c["N"], c["k"], 64, 0, "fp32",
                               B.PR2_F_NORMALIZE_TOPK if c["norm"] else 0)
        else:
            s["dims"] = B.dims(c["T"], c["d"], c["N"], c["k"], 64, 0, c["dtype"])
            if kind == "sort":
                s["ws"] = B.alloc_token_workspace(s["dims"])
    dm = s["dims"]
    if kind == "policy":
        B.check(B.pr2_policy_loss(dm, s["logits"], s["target"], s["weight"], s["advantage"], s["logp_old"],
                                  s["logp_ref"], s["loss"], s["logp"], s["entropy"], s["grad"], s["ws"]))
        got = {"loss": s["loss"], "logp": s["logp"], "entropy": s["entropy"]}
        if c["grad"]:
            got["grad"] = s["grad"][:, :c["V"]]
        return got
    if kind == "sort":
        B.check(B.pr2_token_sort(dm, s["h"], s["idx"], s["x"], s["offsets"], s["perm"], s["inv"], s["ws"]))
        return {n: s[n] for n in ("offsets", "perm", "inv", "x")}
    if kind == "sort_grad":
        B.check(B.pr2_token_sort_backward(dm, s["dx"], s["inv"], s["dh"]))
        return {"dh": s["dh"]}
    if kind == "unsort":
        B.check(B.pr2_token_unsort(dm, s["y"], s["gates"], s["inv"], s["out"]))
        return {"out": s["out"]}
    if kind == "unsort_grad":
        B.check(B.pr2_token_unsort_backward(dm, s["dout"], s["y"], s["gates"], s["inv"], s["offsets"], s["dy"],
                                            s["dgates"]))
        return {"dy": s["dy"], "dgates": s["dgates"]}
    if kind == "gates_grad":
        B.check(B.pr2_replay_gates_backward(dm, s["probs"], s["idx"], s["dgates"], s["dlogits"]))
        return {"dlogits": s["dlogits"]}
    got = {}
    if kind == "act_step":
        B.check(B.pr2_swiglu_checkpoint(dm, s["gate"], s["up"], s["act"], s["q"], s["scale"]))
        got = {"act": s["act"], "scale": s["scale"]}
    B.check(B.pr2_swiglu_checkpoint_backward(dm, s["dact"], s["q"], s["scale"], s["dgate"], s["dup"], s["again"]))
    return dict(got, again=s["again"], dup=s["dup"], dgate=s["dgate"])


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "policy":
        return _policy_plain(state)
    if kind == "sort":
        return _sort_plain(state)
    if kind == "gates_grad":
        return _gates_plain(state)
    return _act_plain(state) if kind.startswith("act") else _tokens_plain(state)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    kind = c["kind"]
    if kind == "policy":
        return _policy_exact(s)
    if kind.startswith("act"):
        return _act_exact(s)
    if kind == "gates_grad":
        rho, idx, dg = s["probs"].double(), s["idx"].long(), s["dgates"].double()
        T, N = rho.shape
        pick = torch.nn.functional.one_hot(idx, N).double()  # [T, k, N]
        g = torch.einsum("tkn,tn->tk", pick, rho)
        # Jacobian of the selected probabilities: d rho_s / d z_j = rho_s ([j = s] - rho_j)
        jac = g[..., None] * (pick - rho[:, None])
        if c["norm"]:
            total = g.sum(1)[:, None, None]
            jac = jac / total - g[..., None] * jac.sum(1, keepdim=True) / total ** 2
        return {"dlogits": torch.einsum("tk,tkn->tn", dg, jac)}
    T, k = c["T"], c["k"]
    if kind == "sort":
        ok = s["idx"].reshape(-1) >= 0
        slots = torch.nonzero(ok)[:, 0]
        slots = slots[torch.argsort(s["idx"].reshape(-1)[slots], stable=True)]
        x = torch.zeros(T * k, c["d"], dtype=torch.float64, device="cuda")
        x[:slots.numel()] = s["h"].double()[slots // k]
        return {"offsets": None, "perm": None, "inv": None, "x": x}
    # one weight per (token, slot) pair, walked in slot order
    inv = s["inv"].reshape(T, k).long()
    if kind in ("sort_grad", "unsort"):
        src = s["dx"] if kind == "sort_grad" else s["y"]
        acc = torch.zeros(T, c["d"], dtype=torch.float64, device="cuda")
        for j in range(k):
            t = torch.nonzero(inv[:, j] >= 0)[:, 0]
            row = src[inv[t, j]].double()
            acc[t] += row if kind == "sort_grad" else s["gates"][t, j, None].double() * row
        return {"dh" if kind == "sort_grad" else "out": acc}
    dy = torch.zeros(T * k, c["d"], dtype=torch.float64, device="cuda")
    dgates = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(inv[:, j] >= 0)[:, 0]
        dout = s["dout"][t].double()
        dy[inv[t, j]] = s["gates"][t, j, None].double() * dout
        dgates[t, j] = (s["y"][inv[t, j]].double() * dout).sum(1)
    return {"dy": dy, "dgates": dgates}


def _policy_exact(s):
    c = s["case"]
    T, V = c["T"], c["V"]
    names = ("logp", "entropy")
    got = {n: torch.zeros(T, dtype=torch.float64, device="cuda") for n in names}
    sums = torch.zeros(3, dtype=torch.float64, device="cuda")
    grad = torch.zeros(T, V, dtype=torch.float64, device="cuda") if c["grad"] else None
    step = max(1, (1 << 28) // V)
    for lo in range(0, T, step):
        rows = torch.arange(lo, min(T, lo + step), device="cuda")
        rows = rows[s["weight"][rows] != 0]  # tokens that do not count are left at zero
        if rows.numel() == 0:
            continue
        lp = torch.log_softmax(s["logits"][rows, :V].double() / c["temp"], 1)
        prob = lp.exp()
        at, a = torch.arange(rows.numel(), device="cuda"), s["target"][rows].long()
        logp = lp[at, a]
        got["logp"][rows] = logp
        got["entropy"][rows] = -torch.where(prob > 0, prob * lp, 0.0).sum(1)
        w, A = s["weight"][rows].double(), s["advantage"][rows].double()
        ratio = (logp - s["logp_old"][rows].double()).exp()
        bound = torch.where(A >= 0, ratio.clamp(max=1.28), ratio.clamp(min=0.8))
        cut = bound != ratio
        sums[0] += (-w * bound * A).sum()
        sums[2] += (w * (cut & (A != 0))).sum()
        slope = torch.where(cut, 0.0, -ratio * A)
        if c["beta"]:
            q = (s["logp_ref"][rows].double() - logp)
            sums[1] += (w * (q.exp() - 1 - q)).sum()
            slope = slope - c["beta"] * (q.exp() - 1)
        if grad is not None:
            prob[at, a] -= 1
            grad[rows] = prob * (-w * slope / c["temp"])[:, None]
    got["loss"] = torch.stack([sums[0] + c["beta"] * sums[1], sums[0], sums[1], sums[2]])
    if grad is not None:
        got["grad"] = grad
    return got


def _act_exact(s):
    c = s["case"]
    m = c["m"]
    span = torch.arange(m, device="cuda") // _GROUP
    got = {}
    if c["kind"] == "act_step":
        gate, up = s["gate"].double(), s["up"].double()
        got["act"] = gate * torch.sigmoid(gate) * up
        held, scales = [], []
        for x in (s["gate"], s["up"]):
            # the format's own roundings are part of the definition: scale and reciprocal in 32 bits
            top = torch.zeros(c["rows"], int(span[-1]) + 1, device="cuda")
            top.scatter_reduce_(1, span.expand(c["rows"], m), x.float().abs(), "amax")
            r = torch.ones_like(top).mul(127.0).div(top)[:, span]
            sc = top * torch.tensor(1 / 127, dtype=torch.float32, device="cuda")
            some = top >= _TINY
            sc = torch.where(some, sc, 0.0)
            held.append(torch.where(some[:, span], (x.float() * r).round(), 0.0).double() * sc[:, span].double())
            scales.append(sc.double())
        got["scale"] = torch.stack(scales, 1)
        gate, up = held
    else:
        gate, up = (s["q"][:, i].double() * s["scale"][:, i].double()[:, span] for i in (0, 1))
    d, sig = s["dact"].double(), torch.sigmoid(gate)
    got.update(again=gate * sig * up, dup=d * gate * sig,
               dgate=d * up * (sig + gate * sig * torch.sigmoid(-gate)))
    return got
