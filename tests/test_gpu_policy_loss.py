"""GPU policy loss (pr2_policy_loss) against the plain 64-bit form.

Tolerances.  z = inv_temp logit is rounded once (2^-24 |z|, |z| < 40 here: 2.4e-6) and the
exponentials are good to a few 2^-22, sums of positive terms add no more than a few roundings in the
depth of their tree, so l has a relative error below 1e-5 and logp an absolute one below 1e-5 plus
the rounding of logp itself (2^-24 |logp|).  The entropy weights |x| < 40 with those errors: 1e-4.
A gradient entry is f ([v = a] - p): p's relative error 1e-5 and f's (through the ratio and the KL
factor) both scale with the row's terms (`scale` of the reference): 3e-5 of it, plus one rounding of
the stored type.  loss is a sum of terms with relative errors 2e-5 of their size.
"""
import math

import pytest
import torch

import train_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -23}


def make(T, V, dtype, seed, pad=0, banned=0.0, shift=0, std=2.0):
    g = torch.Generator().manual_seed(seed)
    ld = V + pad
    buf = torch.empty(T * ld + shift + 64, dtype=DT[dtype])
    logits = buf[shift:shift + T * ld].view(T, ld)
    z = std * torch.randn(T, ld, generator=g)
    target = torch.randint(0, V, (T,), generator=g).int()
    if banned:
        z[torch.rand(T, ld, generator=g) < banned] = -math.inf
    z[torch.arange(T), target.long()] = 6 * torch.rand(T, generator=g)
    z[:, V:] = 1e4  # padding columns hold anything
    logits.copy_(z)
    lp = torch.log_softmax(logits[:, :V].double(), 1)[torch.arange(T), target.long()]
    # ratios stay clear of the clip bounds, where a last bit decides
    drift = torch.tensor([0.05, -0.1, 0.4, -0.5, 0.15])[torch.randint(0, 5, (T,), generator=g)]
    weight = torch.where(torch.rand(T, generator=g) < 0.25, 0.0, torch.rand(T, generator=g) / T + 1e-3)
    return dict(buf=buf, shift=shift, ld=ld, V=V, logits=logits, target=target, weight=weight,
                advantage=torch.randn(T, generator=g), logp_old=(lp - drift).float(),
                logp_ref=(lp + 0.3 * torch.randn(T, generator=g, dtype=torch.float64)).float())


def call(c, dtype, names=("weight", "logp_old", "logp_ref"), grad=True, inplace=False, ld_grad=None,
         **kw):
    T, V, ld = c["logits"].shape[0], c["V"], c["ld"]
    dev = c["buf"].cuda()
    logits = dev[c["shift"]:c["shift"] + T * ld].view(T, ld)
    opt = {n: c[n].cuda() if n in names else None for n in ("weight", "logp_old", "logp_ref")}
    ldg = ld if ld_grad is None else ld_grad
    dm = B.policy_dims(T, V, dtype, ld_logits=ld, ld_grad=ldg, **kw)
    loss = torch.full((4,), math.nan, device="cuda")
    logp, ent = (torch.full((T,), math.nan, device="cuda") for _ in range(2))
    out = logits if inplace else torch.full((T, ldg), 7.0, dtype=DT[dtype], device="cuda") if grad else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.check(B.pr2_policy_loss(dm, logits, c["target"].cuda(), opt["weight"], c["advantage"].cuda(),
                              opt["logp_old"], opt["logp_ref"], loss, logp, ent, out,
                              B.alloc_policy_workspace(dm), status=status), "pr2_policy_loss")
    torch.cuda.synchronize()
    return dict(loss=loss.cpu(), logp=logp.cpu(), entropy=ent.cpu(), status=int(status.item()),
                grad=None if out is None else out.cpu())


def check(c, got, dtype, names=("weight", "logp_old", "logp_ref"), **kw):
    ref = R.policy(c["logits"][:, :c["V"]], c["target"], c["advantage"],
                   **{n: c[n] for n in names}, **kw)
    assert torch.isfinite(ref["loss"]).all()
    live = torch.isfinite(ref["logp"])
    assert torch.equal(got["logp"][~live].double(), ref["logp"][~live])
    err = (got["logp"].double() - ref["logp"])[live].abs()
    assert (err <= 1e-5 + 2.0 ** -24 * ref["logp"][live].abs()).all(), float(err.max())
    assert ((got["entropy"].double() - ref["entropy"]).abs() <= 1e-4).all()
    size = float((ref["scale"].sum() + ref["loss"].abs().sum()))
    assert ((got["loss"].double() - ref["loss"]).abs() <= 2e-5 * size).all()
    if got["grad"] is not None:
        g = got["grad"][:, :c["V"]].double()
        bound = 3e-5 * ref["scale"][:, None] + EPS[dtype] * ref["grad"].abs()
        assert ((g - ref["grad"]).abs() <= bound).all()
    return ref


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,pad,shift", [
    (1, 1, 0, 0), (1, 2, 0, 1), (3, 7, 1, 0), (5, 33, 0, 3), (4, 255, 0, 1), (7, 1000, 24, 0),
    (2, 4097, 0, 5), (9, 8192, 0, 0), (300, 515, 0, 0), (700, 64, 0, 0), (3, 32001, 0, 0),
    (1, 70003, 0, 0), (2, 131072, 8, 8), (1, 300001, 0, 1), (1000, 5003, 0, 1), (600, 6000, 1, 0)])
def test_loss_and_gradient(dtype, T, V, pad, shift):
    c = make(T, V, dtype, T * 31 + V, pad=pad, shift=shift)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05)
    got = call(c, dtype, **kw)
    check(c, got, dtype, **kw)
    assert got["status"] == 0
    if pad:
        assert (got["grad"][:, V:] == 7.0).all()  # the padding columns are left alone


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_rows_a_block(dtype):
    c = make(3001, 130, dtype, 4)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, inv_temp=1.25, grad_scale=3.0)
    check(c, call(c, dtype, **kw), dtype, **kw)


@pytest.mark.parametrize("dtype,T,V,pad,shift", [
    ("bf16", 1217, 53001, 0, 1), ("bf16", 1300, 51200, 0, 0), ("bf16", 1300, 51199, 1, 0),
    ("fp32", 1250, 27003, 5, 0), ("bf16", 1216, 107009, 0, 0), ("fp32", 1216, 66000, 0, 2),
    ("bf16", 1240, 205001, 0, 0), ("bf16", 1215, 65536, 0, 0)])
def test_long_rows_in_large_batches(dtype, T, V, pad, shift):
    """61 different rows in turn, so that each meets the CTAs at several times and alignments."""
    few = make(61, V, dtype, T + V)
    which = torch.arange(T) % 61
    c = {n: few[n][which] for n in ("target", "weight", "advantage", "logp_old", "logp_ref")}
    ld = V + pad
    buf = torch.full((T * ld + shift,), 1e4, dtype=DT[dtype])
    logits = buf[shift:].view(T, ld)
    logits[:, :V] = few["logits"][which]
    c.update(buf=buf, shift=shift, ld=ld, V=V, logits=logits)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05)
    got = call(c, dtype, **kw)
    opt = {n: few[n] for n in ("logp_old", "logp_ref")}
    ref = R.policy(few["logits"], few["target"], few["advantage"], weight=few["weight"], **opt, **kw)
    bound = 3e-5 * ref["scale"][:, None] + EPS[dtype] * ref["grad"].abs()
    for b in range(0, T, 61):
        n = min(61, T - b)
        err = (got["logp"][b:b + n].double() - ref["logp"][:n]).abs()
        assert (err <= 1e-5 + 2.0 ** -24 * ref["logp"][:n].abs()).all(), (b, float(err.max()))
        assert ((got["entropy"][b:b + n].double() - ref["entropy"][:n]).abs() <= 1e-4).all(), b
        assert ((got["grad"][b:b + n, :V].double() - ref["grad"][:n]).abs() <= bound[:n]).all(), b
    assert (got["grad"][:, V:] == 7.0).all() and got["status"] == 0
    # the loss is linear in the weights: each of the 61 rows counts as often as it came
    times = torch.bincount(which).to(torch.float64)
    total = R.policy(few["logits"], few["target"], few["advantage"], weight=few["weight"].double() * times, **opt,
                     **kw)
    size = float(total["scale"].sum() + total["loss"].abs().sum())
    assert ((got["loss"].double() - total["loss"]).abs() <= 2e-5 * size).all()


def masks(T, kind):
    t = torch.arange(T)
    x = torch.rand(T, generator=torch.Generator().manual_seed(T))
    return {"none": t >= 0, "all": t < 0, "first half": t >= T // 2, "second half": t < T // 2,
            "all but the last": t == T - 1, "runs": (t // 100) % 3 != 0, "random": x < 0.4}[kind]


@pytest.mark.parametrize("kind", ["none", "all", "first half", "second half", "all but the last", "runs", "random"])
@pytest.mark.parametrize("dtype,T,V,grad", [
    ("bf16", 1000, 5001, True), ("fp32", 700, 6500, True), ("bf16", 9001, 4200, True), ("bf16", 65536, 4104, False),
    ("bf16", 65537, 4104, False), ("bf16", 1400, 52001, False), ("fp32", 600, 30000, False),
    ("fp32", 3000, 9001, False)])
def test_masked_tokens_in_large_batches(dtype, T, V, grad, kind):
    """Masked tokens and the others reach the CTAs in turns of their own; every token is done once.  61 different
    rows in turn; a row's gradient and its part of the loss are linear in its weight."""
    few = make(61, V, dtype, V)
    few["weight"] = torch.ones(61)
    which = torch.arange(T) % 61
    c = {n: few[n][which] for n in ("target", "advantage", "logp_old", "logp_ref")}
    weight = masks(T, kind) * (0.5 + torch.arange(T) % 7) / T
    c.update(weight=weight.float(), buf=few["logits"][which].flatten(), shift=0, ld=V, V=V)
    c["logits"] = c["buf"].view(T, V)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05)
    got = call(c, dtype, grad=grad, **kw)
    opt = {n: few[n] for n in ("weight", "logp_old", "logp_ref")}
    ref = R.policy(few["logits"], few["target"], few["advantage"], **opt, **kw)
    w, live = c["weight"].double(), c["weight"] != 0
    for n, bound in (("logp", 1e-5 + 2.0 ** -24 * ref["logp"].abs()), ("entropy", torch.full((61,), 1e-4))):
        err = (got[n].double() - torch.where(live, ref[n][which], 0.0)).abs()
        assert (err <= torch.where(live, bound[which].double(), 0.0)).all(), n
    total = R.policy(few["logits"], few["target"], few["advantage"], logp_old=few["logp_old"],
                     logp_ref=few["logp_ref"], weight=torch.bincount(which, w, 61), **kw)
    size = float(total["scale"].sum() + total["loss"].abs().sum())
    assert ((got["loss"].double() - total["loss"]).abs() <= 2e-5 * size).all()
    for b in range(0, T if grad else 0, 61):
        n = min(61, T - b)
        want, row = w[b:b + n, None] * ref["grad"][:n], w[b:b + n] * ref["scale"][:n]
        bound = 3e-5 * row[:, None] + EPS[dtype] * want.abs()
        assert ((got["grad"][b:b + n].double() - want).abs() <= bound).all(), b


@pytest.mark.parametrize("V,ld_grad", [(1000, 1001), (1024, 1040), (333, 334)])
def test_gradient_rows_of_another_stride(V, ld_grad):
    c = make(6, V, "bf16", V)
    got = call(c, "bf16", ld_grad=ld_grad)
    check(c, got, "bf16", clip_low=0.2, clip_high=0.2)
    assert (got["grad"][:, V:] == 7.0).all()


@pytest.mark.parametrize("dtype,V,pad", [("bf16", 1024, 0), ("bf16", 40001, 0), ("fp32", 777, 3)])
def test_gradient_in_place_of_the_logits(dtype, V, pad):
    c = make(37, V, dtype, 11, pad=pad)
    kw = dict(clip_high=0.28, kl_coef=0.1)
    apart, same = call(c, dtype, **kw), call(c, dtype, inplace=True, **kw)
    for n in ("loss", "logp", "entropy"):
        assert torch.equal(apart[n], same[n])
    assert torch.equal(apart["grad"][:, :V], same["grad"][:, :V])


def test_optional_inputs_and_outputs():
    c = make(50, 300, "fp32", 2)
    got = call(c, "fp32", names=(), grad=False)
    check(c, got, "fp32", names=())
    assert float(got["loss"][2]) == 0.0 and got["grad"] is None
    check(c, call(c, "fp32", names=("logp_ref",), kl_coef=0.2), "fp32", names=("logp_ref",), kl_coef=0.2)
    # the KL part is measured even where it has no weight in the loss
    seen = call(c, "fp32", names=("logp_ref",))
    check(c, seen, "fp32", names=("logp_ref",))
    assert float(seen["loss"][0]) == float(seen["loss"][1]) and float(seen["loss"][2]) > 0
    dm = B.policy_dims(50, 300, "fp32")
    loss = torch.empty(4, device="cuda")
    B.check(B.pr2_policy_loss(dm, c["logits"].cuda(), c["target"].cuda(), None, c["advantage"].cuda(),
                              None, None, loss, None, None, None, B.alloc_policy_workspace(dm)))
    assert torch.equal(loss.cpu(), got["loss"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_banned_entries_and_empty_rows(dtype):
    c = make(12, 3000, dtype, 8, banned=0.4)
    c["logits"][3] = -math.inf           # nothing can be sampled
    c["logits"][4] = torch.finfo(DT[dtype]).min  # the type's lowest value everywhere: uniform
    c["logits"][5, :] = -math.inf
    c["logits"][5, c["target"][5].long()] = 1.0  # one token left: p = 1
    c["weight"][:6] = 0.01
    c["logp_old"][4:6] = 0.0
    c["logp_ref"][4:6] = -0.1
    c["logp_old"][4] = c["logp_ref"][4] = -math.log(3000)
    kw = dict(clip_high=0.28, kl_coef=0.05)
    got = call(c, dtype, **kw)
    check(c, got, dtype, **kw)
    assert got["logp"][3] == -math.inf and got["entropy"][3] == 0 and not got["grad"][3].any()
    assert not got["grad"][c["logits"] == -math.inf].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [300, 9000])
def test_a_target_that_is_banned(V, dtype):
    """Its probability is 0: logp -inf, ratio 0, no gradient (without a KL term)."""
    c = make(5, V, dtype, 17)
    c["weight"][:] = 0.2
    c["advantage"][:] = torch.tensor([1.0, 1.0, -1.0, 0.0, 2.0])
    for t in (1, 2, 3):
        c["logits"][t, c["target"][t].long()] = -math.inf
    got = call(c, dtype, names=("weight", "logp_old"))
    assert (got["logp"][1:4] == -math.inf).all() and torch.isfinite(got["entropy"]).all()
    assert not got["grad"][1:4].any() and torch.isfinite(got["loss"]).all() and torch.isfinite(got["grad"]).all()
    check(c, got, dtype, names=("weight", "logp_old"))
    onp = call(c, dtype, names=("weight",))  # on-policy: the ratio is 1 by definition
    assert (onp["logp"][1:4] == -math.inf).all() and torch.isfinite(onp["loss"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset", [-3000.0, -70.0, 45.0, 500.0])
def test_logits_with_an_offset(offset, dtype):
    """The sums' reference is 0 to begin with; rows far from it are summed relative to their maximum.  The
    offset is exact in either type only where the logits are on its grid."""
    c = make(6, 5000, dtype, 18, std=1.0)
    c["logits"][:, :5000] = (c["logits"][:, :5000].float() * 0.25).round() * 16 + offset
    base = torch.log_softmax(c["logits"][:, :5000].double(), 1)[torch.arange(6), c["target"].long()]
    c["weight"][:] = 0.15
    c["logp_old"], c["logp_ref"] = (base - 0.05).float(), (base + 0.1).float()
    kw = dict(kl_coef=0.05)
    check(c, call(c, dtype, **kw), dtype, **kw)


def test_tokens_that_do_not_count_are_not_read():
    c = make(20, 500, "bf16", 9)
    kw = dict(kl_coef=0.05)
    c["weight"][:] = 0.02
    c["weight"][7] = c["weight"][13] = c["weight"][19] = 0.0
    want = call(c, "bf16", **kw)
    for t, bad in ((7, math.nan), (13, math.inf), (19, math.nan)):
        c["logits"][t] = bad
        c["advantage"][t] = c["logp_old"][t] = c["logp_ref"][t] = bad
    c["target"][7] = -100
    got = call(c, "bf16", **kw)
    for n in ("loss", "logp", "entropy", "grad"):
        assert torch.equal(got[n], want[n]), n
    assert got["status"] == 0 and not got["grad"][7].any() and got["logp"][7] == 0


def test_targets_out_of_range_are_flagged_and_left_out():
    c = make(20, 500, "fp32", 10)
    c["weight"][:] = 0.05
    good = dict(c, weight=c["weight"].clone(), target=c["target"].clone())
    good["weight"][4] = good["weight"][9] = 0.0
    c["target"][4], c["target"][9] = 500, -1
    a, b = call(c, "fp32"), call(good, "fp32")
    assert a["status"] == B.PR2_STATUS_BAD_INDEX and b["status"] == 0
    for n in ("loss", "logp", "entropy", "grad"):
        assert torch.equal(a[n], b[n]), n


def test_extremes():
    c = make(8, 200, "fp32", 12)
    c["weight"][:] = 0.125
    c["advantage"][:] = torch.tensor([0.0, 0.0, -1.0, 1.0, 1.0, 1.0, 1.0, 1.0])
    c["logp_old"][0] = -1000.0   # ratio overflows; the advantage is 0
    c["logits"][3] += 80.0       # a large offset changes nothing
    got = call(c, "fp32", names=("weight", "logp_old"))
    assert torch.isfinite(got["loss"]).all() and torch.isfinite(got["grad"]).all()
    assert not got["grad"][0].any()
    for bad in (math.nan, math.inf):  # a row that holds one is loud
        d = dict(c, logits=None)
        d["buf"] = c["buf"].clone()
        d["logits"] = d["buf"][:8 * 200].view(8, 200)
        d["logits"][5, 17] = bad
        got = call(d, "fp32", names=("weight", "logp_old"))
        assert torch.isnan(got["logp"][5]) and torch.isnan(got["loss"][0]) and torch.isnan(got["grad"][5]).all()
        assert torch.isfinite(got["logp"][[0, 1, 2, 3, 4, 6, 7]]).all()


@pytest.mark.parametrize("T,V", [(64, 5000), (2000, 999)])
def test_same_bits_twice_and_on_another_stream(T, V):
    c = make(T, V, "bf16", 13)
    a = call(c, "bf16", kl_coef=0.05)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = call(c, "bf16", kl_coef=0.05)
    for n in ("loss", "logp", "entropy", "grad"):
        assert torch.equal(a[n], b[n]), n


def test_captured_in_a_graph():
    c = make(40, 2000, "bf16", 14)
    want = call(c, "bf16", kl_coef=0.05)
    dm = B.policy_dims(40, 2000, "bf16", kl_coef=0.05)
    t = {n: c[n].cuda() for n in ("logits", "target", "weight", "advantage", "logp_old", "logp_ref")}
    loss, grad, ws = torch.zeros(4, device="cuda"), torch.zeros_like(t["logits"]), B.alloc_policy_workspace(dm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.check(B.pr2_policy_loss(dm, t["logits"], t["target"], t["weight"], t["advantage"], t["logp_old"],
                                  t["logp_ref"], loss, None, None, grad, ws))
    for _ in range(2):
        loss.zero_()
        grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss.cpu(), want["loss"]) and torch.equal(grad.cpu(), want["grad"])


@pytest.mark.parametrize("T,V", [(2, 3000), (5, 40000), (63, 3000), (64, 3000), (65, 3000), (9, 500), (512, 500),
                                 (513, 500)])
def test_loss_in_any_workspace_and_in_replays(T, V):
    """Whatever the workspace holds, one call after another, and a graph replayed with other weights."""
    c = make(T, V, "bf16", T + V)
    dm = B.policy_dims(T, V, "bf16", kl_coef=0.05)
    opt = {n: c[n].cuda() for n in ("logits", "target", "weight", "advantage", "logp_old", "logp_ref")}
    opt["weight"][:] = 1.0 / T
    loss = torch.full((4,), math.nan, device="cuda")
    ws = B.alloc_policy_workspace(dm)

    def run():
        B.check(B.pr2_policy_loss(dm, opt["logits"], opt["target"], opt["weight"], opt["advantage"], opt["logp_old"],
                                  opt["logp_ref"], loss, None, None, None, ws))

    ref = R.policy(c["logits"], c["target"], c["advantage"], logp_old=c["logp_old"], logp_ref=c["logp_ref"],
                   weight=torch.full((T,), 1.0 / T), kl_coef=0.05)
    size = float(ref["scale"].sum() + ref["loss"].abs().sum())

    def right(factor):
        off = (loss.cpu().double() / factor - ref["loss"]).abs()
        assert (off <= 2e-5 * size).all(), (factor, off)

    for i in range(50):
        ws.fill_(i)
        loss.fill_(math.nan)
        run()
        right(1.0)
    for i in range(50):
        loss.fill_(math.nan)
        run()
        right(1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(50):
        opt["weight"][:] = 2.0 ** (i % 5) / T
        loss.fill_(math.nan)
        graph.replay()
        right(2.0 ** (i % 5))


@pytest.mark.parametrize("T,V,grad", [(1000, 5000, True), (1300, 52000, True), (2000, 9000, False), (40, 5000, True)])
def test_calls_follow_what_is_before_them_in_the_stream(T, V, grad):
    """Logits and weights written right before a call, a call right behind another with the same workspace, its
    outputs read and its inputs overwritten right after: the same bits as each call alone."""
    c = make(T, V, "bf16", T)
    base = c["logits"].cuda()
    names = ("target", "weight", "advantage", "logp_old", "logp_ref")
    opt = {n: c[n].cuda() for n in names}
    dm = B.policy_dims(T, V, "bf16", kl_coef=0.05)
    ws = B.alloc_policy_workspace(dm)
    z, w, g = torch.zeros_like(base), torch.zeros_like(opt["weight"]), torch.zeros_like(base) if grad else None
    loss = [torch.zeros(4, device="cuda") for _ in range(2)]
    logp = torch.zeros(T, device="cuda")
    weights = [opt["weight"], opt["weight"].flip(0).contiguous()]

    def run(i):
        B.check(B.pr2_policy_loss(dm, z, opt["target"], w, opt["advantage"], opt["logp_old"], opt["logp_ref"],
                                  loss[i % 2], logp, None, g, ws))

    alone = []
    for i in range(2):
        z.copy_(base)
        w.copy_(weights[i])
        torch.cuda.synchronize()
        run(i)
        torch.cuda.synchronize()
        alone.append([loss[i].clone(), logp.clone(), g.clone() if grad else None])
    seen = []
    for i in range(30):
        z.fill_(-3.0)
        w.fill_(7.0)
        torch.mul(base, 1.0, out=z)
        w.copy_(weights[i % 2])
        run(i)
        run(i)
        seen.append([loss[i % 2].clone(), logp.clone(), g.clone() if grad and i > 27 else None])
    torch.cuda.synchronize()
    for i, got in enumerate(seen):
        want = alone[i % 2]
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
        assert got[2] is None or torch.equal(got[2], want[2]), i


def test_gradient_against_differences_of_the_loss():
    """fp32 differences: loss errors 2e-5 of the terms' size over a step of 2^-6 give 3e-3 of it, the
    step's own error is below 2^-12 of it."""
    c = make(4, 50, "fp32", 21, std=1.0)
    c["weight"][:] = 0.25
    kw = dict(clip_high=0.28, kl_coef=0.1)
    base = call(c, "fp32", **kw)
    size = float(R.policy(c["logits"], c["target"], c["advantage"], weight=c["weight"], logp_old=c["logp_old"],
                          logp_ref=c["logp_ref"], **kw)["scale"].max())
    h = 2.0 ** -6
    for t in range(4):
        for v in (int(c["target"][t]), 3, 49):
            two = []
            for sign in (1, -1):
                keep = c["logits"][t, v].clone()
                c["logits"][t, v] += sign * h
                two.append(float(call(c, "fp32", grad=False, **kw)["loss"][0]))
                c["logits"][t, v] = keep
            assert abs((two[0] - two[1]) / (2 * h) - float(base["grad"][t, v])) <= 4e-3 * size


def test_empty_batch_writes_zero_loss():
    dm = B.policy_dims(0, 100, "bf16")
    loss = torch.ones(4, device="cuda")
    B.check(B.pr2_policy_loss(dm, None, None, None, None, None, None, loss))
    assert not loss.cpu().any()


def test_rows_beyond_32_bit_offsets():
    T, V = 18000, 131072  # 2.36e9 logits; only a few rows count
    dm = B.policy_dims(T, V, "bf16")
    logits = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(T, device="cuda")
    rows = torch.tensor([0, 16384, 17999])
    w[rows.cuda()] = 0.5
    target = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    logits[rows.cuda(), V - 1] = 10.0
    loss, logp = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    B.check(B.pr2_policy_loss(dm, logits, target, w, torch.ones(T, device="cuda"), None, None, loss, logp, None,
                              logits, B.alloc_policy_workspace(dm)))
    p = math.exp(10) / (math.exp(10) + V - 1)
    assert torch.allclose(logp[rows.cuda()].cpu().double(), torch.full((3,), math.log(p), dtype=torch.float64), atol=1e-5)
    got = logits[rows.cuda()].cpu().double()
    assert torch.allclose(got[:, V - 1], torch.full((3,), -0.5 * (1 - p), dtype=torch.float64), rtol=2.0 ** -8)
    assert torch.allclose(got[:, 0], torch.full((3,), 0.5 * (1 - p) / (V - 1), dtype=torch.float64), rtol=2.0 ** -8)
    assert not logits[1].any()
