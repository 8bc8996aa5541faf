"""The losses over logits on the GPU against a plain implementation in 64 bits
(on the CPU, below), where they can go wrong: vocabularies around the sizes of
the kernels' pieces and workgroups, every type, strides, masks, packed
sequences with empty ones, infinities and NaN, in-place gradients, streams,
graphs and offsets beyond 32 bits.

Tolerances (u = 2^-24).  An exponential's argument carries three roundings and
v_exp_f32 one more: the e_j of an argument a is off by at most
(2.1 |a| + 2) u relative; where |a| <= 64, as in all inputs here (what lies
further down is below 2^-64 of its row and enters through absolute errors),
136 u.  A row's sum has at most 100 additions in a chain (20 pieces, a tree in each,
10 exchange steps, 16 waves; 64 pieces where rows do not stay in registers):
100 u more.  So p is within 236 u, 1.5e-5, and log p within 1.5e-5 + 2 u |log p|;
EP below is 2e-5.  A gradient element g (1[y] - p) / T is then within
EP |g| (p + 1[y]) / T plus its coefficient's error, plus its type's rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EP = 2e-5
U = 2.0 ** -24
IGNORE = -100
TINY = {torch.float32: 2.0 ** -125, torch.bfloat16: 2.0 ** -125, torch.float16: 2.0 ** -25}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {d: torch.finfo(d).eps / 2 for d in DTYPES}


@pytest.fixture(scope="module")
def L(gpu_lib):
    from paper_2507_08784_amd import losses
    return losses


def _say(*a):
    print("[losses]", *a, flush=True)


# ----------------------------------------------------------------------------
# 64 bits
# ----------------------------------------------------------------------------
def ref_rows(z, y, T):
    """log p of the targets and p, of 2-D logits."""
    x = z.double() / T
    m = x.max(1, keepdim=True).values
    e = (x - m).exp()
    s = e.sum(1, keepdim=True)
    at = y.clamp(0, z.shape[1] - 1)[:, None]
    return (x.gather(1, at) - m - s.log())[:, 0], e / s


def ref_grad(p, y, coef, T):
    g = -p * (coef / T)[:, None]
    g[torch.arange(len(y)), y.clamp(min=0)] += coef / T
    g[coef == 0] = 0.0
    return g


def close_grad(got, want, p, y, g, dg, T, dtype, what):
    """got against want, with coefficients g known to within dg."""
    got = got.double().cpu().reshape(want.shape)
    near = p.clone()
    near[torch.arange(len(y)), y.clamp(min=0)] += 1.0
    tol = ((EP * g.abs() + dg) / T)[:, None] * near + HALF_ULP[dtype] * 1.001 * want.abs() + TINY[dtype]
    off = (got - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((off / tol)[bad].max()), bad.nonzero()[:3].tolist())


def close(got, want, tol, what):
    got = got.double().cpu().reshape(want.shape)
    off = (got - want).abs()
    assert bool((off <= tol).all()), (what, float((off / tol).max()))


def lp_tol(lp):
    return EP + 2 * U * lp.abs()


def make(rows, V, dtype, seed, masked=0.3, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(rows, V, generator=g) * spread).to(dtype)
    y = torch.randint(0, V, (rows,), generator=g)
    at = torch.rand(rows, generator=g) < 0.6
    z[at, y[at]] = (6 + 2 * torch.randn(int(at.sum()), generator=g)).to(dtype)
    y = torch.where(torch.rand(rows, generator=g) < masked, IGNORE, y)
    return z, y, g


# pieces are 4 or 8 elements; workgroups hold 64 to 20480 pieces
VOCABS = [1, 2, 3, 7, 8, 9, 33, 255, 256, 520, 1000, 2049, 4097, 8200, 16385, 32000, 50265, 66000, 131077, 170003]


# ----------------------------------------------------------------------------
# token log-probabilities
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", VOCABS)
def test_logprobs_and_their_gradient(L, V, dtype):
    rows = 9 if V > 20000 else 37
    z, y, gen = make(rows, V, dtype, V)
    T = [1.0, 0.7, 1.9][V % 3]
    w = torch.randn(rows, generator=gen)
    lp, p = ref_rows(z, y, T)
    live = y != IGNORE
    lp = torch.where(live, lp, 0.0)
    coef = torch.where(live, w.double() * 3.0, 0.0)
    want = ref_grad(p, y, coef, T)
    zg, yg = z.cuda(), y.cuda()
    plain = L.token_logprobs(zg, yg, temperature=T)
    assert plain.dlogits is None
    close(plain.logps, lp, lp_tol(lp), "logps")
    r = L.token_logprobs(zg, yg, weights=w.cuda(), temperature=T, grad_scale=3.0)
    close(r.logps, lp, lp_tol(lp), "logps")
    close_grad(r.dlogits, want, p, y, coef, 2 * U * coef.abs(), T, dtype, "dlogits")
    # the upstream gradient through autograd, from the saved sums
    leaf = zg.clone().requires_grad_(True)
    out = L.token_logprobs(leaf, yg.int(), temperature=T).logps
    out.backward(w.cuda() * 3.0)
    close(out.detach(), lp, lp_tol(lp), "logps")
    close_grad(leaf.grad, want, p, y, coef, 2 * U * coef.abs(), T, dtype, "autograd")


@pytest.mark.parametrize("rows", [0, 1, 2, 1000])
def test_row_counts(L, rows):
    z, y, gen = make(rows, 300, torch.bfloat16, rows)
    lp, p = ref_rows(z, y, 1.0) if rows else (torch.zeros(0), torch.zeros(0, 300))
    live = y != IGNORE
    lp = torch.where(live, lp, 0.0)
    w = torch.ones(rows)
    r = L.token_logprobs(z.cuda(), y.cuda(), weights=w.cuda())
    assert r.logps.shape == (rows,) and r.dlogits.shape == (rows, 300)
    if rows:
        close(r.logps, lp, lp_tol(lp), "logps")
        close_grad(r.dlogits, ref_grad(p, y, live.double(), 1.0), p, y, live.double(), U * w, 1.0, torch.bfloat16, "dlogits")


@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_rows_are_taken_as_they_are(L, dtype):
    # all positions but the last against all tokens but the first; rows padded; a batch turned round
    B, S, V = 3, 6, 1003
    z, y, gen = make(B * (S + 1), V + 13, dtype, 3, masked=0.2)
    z, y = z.view(B, S + 1, V + 13), y.clamp(max=V - 1).view(B, S + 1)
    zg, yg = z.cuda(), y.cuda()
    w = torch.randn(B, 1, generator=gen)
    views = [(zg[:, :-1, :V], yg[:, 1:], z[:, :-1, :V], y[:, 1:]),
             (zg[:, 1:, 13:], yg[:, :-1], z[:, 1:, 13:], y[:, :-1]),
             (zg.transpose(0, 1)[:, :, :V], yg.transpose(0, 1), z.transpose(0, 1)[:, :, :V], y.transpose(0, 1)),
             (zg[0, ::2, :V], yg[0, ::2], z[0, ::2, :V], y[0, ::2])]
    for a, b, c, d in views:
        flat = d.reshape(-1)
        lp, p = ref_rows(c.reshape(-1, V), flat, 1.0)
        live = flat != IGNORE
        ww = w.expand(B, d.shape[-1]) if d.shape[0] == B and d.dim() == 2 else torch.full(d.shape, 0.5)
        wg = w.cuda().expand(B, d.shape[-1]) if d.shape[0] == B and d.dim() == 2 else torch.full(d.shape, 0.5).cuda()
        coef = torch.where(live, ww.reshape(-1).double(), 0.0)
        want = ref_grad(p, flat, coef, 1.0)
        out = torch.empty(*d.shape, V + 5, dtype=dtype, device="cuda")[..., 5:]
        r = L.token_logprobs(a, b, weights=wg, out=out)
        assert r.dlogits.data_ptr() == out.data_ptr()
        close(r.logps, torch.where(live, lp, 0.0), lp_tol(lp), "logps")
        close_grad(out, want, p, flat, coef, U * coef.abs(), 1.0, dtype, "dlogits")


def test_nothing_is_written_outside_the_gradient(L):
    V, rows = 1003, 11
    for dtype in DTYPES:
        z, y, _ = make(rows, V, dtype, 7)
        room = torch.full((rows + 2, V + 9), 3.0, dtype=dtype, device="cuda")
        L.token_logprobs(z.cuda(), y.cuda(), weights=torch.ones(rows, device="cuda"), out=room[1:-1, 4:4 + V])
        edge = room.clone()
        edge[1:-1, 4:4 + V] = 3.0
        assert bool((edge == 3.0).all())


@pytest.mark.parametrize("V", [1000, 32000, 170003])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_gradient_may_replace_the_logits(L, V, dtype):
    z, y, gen = make(8, V, dtype, V + 1)
    w = torch.randn(8, generator=gen).cuda()
    ids = torch.stack([torch.randperm(V, generator=gen)[:5] for _ in range(8)])
    t = torch.randn(8, 5, generator=gen).cuda()
    zg, yg = z.cuda(), y.cuda()
    apart = L.token_logprobs(zg, yg, weights=w).dlogits
    mine = zg.clone()
    assert torch.equal(L.token_logprobs(mine, yg, weights=w, out=mine).dlogits, apart) and torch.equal(mine, apart)
    one = dict(temperature=2.0, targets=yg, hard_weight=0.3, grad=True)
    apart = L.distill_loss(zg, ids.cuda(), t, **one).dlogits
    mine = zg.clone()
    L.distill_loss(mine, ids.cuda(), t, out=mine, **one)
    assert torch.equal(mine, apart)
    ref = torch.zeros(4, device="cuda")
    cu = torch.tensor([0, 3, 4, 6, 8], device="cuda")
    apart = L.preference_loss(zg, yg, ref, cu_seqlens=cu, grad=True).dlogits
    mine = zg.clone()
    L.preference_loss(mine, yg, ref, cu_seqlens=cu, grad=True, out=mine)
    assert torch.equal(mine, apart)


# ----------------------------------------------------------------------------
# infinities, masks of the lowest value, NaN, targets outside the vocabulary
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [6, 700, 5003, 32001, 170003])
@pytest.mark.parametrize("T", [1.0, 0.25])
def test_unusual_logits_stay_in_their_rows(L, V, dtype, T):
    low = torch.finfo(dtype).min
    z, _, gen = make(12, V, dtype, V)
    y = torch.randint(0, V, (12,), generator=gen)
    z[1, V // 2:] = -math.inf            # a padded vocabulary
    y[1] = 0
    z[2] = -math.inf                     # nothing left: NaN
    z[3, 0] = math.inf                   # NaN
    z[4, V - 1] = math.nan               # NaN
    z[5] = low                           # all masked by the lowest value: uniform
    z[6, 1:] = low
    y[6] = 0
    z[7, V - 1] = -math.inf              # the target itself impossible
    y[7] = V - 1
    z[8] = math.nan
    y[8] = IGNORE                        # not read
    y[9] = V                             # outside: NaN
    y[10] = -3
    w = torch.ones(12)
    r = L.token_logprobs(z.cuda(), y.cuda(), weights=w.cuda(), temperature=T)
    lps, grads = r.logps.cpu(), r.dlogits.cpu()
    for t in (2, 3, 4, 9, 10):
        assert math.isnan(lps[t]) and bool(grads[t].isnan().all()), t
    assert lps[8] == 0.0 and not grads[8].any()
    assert lps[7] == -math.inf
    ok = torch.tensor([0, 1, 5, 6, 7, 11])
    lp, p = ref_rows(z[ok], y[ok], T)
    close(lps[ok][lp.isfinite()], lp[lp.isfinite()], lp_tol(lp[lp.isfinite()]) / min(T, 1.0), "logps")
    close_grad(grads[ok], ref_grad(p, y[ok], torch.ones(6).double(), T), p, y[ok], torch.ones(6), U * torch.ones(6), T, dtype, "dlogits")
    assert not grads[1, V // 2:].any()


def test_impossible_targets_in_losses(L):
    # log-probability -inf: the terms are the limits, not NaN
    V = 40
    z, _, gen = make(4, V, torch.float32, 9, masked=0.0)
    z[1, 7] = -math.inf
    y = torch.full((4,), 7)
    zg, yg, f = z.cuda(), y.cuda(), torch.full((4,), -3.0, device="cuda")
    r = L.policy_loss(zg, yg, f, torch.ones(4, device="cuda"), ref_logps=f, kl_coef=0.0, grad=True)
    assert math.isfinite(r.loss) and float(r.kl) == math.inf and not bool(r.dlogits.isnan().any())
    r = L.policy_loss(zg, yg, f, torch.ones(4, device="cuda"), ref_logps=f, kl_coef=0.1)
    assert float(r.loss) == math.inf
    ref = torch.tensor([-3.0, -3.0], device="cuda")
    for rows, want in (([0, 1], 0.0), ([1, 0], math.inf)):         # the rejected, the chosen one impossible
        r = L.preference_loss(zg[rows].view(2, 1, V), yg[:2].view(2, 1), ref)
        assert float(r.loss) == want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_logits_keep_their_differences(L, dtype):
    # 1e4 and more above zero: what counts is the distance to the row's maximum
    z, y, _ = make(6, 1000, dtype, 5, masked=0.0)
    z = (z.double() * 8 + torch.tensor([0, 1e3, -1e4, 3e4, 1e5, -3e5])[:, None]).to(dtype)
    lp, p = ref_rows(z, y, 1.0)
    r = L.token_logprobs(z.cuda(), y.cuda(), weights=torch.ones(6, device="cuda"))
    # distances reach some hundreds here: 2.1 |a| u of those that count stays below EP
    close(r.logps, lp, lp_tol(lp), "logps")
    # (an element at distance d of its maximum is off by 3 d u)
    far = (z.double().max(1, keepdim=True).values - z.double()) * 3 * U
    got, want = r.dlogits.double().cpu(), ref_grad(p, y, torch.ones(6).double(), 1.0)
    near = p * (1 + far / EP)
    near[torch.arange(6), y] += 1
    assert bool(((got - want).abs() <= EP * near + HALF_ULP[dtype] * 1.001 * want.abs() + TINY[dtype]).all())


# ----------------------------------------------------------------------------
# preference
# ----------------------------------------------------------------------------
def ref_preference(lp, y, spans, ref, beta, kind, smooth, average):
    """loss, logps, coefficients of the rows, and how much the coefficient of a
    row can move with an error of 1 in its pair's log ratio."""
    n = len(spans)
    live = y != IGNORE
    seq = torch.zeros(n, dtype=torch.float64)
    err = torch.zeros(n, dtype=torch.float64)
    cnt = [1.0] * n
    for i, (a, b) in enumerate(spans):
        k = live[a:b]
        if average:
            cnt[i] = max(1.0, float(k.sum()))
        seq[i] = lp[a:b][k].sum() / cnt[i]
        err[i] = (lp_tol(lp[a:b][k]) + U * lp[a:b][k].abs()).sum() / cnt[i]
    half = n // 2
    coef, dcoef, losses_, dl = torch.zeros(len(y)).double(), torch.zeros(len(y)).double(), [], []
    for i in range(half):
        D = (seq[i] - ref[i]) - (seq[i + half] - ref[i + half])
        e = err[i] + err[i + half]
        h = beta * D
        if kind == "sigmoid":
            ls = torch.nn.functional.logsigmoid
            losses_.append(-(1 - smooth) * ls(h) - smooth * ls(-h))
            slope, bend = beta * (smooth - torch.sigmoid(-h)), beta * beta / 4
        elif kind == "hinge":
            losses_.append(torch.clamp(1 - h, min=0))
            slope, bend = torch.where(h < 1, -beta, 0.0), 0.0
        else:
            off = D - 1 / (2 * beta)
            losses_.append(off * off)
            slope, bend = 2 * off, 2.0
        dl.append(slope.abs() * e + bend * e * e + 2 * U * losses_[-1].abs())
        for j, sign in ((i, 1.0), (i + half, -1.0)):
            a, b = spans[j]
            coef[a:b] = torch.where(live[a:b], sign * slope / half / cnt[j], 0.0)
            dcoef[a:b] = (bend * e + 2 * U * slope.abs()) / half / cnt[j]
    return torch.stack(losses_).mean(), torch.stack(dl).mean(), seq, err, coef, dcoef


@pytest.mark.parametrize("kind,smooth,average", [("sigmoid", 0.0, False), ("sigmoid", 0.2, True), ("hinge", 0.0, False),
                                                 ("squared", 0.0, True)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,layout", [(50, "padded"), (1003, "packed"), (33000, "padded"), (131077, "packed")])
def test_preference_loss(L, kind, smooth, average, dtype, V, layout):
    gs = 64.0
    if layout == "padded":
        B, S = 6, 5
        spans = [(i * S, (i + 1) * S) for i in range(B)]
        rows = B * S
    else:
        ends = [2, 2, 5, 9, 10, 10, 16, 17, 20]      # an empty one on either side; rows 0, 1 and the last belong to none
        B = len(ends) - 1
        spans = list(zip(ends[:-1], ends[1:]))
        rows = 23
    z, y, gen = make(rows, V, dtype, V, masked=0.25)
    lp, p = ref_rows(z, y, 1.0)
    ref = -8.0 * torch.rand(B, generator=gen) * (1.0 if average else 4.0)
    loss, dl, seq, err, coef, dcoef = ref_preference(lp, y, spans, ref.double(), 0.1, kind, smooth, average)
    kw = dict(beta=0.1, kind=kind, label_smoothing=smooth, average=average)
    zg, yg, rg = z.cuda(), y.cuda(), ref.cuda()
    if layout == "padded":
        zg, yg = zg.view(B, S, V), yg.view(B, S)
    else:
        kw["cu_seqlens"] = torch.tensor(ends, dtype=torch.int64 if average else torch.int32, device="cuda")
    r = L.preference_loss(zg, yg, rg, grad=True, grad_scale=gs, **kw)
    close(r.loss, loss, dl, "loss")
    close(r.logps, seq, err + 2 * U * seq.abs(), "logps")
    close(r.rewards, 0.1 * (seq - ref.double()), 0.1 * err + 2 * U * (seq.abs() + ref.abs()), "rewards")
    close_grad(r.dlogits, ref_grad(p, y, coef * gs, 1.0), p, y, coef * gs, dcoef * gs, 1.0, dtype, "dlogits")
    only = L.preference_loss(zg, yg, rg, **kw)
    assert only.dlogits is None and torch.equal(only.loss, r.loss) and torch.equal(only.logps, r.logps)
    leaf = zg.clone().requires_grad_(True)
    auto = L.preference_loss(leaf, yg, rg, **kw)
    assert auto.loss.requires_grad and not auto.rewards.requires_grad and auto.dlogits is None
    (auto.loss * gs).backward()
    if dtype != torch.float16:      # (there, what is subnormal before the product with gs keeps fewer bits)
        close_grad(leaf.grad, ref_grad(p, y, coef * gs, 1.0), p, y, coef * gs, dcoef * gs, 1.0, dtype, "autograd")
    with pytest.raises(RuntimeError):
        auto.loss.backward()


# ----------------------------------------------------------------------------
# policy
# ----------------------------------------------------------------------------
def ref_policy(lp, y, w, old, adv, ref, low, high, kl):
    live = y != IGNORE
    r = torch.exp(lp - old)
    inside = torch.clip(r, 1 - low, 1 + high)
    free, bound = r * adv, inside * adv
    k, x = torch.zeros_like(lp), torch.zeros_like(lp)
    if ref is not None:
        d = ref - lp
        x = torch.expm1(d)
        k = x - d
    term = -torch.minimum(free, bound) + kl * k
    cut = free > bound
    coef = torch.where(live, w * (torch.where(cut, 0.0, -free) - kl * x), 0.0)
    z = torch.zeros(())
    scale = free.abs() + kl * (x.abs() + 1)      # what an error of the log-probability is multiplied by
    dcoef = torch.where(live, w * (scale * lp_tol(lp) + 4 * U * scale), z)
    dloss = torch.where(live, w * (scale * lp_tol(lp) + 4 * U * (term.abs() + 1)), z).sum()
    return (torch.where(live, w * term, z).sum(), dloss, torch.where(live, w * k, z).sum(),
            torch.where(live, w * cut, z).sum(), coef, dcoef)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,layout,reduction,kl", [(50, "padded", "token", 0.0), (1003, "packed", "sequence", 0.1),
                                                   (33000, "padded", "sequence", 0.05), (170003, "packed", "token", 0.1)])
def test_policy_loss(L, dtype, V, layout, reduction, kl):
    low, high, T, gs = 0.2, 0.3, 0.9, 16.0
    if layout == "padded":
        B, S = 4, 6
        spans, rows = [(i * S, (i + 1) * S) for i in range(B)], B * S
    else:
        ends = [1, 1, 7, 8, 8, 19]
        B, spans, rows = len(ends) - 1, list(zip(ends[:-1], ends[1:])), 21
    z, y, gen = make(rows, V, dtype, V + 5, masked=0.3)
    y[spans[-1][0]] = 3 % V
    lp, p = ref_rows(z, y, T)
    d = 0.3 * torch.randn(rows, generator=gen).double()
    for edge in (math.log1p(-low), math.log1p(high)):     # not on the edge itself
        d = torch.where((d - edge).abs() < 1e-3, d + 4e-3, d)
    old, adv = (lp - d).float(), torch.randn(rows, generator=gen)
    ref = (lp + 0.5 * torch.randn(rows, generator=gen)).float() if kl else None
    yy = y.clone()
    if layout == "packed":
        yy[:spans[0][0]] = IGNORE
        yy[spans[-1][1]:] = IGNORE
    live = yy != IGNORE
    if reduction == "token":
        w = torch.full((rows,), 1.0 / int(live.sum())).double()
    else:
        w = torch.zeros(rows).double()
        for a, b in spans:
            w[a:b] = 1.0 / (B * max(1, int(live[a:b].sum())))
    loss, dloss, k, cut, coef, dcoef = ref_policy(lp, yy, w, old.double(), adv.double(), ref.double() if kl else None,
                                                  low, high, kl)
    zg, args = z.cuda(), [x.cuda() for x in (y, old, adv)]
    refg = ref.cuda() if kl else None
    kw = dict(clip_low=low, clip_high=high, kl_coef=kl, reduction=reduction, temperature=T)
    if layout == "padded":
        zg, args = zg.view(B, S, V), [x.view(B, S) for x in args]
        refg = refg.view(B, S) if kl else None
    else:
        kw["cu_seqlens"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    r = L.policy_loss(zg, *args, ref_logps=refg, grad=True, grad_scale=gs, **kw)
    close(r.loss, loss, dloss, "loss")
    close(r.kl, k, dloss, "kl")
    close(r.clipped, cut, 4 * U, "clipped")
    close(r.logps, torch.where(live, lp, 0.0), lp_tol(lp), "logps")
    close_grad(r.dlogits, ref_grad(p, yy, coef * gs, T), p, yy, coef * gs, dcoef * gs, T, dtype, "dlogits")
    only = L.policy_loss(zg, *args, ref_logps=refg, **kw)
    assert only.dlogits is None and abs(float(only.loss) - float(r.loss)) <= float(dloss)
    leaf = zg.clone().requires_grad_(True)
    L.policy_loss(leaf, *args, ref_logps=refg, grad_scale=gs, **kw).loss.backward()
    assert torch.equal(leaf.grad, r.dlogits)
    if reduction == "token":
        n = float(live.sum())
        s = L.policy_loss(zg, *args, ref_logps=refg, denominator=4 * n, **kw)
        close(s.loss, loss / 4, dloss, "loss over a given count")


# calls of up to 256 rows make their totals themselves, from 8193 rows on short rows share a wave
@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,S,V", [(5, 51, 77), (1, 256, 300), (257, 1, 1100), (3, 2735, 90), (2, 4099, 333), (41, 200, 700),
                                   (7, 1200, 1500), (3, 100, 5000)])
def test_policy_loss_over_many_rows(L, B, S, V, dtype, reduction):
    rows, kl = B * S, 0.1
    z, y, gen = make(rows, V, dtype, rows + V, masked=0.4)
    y.view(B, S)[B // 2] = IGNORE              # a sequence with nothing to train on
    y[0] = 1
    lp, p = ref_rows(z, y, 1.0)
    d = 0.3 * torch.randn(rows, generator=gen).double()
    for edge in (math.log1p(-0.2), math.log1p(0.2)):
        d = torch.where((d - edge).abs() < 1e-3, d + 4e-3, d)
    old, adv = (lp - d).float(), torch.randn(rows, generator=gen)
    ref = (lp + 0.5 * torch.randn(rows, generator=gen)).float()
    live = y != IGNORE
    if reduction == "token":
        w = torch.full((rows,), 1.0 / int(live.sum())).double()
    else:
        w = (1.0 / (B * live.view(B, S).sum(1, keepdim=True).clamp(min=1).double())).expand(B, S).reshape(-1)
    loss, dloss, k, cut, coef, dcoef = ref_policy(lp, y, w, old.double(), adv.double(), ref.double(), 0.2, 0.2, kl)
    r = L.policy_loss(z.cuda().view(B, S, V), *[x.cuda().view(B, S) for x in (y, old, adv)], ref_logps=ref.cuda().view(B, S),
                      kl_coef=kl, reduction=reduction, grad=True)
    close(r.loss, loss, dloss, "loss")
    close(r.kl, k, dloss, "kl")
    close(r.clipped, cut, 4 * U, "clipped")
    close(r.logps, torch.where(live, lp, 0.0), lp_tol(lp), "logps")
    close_grad(r.dlogits, ref_grad(p, y, coef, 1.0), p, y, coef, dcoef, 1.0, dtype, "dlogits")


@pytest.mark.parametrize("rows", [255, 256, 257, 1500])
def test_distillation_totals(L, rows):
    V, K = 260, 9
    z, y, gen = make(rows, V, torch.bfloat16, rows)
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(rows)])
    t = torch.randn(rows, K, generator=gen)
    r = L.distill_loss(z.cuda(), ids.cuda(), t.cuda(), targets=y.cuda(), hard_weight=0.2, temperature=1.5, grad=True)
    n = int((y != IGNORE).sum())
    per, grad, ptol, tol = ref_distill(z, ids, t, y, 1.5, None, 0.2, n)
    close(r.losses, per, ptol, "losses")
    close(r.loss, per.sum() / n, ptol.sum() / n, "loss")
    off = (r.dlogits.double().cpu() - grad).abs()
    assert bool((off <= tol + HALF_ULP[torch.bfloat16] * 1.001 * grad.abs() + TINY[torch.bfloat16]).all())


def test_many_pairs(L):
    n, V = 600, 64                              # 300 pairs of one to four rows
    gen = torch.Generator().manual_seed(3)
    ends = [0] + torch.randint(0, 5, (n,), generator=gen).cumsum(0).tolist()
    rows = ends[-1]
    z, y, gen = make(rows, V, torch.float32, 8, masked=0.2)
    lp, p = ref_rows(z, y, 1.0)
    ref = -6.0 * torch.rand(n, generator=gen)
    spans = list(zip(ends[:-1], ends[1:]))
    loss, dl, seq, err, coef, dcoef = ref_preference(lp, y, spans, ref.double(), 0.2, "sigmoid", 0.0, False)
    r = L.preference_loss(z.cuda(), y.cuda(), ref.cuda(), beta=0.2, cu_seqlens=torch.tensor(ends, device="cuda"), grad=True)
    close(r.loss, loss, dl, "loss")
    close(r.logps, seq, err + 2 * U * seq.abs(), "logps")
    close_grad(r.dlogits, ref_grad(p, y, coef, 1.0), p, y, coef, dcoef, 1.0, torch.float32, "dlogits")


def test_fp16_gradients_survive_until_a_loss_scaler_multiplies_them(L):
    # averaged over 4096 rows most elements lie below fp16's smallest value;
    # made with the scale, or recorded (times the power of two in the number of
    # rows, or pairs) and scaled in backward, they are the same up to a second
    # rounding, and up to what a subnormal element lost before the scale
    B, S, V, scale = 32, 128, 600, 2.0 ** 16
    z, y, gen = make(B * S, V, torch.float16, 21)
    zg, yg = z.cuda().view(B, S, V), y.cuda().view(B, S)
    f = torch.full((B, S), -6.0, device="cuda")
    adv = torch.randn(B, S, generator=gen).cuda()
    ids = torch.stack([torch.randperm(V, generator=gen)[:4] for _ in range(B * S)]).cuda().view(B, S, 4)
    t = torch.randn(B, S, 4, generator=gen).cuda()
    base = torch.full((B,), -600.0, device="cuda")
    calls = [(lambda x, **k: L.policy_loss(x, yg, f, adv, **k), 4096),
             (lambda x, **k: L.distill_loss(x, ids, t, targets=yg, **k), 4096),
             (lambda x, **k: L.preference_loss(x, yg, base, beta=0.1, **k), 16)]
    for call, ahead in calls:
        want = call(zg, grad=True, grad_scale=scale).dlogits.double()
        leaf = zg.clone().requires_grad_(True)
        (call(leaf).loss * scale).backward()
        off = (leaf.grad.double() - want).abs()
        assert bool((off <= 2.0 ** -10 * want.abs() + 2.0 ** -25 * scale / ahead + 2.0 ** -24).all())


def test_advantages_of_a_sequence_are_expanded_not_copied(L):
    B, S, V = 3, 5, 200
    z, y, gen = make(B * S, V, torch.bfloat16, 2)
    a = torch.randn(B, 1, generator=gen).cuda().expand(B, S)
    old = torch.full((B, S), -3.0, device="cuda")
    zg, yg = z.cuda().view(B, S, V), y.cuda().view(B, S)
    one, two = (L.policy_loss(zg, yg, old, x, grad=True) for x in (a, a.contiguous()))
    assert torch.equal(one.loss, two.loss) and torch.equal(one.dlogits, two.dlogits)


def test_without_trained_rows_everything_is_zero(L):
    B, S, V = 4, 3, 1000
    z = torch.randn(B, S, V, device="cuda")
    y = torch.full((B, S), IGNORE, device="cuda")
    f = torch.full((B, S), math.nan, device="cuda")
    ids = torch.zeros(B, S, 2, dtype=torch.int64, device="cuda")
    for red in ("token", "sequence"):
        r = L.policy_loss(z, y, f, f, ref_logps=f, kl_coef=0.1, reduction=red, grad=True)
        assert float(r.loss) == 0.0 and float(r.kl) == 0.0 and not r.dlogits.any() and not r.logps.any()
    r = L.distill_loss(z, ids, torch.ones(B, S, 2, device="cuda"), targets=y, grad=True)
    assert float(r.loss) == 0.0 and not r.losses.any() and not r.dlogits.any()
    r = L.preference_loss(z, y, torch.zeros(B, device="cuda"), grad=True)
    assert abs(float(r.loss) - math.log(2.0)) < 1e-6 and not r.dlogits.any()


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------
def ref_distill(z, ids, t, y, T, lse, hard, n):
    """Row losses, gradient and the tolerance of both, row by row as defined."""
    rows, V = z.shape
    grad, tol = torch.zeros(rows, V).double(), torch.zeros(rows, V).double()
    per, ptol = torch.zeros(rows).double(), torch.zeros(rows).double()
    for i in range(rows):
        if y is not None and int(y[i]) == IGNORE:
            continue
        x = z[i].double()
        logq = torch.log_softmax(x / T, 0)
        q = logq.exp()
        ent = [(int(j), float(v) / T) for j, v in zip(ids[i], t[i].double()) if int(j) >= 0 and float(v) != -math.inf]
        mass = torch.zeros(V).double()
        kl, rest, dkl = 0.0, 0.0, 0.0
        out = torch.ones(V, dtype=torch.bool)
        if ent:
            a = torch.tensor([v for _, v in ent]).double()
            logp = a - (torch.logsumexp(a, 0) if lse is None else float(lse[i]))
            for (j, _), lk in zip(ent, logp):
                mass[j] += lk.exp()
                out[j] = False
                kl += float(lk.exp() * (lk - logq[j]))
            if lse is not None and bool(out.any()):
                rest = 1.0 - float(logp.exp().sum())
                rest = rest if rest >= 2.0 ** -20 else 0.0
        lead = float(mass.sum()) + rest
        g = q * lead - mass
        e = q * lead * EP + 2 * U * mass
        if rest:
            logr = torch.logsumexp(logq[out], 0)
            kl += rest * float(math.log(rest) - logr)
            g = g - rest * torch.where(out, (logq - logr).exp(), 0.0)
            e = e + 2 * EP * rest * torch.where(out, (logq - logr).exp(), 0.0)
        dkl = 2 * EP * lead + 4 * U * abs(kl)
        per[i], grad[i], tol[i], ptol[i] = (1 - hard) * T * T * kl, (1 - hard) * T * g, (1 - hard) * T * e, (1 - hard) * T * T * dkl
        if hard:
            l1 = torch.log_softmax(x, 0)
            per[i] -= hard * float(l1[int(y[i])])
            ptol[i] += hard * float(lp_tol(l1[int(y[i])]))
            grad[i] += hard * l1.exp()
            grad[i, int(y[i])] -= hard
            tol[i] += hard * l1.exp() * EP
            tol[i, int(y[i])] += 2 * U * hard
    return per, grad / n, ptol + 4 * U * per.abs(), tol / n


@pytest.mark.parametrize("V,K", [(5, 5), (40, 1), (300, 300), (1003, 16), (4100, 64), (32000, 7), (50265, 130), (131077, 1024),
                                 (170003, 33)])
@pytest.mark.parametrize("lse,hard,T", [(False, 0.0, 1.0), (False, 0.4, 2.0), (True, 0.0, 2.0), (True, 0.3, 1.0), (True, 0.3, 0.5)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_distillation(L, V, K, lse, hard, T, dtype):
    rows, gs = (6 if V > 20000 else 11), 8.0
    z, y, gen = make(rows, V, dtype, V + K, masked=0.2)
    y[3] = 2 % V
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(rows)])
    t = (3.0 * torch.randn(rows, K, generator=gen)).to(dtype)
    ids[0, K // 2:] = -1                  # a shorter list
    ids[1] = -1                           # none
    y[0], y[1] = int(ids[0, 0].clamp(min=0)), 1 % V
    if K > 3:
        t[2, 1] = -math.inf               # absent by its logit
        ids[4, 2] = ids[4, 0]             # a repeated token
        ids[4, 3] = ids[4, 0]
        y[4] = ids[4, 0]                  # which is the target, too
    if K == V:
        ids[5] = torch.randperm(V, generator=gen)       # nothing outside the list
    a = torch.where(ids >= 0, t.double() / T, -math.inf)
    full = torch.logsumexp(a, 1)
    share = torch.tensor([0.9, 0.5, 0.7, 0.999, 0.6, 0.8] * 2)[:rows].double()
    ls = torch.where(full.isfinite(), full - share.log(), 0.0).float() if lse else None
    n = int((y != IGNORE).sum())
    per, grad, ptol, tol = ref_distill(z, ids, t, y, T, ls, hard, n)
    kw = dict(temperature=T, teacher_lse=ls.cuda() if lse else None, targets=y.cuda(), hard_weight=hard)
    zg, ig, tg = z.cuda(), (ids.int() if K % 2 else ids).cuda(), t.cuda()
    r = L.distill_loss(zg, ig, tg, grad=True, grad_scale=gs, **kw)
    close(r.losses, per, ptol, "losses")
    close(r.loss, per.sum() / n, ptol.sum() / n, "loss")
    got, want = r.dlogits.double().cpu(), grad * gs
    lim = tol * gs + HALF_ULP[dtype] * 1.001 * want.abs() + TINY[dtype]
    off = (got - want).abs()
    assert bool((off <= lim).all()), (float((off / lim).max()), (off > lim).nonzero()[:3].tolist())
    only = L.distill_loss(zg, ig, tg, **kw)
    assert only.dlogits is None and torch.equal(only.losses, r.losses)
    leaf = zg.clone().requires_grad_(True)
    L.distill_loss(leaf, ig, tg, **kw).loss.backward(torch.tensor(gs, device="cuda"))
    assert torch.equal(leaf.grad, r.dlogits)


def test_distillation_without_targets_counts_every_row(L):
    z, _, gen = make(10, 500, torch.float16, 1)
    ids = torch.stack([torch.randperm(500, generator=gen)[:4] for _ in range(10)])
    t = torch.randn(10, 4, generator=gen)
    per, grad, ptol, tol = ref_distill(z, ids, t, None, 1.5, None, 0.0, 10)
    three = L.distill_loss(z.cuda().view(2, 5, 500), ids.cuda().view(2, 5, 4), t.cuda().view(2, 5, 4), temperature=1.5, grad=True)
    close(three.loss, per.sum() / 10, ptol.sum() / 10, "loss")
    off = (three.dlogits.double().cpu().view(10, 500) - grad).abs()
    assert bool((off <= tol + HALF_ULP[torch.float16] * 1.001 * grad.abs() + TINY[torch.float16]).all())
    given = L.distill_loss(z.cuda(), ids.cuda(), t.cuda(), temperature=1.5, denominator=40)
    close(given.loss, per.sum() / 40, ptol.sum() / 40, "loss over a given count")


def test_distillation_with_bad_indices_and_rows(L):
    V = 300
    z, y, gen = make(6, V, torch.float32, 4, masked=0.0)
    ids = torch.stack([torch.randperm(V, generator=gen)[:4] for _ in range(6)])
    t = torch.randn(6, 4, generator=gen)
    ids[1, 2] = V                     # outside: the row is NaN
    ids[2, 1] = 1 << 40
    z[3, 5] = math.nan
    y[4] = V + 1
    r = L.distill_loss(z.cuda(), ids.cuda(), t.cuda(), targets=y.cuda(), hard_weight=0.5, grad=True)
    bad = r.losses.isnan().cpu()
    assert bad.tolist() == [False, True, True, True, True, False]
    assert bool(r.dlogits[bad.cuda()].isnan().all()) and not bool(r.dlogits[~bad.cuda()].isnan().any())


# ----------------------------------------------------------------------------
# gradients against differences
# ----------------------------------------------------------------------------
def test_gradients_against_differences(L):
    # (L(z + h v) - L(z - h v)) / 2h with v of norm 1: off by at most
    # max|L'''| h^2 / 6 and by the rounding of the two losses, u |L| / h
    V, B, S, h = 40, 4, 3, 2.0 ** -7
    z, y, gen = make(B * S, V, torch.float32, 11, masked=0.2)
    zg, yg = z.cuda().view(B, S, V), y.cuda().view(B, S)
    lp = torch.where(yg >= 0, L.token_logprobs(zg, yg).logps, torch.zeros((), device="cuda"))
    old, adv = lp - 0.05, torch.randn(B, S, generator=gen).cuda()
    refs = lp + 0.3
    ids = torch.stack([torch.randperm(V, generator=gen)[:6] for _ in range(B * S)]).cuda().view(B, S, 6)
    t = torch.randn(B, S, 6, generator=gen).cuda()
    lse = t.div(2.0).logsumexp(-1) + 0.3
    calls = [
        lambda x: L.preference_loss(x, yg, torch.full((B,), -9.0, device="cuda"), beta=0.3, label_smoothing=0.1, grad=True),
        lambda x: L.policy_loss(x, yg, old, adv, ref_logps=refs, kl_coef=0.2, grad=True),
        lambda x: L.distill_loss(x, ids, t, temperature=2.0, teacher_lse=lse, targets=yg, hard_weight=0.3, grad=True),
    ]
    for k, f in enumerate(calls):
        base = f(zg)
        for _ in range(4):
            v = torch.randn(B, S, V, generator=gen).cuda()
            v /= v.norm()
            diff = (float(f(zg + h * v).loss.double()) - float(f(zg - h * v).loss.double())) / (2 * h)
            along = float((base.dlogits.double() * v.double()).sum())
            assert abs(diff - along) <= 6.0 * h * h + (4 * U + EP / 8) * abs(float(base.loss)) / h + 2 * EP, (k, diff, along)


# ----------------------------------------------------------------------------
# streams, graphs, repeats, long offsets
# ----------------------------------------------------------------------------
def _all(L, z, y, f, g, ids, t):
    r = [L.token_logprobs(z, y, weights=f), L.preference_loss(z, y, g, grad=True),
         L.policy_loss(z, y, f, f, ref_logps=f, kl_coef=0.1, grad=True),
         L.policy_loss(z, y, f, f, reduction="sequence", grad=True),
         L.distill_loss(z, ids, t, temperature=2.0, targets=y, hard_weight=0.2, grad=True)]
    return [x for one in r for x in one if x is not None]


def _inputs(B, S, V, seed, dtype=torch.bfloat16):
    z, y, gen = make(B * S, V, dtype, seed)
    ids = torch.stack([torch.randperm(V, generator=gen)[:6] for _ in range(B * S)]).view(B, S, 6)
    return [x.cuda() for x in (z.view(B, S, V), y.view(B, S), torch.randn(B, S, generator=gen) - 3, torch.randn(B, generator=gen) - 9,
                               ids, torch.randn(B, S, 6, generator=gen))]


def test_repeated_calls_give_the_same_bits(L):
    a = _inputs(4, 100, 5003, 1)
    first = _all(L, *a)
    for _ in range(3):
        for x, y in zip(first, _all(L, *a)):
            assert torch.equal(x, y)


def test_another_stream(L):
    a = _inputs(4, 50, 32000, 2)
    want = _all(L, *a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            big = big @ big * 1e-2       # work the losses have to come after
        z = (a[0].float() + big.sum().nan_to_num(0.0, 0.0, 0.0) * 0).to(a[0].dtype)
        got = _all(L, z, *a[1:])
    side.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_calls_on_two_streams_at_once(L):
    # each stream has scratch of its own
    a, b = _inputs(4, 50, 9001, 7), _inputs(4, 60, 9001, 8)
    want = [_all(L, *x) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for k, x in enumerate((a, b)):
            with torch.cuda.stream(streams[k]):
                got[k].append(_all(L, *x))
    torch.cuda.synchronize()
    for k in range(2):
        for one in got[k]:
            for x, y in zip(one, want[k]):
                assert torch.equal(x, y)


def test_captured_calls_replay(L):
    a, b = _inputs(4, 50, 5003, 3), _inputs(4, 50, 5003, 4)
    static = [x.clone() for x in a]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _all(L, *static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all(L, *static)
    for k in range(6):
        src = (a, b)[k % 2]
        for s, x in zip(static, src):
            s.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, _all(L, *src)):
            assert torch.equal(x, y), k


def test_more_rows_than_one_launch_holds(L):
    # 2^21 workgroups of 32 rows (of one in the backward pass) and more; a row of two logits
    rows = (1 << 26) + 5
    z = torch.randn(rows, 2, device="cuda")
    y = (torch.arange(rows, device="cuda") % 2)
    r = L.token_logprobs(z, y, weights=torch.ones(rows, device="cuda"))
    some = torch.tensor([0, 1, (1 << 26) - 1, 1 << 26, rows - 1], device="cuda")
    lp, p = ref_rows(z[some].cpu(), y[some].cpu(), 1.0)
    close(r.logps[some], lp, lp_tol(lp), "logps")
    d = (z[:, 0] - z[:, 1]) * torch.where(y == 0, 1.0, -1.0)
    assert bool(((r.logps + torch.log1p(torch.exp(-d.abs())) + (-d).clamp(min=0)).abs() < 1e-4).all())
    out = L.token_logprobs(z.requires_grad_(True), y).logps      # its backward: a workgroup a row
    out.sum().backward()
    assert torch.allclose(z.grad, r.dlogits, rtol=0, atol=4e-5)


def test_offsets_beyond_32_bits(L):
    V, rows = 131077, 16500                     # 2.16e9 logits
    z = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    z.normal_()
    y = torch.randint(0, V, (rows,), device="cuda")
    some = torch.tensor([0, 8191, 16384, rows - 2, rows - 1], device="cuda")
    lp, p = ref_rows(z[some].cpu(), y[some].cpu(), 1.0)
    r = L.token_logprobs(z, y, weights=torch.ones(rows, device="cuda"), out=z)
    close(r.logps[some], lp, lp_tol(lp), "logps")
    one = torch.ones(5)
    close_grad(z[some], ref_grad(p, y[some].cpu(), one.double(), 1.0), p, y[some].cpu(), one, U * one, 1.0, torch.bfloat16, "dlogits")
    # a batch stride beyond 2^31 elements
    z.normal_()
    far = z.as_strided((2, 3, V), (rows // 2 * 2 * V - 3 * V, V, 1))
    yy = y[:6].view(2, 3)
    lp, _ = ref_rows(far.reshape(6, V).cpu(), yy.reshape(-1).cpu(), 1.0)
    close(L.token_logprobs(far, yy).logps, lp.view(2, 3), lp_tol(lp).view(2, 3), "logps")


# ----------------------------------------------------------------------------
# refusals
# ----------------------------------------------------------------------------
def test_refusals(L, gpu_lib):
    z, y = torch.zeros(4, 9, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    with pytest.raises(TypeError, match="targets"):
        L.token_logprobs(z, f)
    with pytest.raises(ValueError, match="targets"):
        L.token_logprobs(z, y[:3])
    with pytest.raises(ValueError, match="targets must live"):
        L.token_logprobs(z, y.cpu())
    with pytest.raises(ValueError, match="contiguous"):
        L.token_logprobs(z.T.contiguous().T, y)
    with pytest.raises(TypeError, match="weights"):
        L.token_logprobs(z, y, weights=f.double())
    with pytest.raises(ValueError, match="weights"):
        L.token_logprobs(z, y, weights=f[:1])
    with pytest.raises(ValueError, match="out"):
        L.token_logprobs(z, y, out=z)
    with pytest.raises(TypeError, match="out"):
        L.token_logprobs(z, y, weights=f, out=z.half())
    with pytest.raises(ValueError, match="strides"):
        L.token_logprobs(z[:2], y[:2], weights=f[:2], out=z.as_strided((2, 9), (18, 1)))
    with pytest.raises(gpu_lib.GlrError, match="overlap"):
        L.token_logprobs(z, y, weights=f, out=torch.zeros(1, 9, device="cuda").expand(4, 9))
    with pytest.raises(gpu_lib.GlrError, match="temperature"):
        L.token_logprobs(z, y, temperature=0.0)
    with pytest.raises(ValueError, match="cu_seqlens"):
        L.preference_loss(z, y, f)
    with pytest.raises(ValueError, match="ref_logps"):
        L.preference_loss(z.view(2, 2, 9), y.view(2, 2), f)
    with pytest.raises(ValueError, match="packed"):
        L.preference_loss(z.view(2, 2, 9), y.view(2, 2), f[:2], cu_seqlens=torch.tensor([0, 2, 4], device="cuda"))
    with pytest.raises(TypeError, match="cu_seqlens"):
        L.preference_loss(z, y, f[:2], cu_seqlens=torch.tensor([0.0, 2, 4], device="cuda"))
    with pytest.raises(gpu_lib.GlrError, match="even"):
        L.preference_loss(z, y, f[:3], cu_seqlens=torch.tensor([0, 2, 3, 4], device="cuda"))
    with pytest.raises(gpu_lib.GlrError, match="ref_logps"):
        L.policy_loss(z, y, f, f, kl_coef=0.1)
    with pytest.raises(ValueError, match="advantages"):
        L.policy_loss(z, y, f, f[:2])
    with pytest.raises(gpu_lib.GlrError, match="token reduction"):
        L.policy_loss(z.view(2, 2, 9), y.view(2, 2), f.view(2, 2), f.view(2, 2), reduction="sequence", denominator=3.0)
    with pytest.raises(ValueError, match="teacher_logits"):
        L.distill_loss(z, y[:, None], f[:, None, None])
    with pytest.raises(ValueError, match="teacher_ids"):
        L.distill_loss(z, y, f)
    with pytest.raises(gpu_lib.GlrError, match="hard_weight"):
        L.distill_loss(z, y[:, None], f[:, None], hard_weight=0.5)
    with pytest.raises(gpu_lib.GlrError, match="top"):
        L.distill_loss(z, torch.zeros(4, 1025, dtype=torch.int64, device="cuda"), torch.zeros(4, 1025, device="cuda"))


def test_sequence_offsets_outside_the_rows_are_clamped(L):
    z, y, _ = make(8, 100, torch.float32, 6, masked=0.0)
    zg, yg = z.cuda(), y.cuda()
    ref = torch.zeros(2, device="cuda")
    want = L.preference_loss(zg, yg, ref, cu_seqlens=torch.tensor([0, 3, 8], device="cuda"), grad=True)
    got = L.preference_loss(zg, yg, ref, cu_seqlens=torch.tensor([-5, 3, 1 << 40], device="cuda"), grad=True)
    assert torch.equal(want.loss, got.loss) and torch.equal(want.dlogits, got.dlogits)


# ----------------------------------------------------------------------------
# together, under DistributedDataParallel with the compression hook
# ----------------------------------------------------------------------------
def test_the_example_trains(gpu_lib):
    import importlib.util
    import os
    import socket
    from datetime import timedelta

    import torch.distributed as dist

    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_losses.py")
    spec = importlib.util.spec_from_file_location("train_losses", at)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    dist.init_process_group("nccl", init_method=f"tcp://127.0.0.1:{port}", rank=0, world_size=1,
                            timeout=timedelta(seconds=60))
    try:
        out = example.main(steps=30)
    finally:
        dist.destroy_process_group()
    assert out["pretrain"][1] < 0.9 * out["pretrain"][0]
    assert out["distill"][1] < 0.9 * out["distill"][0]
    assert out["preference"][1] < out["preference"][0] + 0.02       # (starts at log 2, where the reference is)
    assert out["reward"][1] > out["reward"][0] + 0.05
