"""Log-probabilities, the policy loss and the preference loss on the GPU against their plain 64-bit forms (loss_ref.py, which also
derives the tolerances)."""
import math

import pytest
import torch

import loss_ref as R

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def am():
    import paper_2512_11280_amd as am
    am.load_library()
    assert torch.cuda.is_available()
    return am


class Case:
    """Inputs of one call on the CPU: rows with a peak, tokens on and off it, weights with masked positions."""

    def __init__(self, B, T, V, dtype, seed=0, masked=0.3, std=3.0):
        g = torch.Generator().manual_seed(1000 * seed + 7 * B + 3 * T + V)
        self.n = lambda *s: torch.randn(*s, generator=g)                                     # noqa: E731
        z = std * self.n(B, T, V)
        peak = torch.randint(0, V, (B, T), generator=g)
        z.scatter_add_(-1, peak[..., None], torch.full((B, T, 1), 8.0))
        self.z = z.to(dtype)
        other = torch.randint(0, V, (B, T), generator=g)
        self.x = torch.where(torch.rand(B, T, generator=g) < 0.6, peak, other).to(torch.int32)
        self.w = torch.rand(B, T, generator=g) * (torch.rand(B, T, generator=g) >= masked)
        self.lp = torch.nan_to_num(R.rows(self.z, self.x)["lp"])
        self.B, self.T, self.V, self.dtype = B, T, V, dtype

    def ws(self, am):
        return am.LossWorkspace(self.B, self.T, self.V, self.dtype)

    def old(self):
        """Earlier log-probabilities whose ratio to the present ones is off the clipping's borders (0.8, 1.2) and off 1."""
        d = 0.3 * self.n(self.B, self.T).double()
        for border in (math.log(0.8), math.log(1.2)):
            d = torch.where((d - border).abs() < 1e-3, d + 2e-3, d)
        return (self.lp - d).float()


def cu(t):
    return None if t is None else t.cuda()


SHAPES = [(1, 1, 1), (2, 3, 7), (2, 2, 8), (3, 5, 9), (2, 17, 255), (4, 3, 2049), (2, 65, 5003), (6, 7, 32003), (2, 2, 128256), (2, 1, 152064)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("shape", SHAPES)
def test_logprob_and_its_gradient(am, shape, dtype):
    c = Case(*shape, dtype)
    active = (c.w != 0).to(torch.uint8)
    ws = c.ws(am)
    lp, H, st = am.token_logprob(c.z.cuda(), c.x.cuda(), ws, active=active.cuda())
    o, on = R.rows(c.z, c.x), active.bool()
    R.near(lp, torch.where(on, o["lp"], 0.0), R.tol_lp(o), "logprob")
    R.near(H, torch.where(on, o["H"], 0.0), R.tol_H(o), "entropy")
    assert not st.any()
    a, h = c.n(*c.x.shape), c.n(*c.x.shape)
    for dH in (None, h):
        got = am.token_logprob_grad(c.z.cuda(), c.x.cuda(), ws, a.cuda(), cu(dH), active=active.cuda())
        g, tol = R.grad(o, torch.where(on, a, 0.0), None if dH is None else torch.where(on, h, 0.0), dtype=dtype)
        R.near(got, g, tol, "dlogits")
        assert got.dtype == dtype


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [1, 13, 4099, 128256])
def test_single_tokens(am, V, dtype):
    """The serving form: logits [B, V], one token each."""
    c = Case(5, 1, V, dtype)
    ws = am.LossWorkspace(5, 1, V, dtype)
    lp, H, st = am.token_logprob(c.z[:, 0].cuda(), c.x[:, 0].cuda(), ws)
    o = R.rows(c.z[:, 0], c.x[:, 0])
    assert lp.shape == H.shape == st.shape == (5,)
    R.near(lp, o["lp"], R.tol_lp(o), "logprob")
    R.near(H, o["H"], R.tol_H(o), "entropy")
    g = am.token_logprob_grad(c.z[:, 0].cuda(), c.x[:, 0].cuda(), ws, torch.ones(5, device="cuda"))
    R.near(g, *R.grad(o, torch.ones(5), dtype=dtype), "dlogits")


def _policy(am, c, kl="none", ent=0.0, kl_coef=0.05, old=True, weight=True, scale=None, z=None, zref=None, per_seq=False, ws=None, **kw):
    adv = c.n(c.B) if per_seq else c.n(c.B, c.T)
    adv.view(-1)[0] = 0.0
    old = c.old() if old else None
    ref = (c.lp + 0.4 * c.n(c.B, c.T).double()).float() if kl == "sampled" else None
    if kl == "full" and zref is None:
        zref = (c.z.float() + 0.7 * c.n(c.B, c.T, c.V)).to(c.dtype)
    w = c.w if weight else None
    o = am.policy_loss((c.z if z is None else z).cuda(), c.x.cuda(), adv.cuda(), ws or c.ws(am), weight=cu(w), old_logprob=cu(old),
                       ref_logprob=cu(ref), ref_logits=cu(zref), options=am.PolicyOptions(kl_coef=kl_coef, entropy_coef=ent),
                       grad_scale=None if scale is None else torch.tensor([scale], device="cuda"), **kw)
    e = R.policy(c.z if z is None else z, c.x, adv, weight=w, old=old, ref=ref, zref=zref, kl_coef=kl_coef if kl != "none" else 0.0, ent=ent,
                 scale=1.0 if scale is None else scale)
    R.near(o.token_loss, e["term"], e["term_tol"], "token_loss")
    R.near(o.logprob, e["lp"], e["lp_tol"], "logprob")
    R.near(o.entropy, e["H"], e["H_tol"], "entropy")
    R.near(o.kl, e["kl"], e["kl_tol"], "kl")
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    if o.dlogits is not None:
        R.near(o.dlogits, e["g"], e["g_tol"], "dlogits")
    return o, e


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("ent", [0.0, 0.02])
@pytest.mark.parametrize("shape", [(2, 3, 7), (3, 5, 9), (2, 17, 2049), (6, 7, 32003), (2, 2, 128256)])
def test_policy_loss(am, shape, kl, ent, dtype):
    _policy(am, Case(*shape, dtype, seed=1), kl, ent)


@pytest.mark.parametrize("dtype", [BF, F])
def test_policy_loss_forms(am, dtype):
    """Advantages per sequence, no weights, no old log-probabilities, a loss scale, no gradient, a coefficient of zero."""
    _policy(am, Case(4, 9, 1003, dtype, seed=2), per_seq=True, scale=16.0)
    _policy(am, Case(4, 9, 1003, dtype, seed=3), "sampled", weight=False)
    _policy(am, Case(4, 9, 1003, dtype, seed=4), "full", 0.1, old=False)
    o, _ = _policy(am, Case(4, 9, 1003, dtype, seed=5), "full", 0.1, need_grad=False)
    assert o.dlogits is None
    _policy(am, Case(4, 9, 1003, dtype, seed=6), "full", kl_coef=0.0)
    _policy(am, Case(4, 9, 1003, dtype, seed=6), "sampled", kl_coef=0.0)


def _preference(am, c, kind="logistic", beta=0.1, margin=0.0, smoothing=0.0, ref=True, pair_weight=None, weight="mask", scale=None, ws=None, **kw):
    w = (c.w != 0).float() if weight == "mask" else c.w if weight == "any" else None
    r = (c.lp + 0.3 * c.n(c.B, c.T).double()).float() if ref else None
    o = am.preference_loss(c.z.cuda(), c.x.cuda(), ws or c.ws(am), weight=cu(w), ref_logprob=cu(r), pair_weight=cu(pair_weight),
                           options=am.PreferenceOptions(kind=kind, beta=beta, margin=margin, label_smoothing=smoothing),
                           grad_scale=None if scale is None else torch.tensor([scale], device="cuda"), **kw)
    e = R.preference(c.z, c.x, weight=w, ref=r, pair_weight=pair_weight, kind=kind, beta=beta, margin=margin, smoothing=smoothing,
                     scale=1.0 if scale is None else scale)
    R.near(o.logprob, e["lp"], e["lp_tol"], "logprob")
    R.near(o.score, e["score"], e["score_tol"], "score")
    R.near(o.margin, e["margin"], e["margin_tol"], "margin")
    R.near(o.pair_loss, e["pair"], e["pair_tol"], "pair_loss")
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    if o.dlogits is not None:
        R.near(o.dlogits, e["g"], e["g_tol"], "dlogits")
    return o, e


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind", ["logistic", "squared", "hinge"])
@pytest.mark.parametrize("shape", [(2, 1, 7), (2, 3, 9), (6, 17, 2049), (4, 7, 32003), (2, 2, 128256)])
def test_preference_loss(am, shape, kind, dtype):
    _preference(am, Case(*shape, dtype, seed=1), kind, smoothing=0.1 if kind == "logistic" else 0.0)


@pytest.mark.parametrize("dtype", [BF, F])
def test_preference_loss_forms(am, dtype):
    _preference(am, Case(6, 9, 1003, dtype, seed=2), margin=0.5, ref=False, weight="any", scale=8.0)
    _preference(am, Case(6, 9, 1003, dtype, seed=3), weight=None, pair_weight=torch.tensor([0.5, 0.0, 2.0]))
    _preference(am, Case(6, 9, 1003, dtype, seed=4), "hinge", beta=3.0)           # margins on both sides of the corner
    o, _ = _preference(am, Case(6, 9, 1003, dtype, seed=5), "squared", need_grad=False)
    assert o.dlogits is None
    c = Case(4, 3, 50, dtype, seed=6)
    c.w[1] = 0.0                                                                   # a sequence of which nothing counts
    c.w[3] = 0.0
    _preference(am, c)


def test_rows_that_do_not_count_are_not_read(am):
    """NaN logits, tokens outside the vocabulary and other inputs that are no numbers, in positions of weight 0."""
    c = Case(3, 5, 2050, BF, seed=8, masked=0.5)
    off = c.w == 0
    assert off.any() and not off.all()
    z, x, nan = c.z.clone(), c.x.clone(), torch.tensor(math.nan)
    z[off], x[off] = math.nan, -100
    adv, old = torch.where(off, nan, c.n(3, 5)), torch.where(off, nan, c.old())
    o = am.policy_loss(z.cuda(), x.cuda(), adv.cuda(), c.ws(am), weight=c.w.cuda(), old_logprob=old.cuda(), ref_logits=z.cuda(),
                       options=am.PolicyOptions(kl_coef=0.1, entropy_coef=0.1))
    e = R.policy(c.z, c.x, torch.nan_to_num(adv), weight=c.w, old=torch.nan_to_num(old), zref=c.z, kl_coef=0.1, ent=0.1)
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    R.near(o.dlogits, e["g"], e["g_tol"], "dlogits")
    assert not o.status.any() and not o.dlogits.cpu()[off].float().any() and not o.logprob.cpu()[off].any()
    c = Case(2, 3, 100, F)
    o = am.policy_loss(c.z.cuda() * math.nan, c.x.cuda(), c.n(2, 3).cuda(), c.ws(am), weight=torch.zeros(2, 3, device="cuda"))
    assert o.loss.item() == 0 and not o.dlogits.any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_masked_vocabulary(am, dtype):
    """Tokens masked with -inf or with the type's lowest value, in the reference too; one token left; the reference masks more."""
    c = Case(4, 6, 3001, dtype, seed=9, masked=0.0)
    for value in (-math.inf, torch.finfo(dtype).min):
        z = c.z.clone()
        z[:2, :, 1::3] = value
        z[2, 0] = value
        z[2, 0, int(c.x[2, 0])] = 1.5                         # one token left: probability 1
        x = c.x.long()
        z.scatter_(-1, x[..., None], torch.where(torch.isfinite(c.z.gather(-1, x[..., None])), c.z.gather(-1, x[..., None]), 0))
        zref = (z.float() + 0.5 * c.n(*z.shape).clamp(-1, 1)).clamp_min(-math.inf if value == -math.inf else value).to(dtype)
        o, e = _policy(am, c, "full", 0.05, z=z, zref=zref)
        assert not o.status.any() and not torch.isnan(o.dlogits).any()
        R.near(o.entropy[2, 0], torch.tensor(0.0), 1e-6)
        assert not o.dlogits[:2, :, 1::3].cpu()[(x[:2] % 3 != 1)].any()
    zref = c.z.clone()
    zref[0, 0, :] = -math.inf
    zref[0, 0, 5] = 0.0                                       # the reference allows one token only: the KL is infinite
    o = am.policy_loss(c.z.cuda(), c.x.cuda(), c.n(4, 6).cuda(), c.ws(am), ref_logits=zref.cuda(), options=am.PolicyOptions(kl_coef=0.1))
    assert o.kl[0, 0].item() == math.inf and o.token_loss[0, 0].item() == math.inf and torch.isnan(o.dlogits[0, 0]).any()
    assert torch.isfinite(o.kl.cpu().view(-1)[1:]).all() and torch.isfinite(o.dlogits.cpu().view(24, -1)[1:]).all()
    # a sampled token that is masked: no probability left, the ratio is 0
    z = c.z.clone()
    z[0, 0, int(c.x[0, 0])] = -math.inf
    o, e = _policy(am, c, z=z)
    assert o.logprob[0, 0].item() == -math.inf and torch.isfinite(o.dlogits).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_broken_rows_and_tokens(am, dtype):
    c = Case(2, 6, 777, dtype, masked=0.0)
    z, x = c.z.clone(), c.x.clone()
    z[0, 0, 700] = math.nan
    z[0, 1, 3] = math.inf
    z[0, 2] = -math.inf
    x[1, 0], x[1, 1] = 777, -1
    ws = c.ws(am)
    lp, H, st = am.token_logprob(z.cuda(), x.cuda(), ws)
    assert st.cpu().view(-1).tolist() == [2, 2, 2, 0, 0, 0, 1, 1, 0, 0, 0, 0]
    assert torch.isnan(lp.cpu().view(-1)).tolist() == [True] * 3 + [False] * 3 + [True] * 2 + [False] * 4
    assert torch.isnan(H.cpu().view(-1)).tolist() == [True] * 3 + [False] * 9
    o = am.policy_loss(z.cuda(), x.cuda(), torch.ones(2, 6, device="cuda"), ws)
    bad = torch.isnan(lp.cpu())
    assert math.isnan(o.loss.item()) and torch.equal(torch.isnan(o.token_loss.cpu()), bad) and torch.equal(o.status, st)
    assert torch.isnan(o.dlogits.cpu()[bad]).all() and torch.isfinite(o.dlogits.cpu()[~bad]).all()
    w = (~bad).float().cuda()
    o = am.policy_loss(z.cuda(), x.cuda(), torch.ones(2, 6, device="cuda"), ws, weight=w)
    assert math.isfinite(o.loss.item()) and torch.isfinite(o.dlogits).all() and not o.status.any()
    o = am.preference_loss(z.cuda(), x.cuda(), ws)
    assert math.isnan(o.loss.item()) and torch.isnan(o.dlogits).all()             # the one pair there is
    o = am.preference_loss(z.cuda(), x.cuda(), ws, weight=w)
    assert math.isfinite(o.loss.item()) and torch.isfinite(o.dlogits).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_large_offsets(am, dtype):
    """Rows that carry large and different offsets (softmax does not see them; the type's rounding of the shifted logits does)."""
    c = Case(2, 4, 4001, dtype, seed=11, masked=0.0)
    z, zref = (c.z.float() + 300.0).to(dtype), (c.z.float() - 500.0).to(dtype)
    c.lp = R.rows(z, c.x)["lp"]
    _policy(am, c, "full", 0.1, z=z, zref=zref)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("layout", ["view", "transposed", "padded", "offset", "in_place", "gap"])
def test_layouts(am, layout, dtype):
    """Next-token views, [T, B, V] arrays, padded rows, rows off any alignment, gradients in the logits' place; memory beside the rows
    stays as it was."""
    B, T, V = 4, 5, 1037
    c = Case(B, T, V, dtype, seed=12)
    if layout == "view":
        buf = torch.full((B, T + 1, V), 7.0, dtype=dtype, device="cuda")
        z, g = buf[:, :T], torch.full_like(buf, 7.0)[:, :T]
    elif layout == "transposed":
        z, g = (torch.full((T, B, V), 7.0, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(2))
    elif layout in ("padded", "in_place"):
        z, g = (torch.full((B, T, V + 3), 7.0, dtype=dtype, device="cuda")[..., :V] for _ in range(2))
    elif layout == "offset":
        z, g = (torch.full((B * T * V + 8,), 7.0, dtype=dtype, device="cuda")[k:k + B * T * V].view(B, T, V) for k in (1, 3))
    else:
        z, g = (torch.full((B, T, 2, V), 7.0, dtype=dtype, device="cuda")[:, :, 0] for _ in range(2))
    z.copy_(c.z)
    g = z if layout == "in_place" else g
    adv, old = c.n(B, T), c.old()
    zref = (c.z.float() + 0.5 * c.n(B, T, V)).to(dtype)
    rbuf = torch.zeros(B * T * V + 1, dtype=dtype, device="cuda")
    rbuf[1:] = zref.cuda().view(-1)
    o = am.policy_loss(z, c.x.cuda(), adv.cuda(), c.ws(am), weight=c.w.cuda(), old_logprob=old.cuda(), ref_logits=rbuf[1:].view(B, T, V),
                       options=am.PolicyOptions(kl_coef=0.1, entropy_coef=0.01), dlogits=g)
    e = R.policy(c.z, c.x, adv, weight=c.w, old=old, zref=zref, kl_coef=0.1, ent=0.01)
    assert o.dlogits is g
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    R.near(g, e["g"], e["g_tol"], "dlogits")
    total = g._base if g._base is not None else g
    inside = torch.zeros_like(total, dtype=torch.bool)
    inside.as_strided(g.shape, g.stride(), g.storage_offset()).fill_(True)
    assert (total[~inside] == 7.0).all()
    if layout != "in_place":
        assert torch.equal(z.cpu(), c.z)
    # the preference loss reads the rows twice
    z.copy_(c.z)
    e = R.preference(c.z, c.x, weight=c.w)
    o = am.preference_loss(z, c.x.cuda(), c.ws(am), weight=c.w.cuda(), dlogits=g)
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    R.near(g, e["g"], e["g_tol"], "dlogits")
    assert (total[~inside] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_rows(am, dtype):
    """As many rows as there are workgroups on the chip and more, of several lengths of the vocabulary."""
    for B, T, V in ((9, 100, 520), (4, 600, 1111), (3, 700, 4097)):
        c = Case(B, T, V, dtype, seed=13)
        _policy(am, c, "full", 0.01)
        _policy(am, c, "sampled")
        c = Case(B + B % 2, T, V, dtype, seed=14)
        _preference(am, c)


def test_rows_behind_the_four_gigabyte(am):
    """Offsets that pass 32 bits, in elements too."""
    V, T = 128256, 1
    B = (1 << 31) // V + 9
    z = torch.empty(B, T, V, dtype=BF, device="cuda")
    z.normal_(generator=torch.Generator("cuda").manual_seed(3))
    x = torch.randint(0, V, (B, T), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(4))
    adv = torch.linspace(-1, 1, B, device="cuda")
    ws = am.LossWorkspace(B, T, V, BF)
    o = am.policy_loss(z, x, adv, ws, options=am.PolicyOptions(entropy_coef=0.1))
    rows = [0, 1, B // 2, B - 9, B - 2, B - 1]
    e = R.policy(z[rows].cpu(), x[rows].cpu(), adv[rows].cpu(), ent=0.1)
    R.near(o.token_loss[rows], e["term"], e["term_tol"], "token_loss")
    R.near(o.dlogits[rows], e["g"], e["g_tol"], "dlogits")
    before = z[rows].cpu()
    g = am.token_logprob_grad(z, x, ws, adv[:, None].contiguous(), dlogits=z)       # in place
    assert g is z
    R.near(g[rows], *R.grad(R.rows(before, x[rows].cpu()), adv[rows][:, None].cpu(), dtype=BF), "dlogits in place")


def test_same_bits_again_and_smaller_shapes_on_one_workspace(am):
    big, small = Case(8, 16, 5003, BF, seed=15), Case(3, 2, 301, BF, seed=16)
    ws = big.ws(am)

    def call(c):
        adv = torch.ones(c.B, c.T, device="cuda")
        o = am.policy_loss(c.z.cuda(), c.x.cuda(), adv, ws, weight=c.w.cuda(), ref_logits=c.z.cuda().roll(1, 0),
                           options=am.PolicyOptions(kl_coef=0.1, entropy_coef=0.01))
        return [o.loss, o.token_loss, o.kl, o.entropy, o.dlogits]
    first, other = call(big), call(small)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, call(big)))
        assert all(torch.equal(a, b) for a, b in zip(other, call(small)))


def test_empty_batches(am):
    ws = am.LossWorkspace(2, 2, 50, F)
    e = lambda *s, dt=F: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    o = am.policy_loss(e(0, 3, 50), e(0, 3, dt=torch.int32), e(0, 3), ws)
    assert o.loss.item() == 0.0 and o.dlogits.shape == (0, 3, 50)
    o = am.policy_loss(e(2, 0, 50), e(2, 0, dt=torch.int32), e(2, 0), ws)
    assert o.loss.item() == 0.0
    o = am.preference_loss(e(0, 3, 50), e(0, 3, dt=torch.int32), ws)
    assert o.loss.item() == 0.0 and o.score.shape == (0,)
    lp, H, st = am.token_logprob(e(0, 50), e(0, dt=torch.int32), ws)
    assert lp.shape == (0,)


def test_refusals_of_the_binding(am):
    c = Case(2, 3, 50, F)
    z, x, ws = c.z.cuda(), c.x.cuda(), c.ws(am)
    adv = torch.ones(2, 3, device="cuda")
    for bad in (lambda: am.token_logprob(z, x[:, :2].contiguous(), ws), lambda: am.token_logprob(z, x.long(), ws),
                lambda: am.token_logprob(z, x.cpu(), ws), lambda: am.token_logprob(z.transpose(1, 2), x, ws),
                lambda: am.token_logprob(z, x, ws, active=torch.ones(2, 3, device="cuda")),
                lambda: am.token_logprob_grad(z, x, ws, adv[:, :2].contiguous()),
                lambda: am.token_logprob_grad(z, x, ws, adv, dlogits=z.bfloat16()),
                lambda: am.policy_loss(z, x, adv[0], ws), lambda: am.policy_loss(z, x, adv, ws, weight=adv.double()),
                lambda: am.policy_loss(z, x, adv, ws, ref_logits=z.bfloat16()),
                lambda: am.policy_loss(z, x, adv, ws, grad_scale=torch.ones(2, device="cuda")),
                lambda: am.preference_loss(z, x, ws, pair_weight=torch.ones(2, device="cuda")),
                lambda: am.preference_loss(z, x, ws, options=am.PreferenceOptions(kind="other"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        am.token_logprob(z.half(), x, ws)
    for bad, code in ((lambda: am.policy_loss(z, x, adv, ws, ref_logits=z, ref_logprob=adv), -1),
                      (lambda: am.policy_loss(z, x, adv, ws, options=am.PolicyOptions(clip_low=2.0)), -1),
                      (lambda: am.policy_loss(z, x, adv, ws, ref_logits=z, dlogits=z), -1),
                      (lambda: am.token_logprob_grad(z[:, :2], x[:, :2].contiguous(), ws, adv[:, :2].contiguous(), dlogits=z[:, 1:]), -1),
                      (lambda: am.token_logprob(z[:1].expand(2, 3, 50), x, ws), -1),
                      (lambda: am.preference_loss(z[:1], x[:1], ws), -1),
                      (lambda: am.token_logprob(torch.zeros(40, 30, 50, device="cuda"), torch.zeros(40, 30, device="cuda", dtype=torch.int32), ws), -4)):
        with pytest.raises(am.AdasdError) as e:
            bad()
        assert e.value.code == code


def test_another_stream_and_captured_calls(am):
    """A captured step replayed with new inputs in its buffers, between eager calls on the same workspace, against the eager results."""
    c = Case(4, 33, 5003, BF, seed=17)
    z, x, ws = c.z.cuda(), c.x.cuda(), c.ws(am)
    adv, old, w = c.n(4, 33).cuda(), c.old().cuda(), c.w.cuda()
    opt = am.PolicyOptions(kl_coef=0.1, entropy_coef=0.01)
    zref = (c.z.float() + 0.3 * c.n(4, 33, 5003)).to(BF).cuda()

    def step():
        lp, H, _ = am.token_logprob(z, x, ws)
        o = am.policy_loss(z, x, adv, ws, weight=w, old_logprob=old, ref_logits=zref, options=opt)
        p = am.preference_loss(z, x, ws, weight=w)
        return [lp, H, o.loss, o.token_loss, o.kl, o.dlogits, p.loss, p.score, p.dlogits]
    eager = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, there))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    keep = z.clone()
    for k in range(4):
        z.copy_(keep.roll(k, 0))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in captured:
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, captured)), k


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_training_step_on_verified_tokens(am, dtype):
    """What the calls are for, together: a round is verified; the log-probabilities of its tokens under the target are kept; then the
    draft's output layer is trained on them with the policy loss (KL against the target's logits), and with the preference loss, the
    gradients handed to torch.  The weights' gradients against differentiation in 64 bits."""
    B, K, V, D = 4, 6, 2003, 32
    g = torch.Generator().manual_seed(21)
    h, W = torch.randn(B, K, D, generator=g), (0.4 * torch.randn(V, D, generator=g))
    target = (torch.randn(B, K + 1, V, generator=g) * 2).to(dtype).cuda()
    h, W = h.cuda(), W.cuda().requires_grad_(True)
    z = (h @ W.t()).to(dtype)
    ws, state = am.Workspace(B, K, V, dtype), am.State(B, 64)
    x = torch.stack([am.draft_step(z[:, i].detach(), ws, step=i, k_max=20, seed=5)[2] for i in range(K)], 1).contiguous()
    out = am.verify(target, z.detach(), x, ws, state=state, seed=5, options=am.Options(apply_update=1))
    accepted = (torch.arange(K, device="cuda")[None] < out.n_accept[:, None]).float()
    weight = (torch.arange(K, device="cuda")[None] <= out.n_accept[:, None]).float() / (B * K)
    lws = am.LossWorkspace(B, K, V, dtype)
    zp = target[:, :K]
    ref, H, status = am.token_logprob(zp, x, lws)
    assert not status.any()
    R.near(H, out.H_p.double(), 1e-5 * out.H_p.abs().cpu().double() + 1e-6 + R.tol_H(R.rows(zp.cpu(), x.cpu())), "entropy of the target")
    adv = 2.0 * accepted - 1.0
    o = am.policy_loss(z, x, adv, lws, weight=weight, ref_logits=zp, options=am.PolicyOptions(kl_coef=0.5, entropy_coef=0.01))
    z.backward(o.dlogits)
    got = W.grad.clone()
    Wd = W.detach().double().requires_grad_(True)
    zd = h.double() @ Wd.t()
    zd = zd + (z.detach().double() - zd.detach())             # the logits as they were rounded
    l, lq = torch.log_softmax(zd, -1), torch.log_softmax(zp.double(), -1)
    lp = l.gather(-1, x.long()[..., None])[..., 0]
    term = -adv.double() * torch.exp(lp - lp.detach()) + 0.5 * (l.exp() * (l - lq)).sum(-1) + 0.01 * (l.exp() * l).sum(-1)
    loss = (weight.double() * term).sum()
    loss.backward()
    # each gradient element is within half a step of the type (and the arithmetic's 1e-5): so is the sum, in the norm, of products
    # with the same hidden states; 2x for the product that torch forms in the logits' type or in float
    bound = 2 * R.HALF[dtype] + 2e-5
    assert abs(loss.item() - o.loss.item()) < 2e-5 * (1 + abs(loss.item()))
    assert (got.double() - Wd.grad).norm() < bound * Wd.grad.norm()
    W.grad = None
    z = (h @ W.t()).to(dtype)
    p = am.preference_loss(z, x, lws, weight=(weight > 0).float(), ref_logprob=ref)
    z.backward(p.dlogits)
    Wd.grad = None
    zd = h.double() @ Wd.t()
    zd = zd + (z.detach().double() - zd.detach())
    lp = torch.log_softmax(zd, -1).gather(-1, x.long()[..., None])[..., 0]
    s = ((weight > 0).double() * (lp - ref.double())).sum(1)
    loss = -torch.nn.functional.logsigmoid(0.1 * (s[:2] - s[2:])).mean()
    loss.backward()
    assert abs(loss.item() - p.loss.item()) < 2e-5
    assert (W.grad.double() - Wd.grad).norm() < bound * Wd.grad.norm()


@pytest.mark.parametrize("dtype", [BF, F])
def test_rows_of_every_cut(am, dtype):
    """One to four wavefronts per row, a workgroup per row, slices; with as many rows as make the cuts differ."""
    for B, T, V in ((43, 31, 40), (29, 45, 2003), (27, 48, 4009), (53, 25, 6007), (21, 63, 9001)):     # above 1280 rows
        c = Case(B, T, V, dtype, seed=18)
        _policy(am, c, "full", 0.01)
        _policy(am, c, "none", 0.01)
    c = Case(2, 667, 2003, dtype, seed=19)
    _preference(am, c)
    act = (c.w != 0).to(torch.uint8)
    lp, H, st = am.token_logprob(c.z.cuda(), c.x.cuda(), c.ws(am), active=act.cuda())
    o = R.rows(c.z, c.x)
    R.near(lp, torch.where(act.bool(), o["lp"], 0.0), R.tol_lp(o), "logprob")
    R.near(H, torch.where(act.bool(), o["H"], 0.0), R.tol_H(o), "entropy")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [300001, 1100003])
def test_long_vocabularies(am, V, dtype):
    """Rows of more slices than there are records in a wavefront's lanes, and nearly so."""
    c = Case(1, 3, V, dtype, seed=20, masked=0.0)
    _policy(am, c, "full", 0.01)
    _policy(am, c, "sampled")
    c = Case(2, 2, V, dtype, seed=21)
    _preference(am, c)


def test_many_positions(am):
    """More positions than the last one adds up by itself; pairs as many and as long."""
    c = Case(70, 71, 33, BF, seed=22)
    _policy(am, c, "sampled", 0.01)
    _preference(am, c)
    c = Case(2, 2600, 33, F, seed=23)
    _policy(am, c)
    _preference(am, c)
    c = Case(5200, 1, 33, F, seed=24)
    _preference(am, c)


@pytest.mark.parametrize("how", ["unarrived", "given_up"])
@pytest.mark.parametrize("dtype", [BF, F])
def test_slices_whose_records_are_not_waited_for(am, how, dtype):
    """The same results (to the last bits) where no slice waits for the others' sums, or all count as not there; and the next call finds
    the workspace as it should be."""
    import ctypes
    from test_losses import _Rows
    lib = am.load_library()
    for B, T, V in ((1, 1, 128256), (3, 5, 32003), (2, 40, 70001), (1, 700, 20011)):
        c = Case(B, T, V, dtype, seed=25)
        z, x, ws = c.z.cuda(), c.x.cuda(), c.ws(am)
        o = R.rows(c.z, c.x)
        a, h = c.n(B, T), c.n(B, T)
        for again in range(2):
            lp, H = (torch.full((B, T), 9.0, device="cuda") for _ in range(2))
            st = torch.full((B, T), 9, dtype=torch.int32, device="cuda")
            g = torch.full_like(z, 9.0)
            rows = _Rows(z.data_ptr(), int(dtype == BF), B, T, V, z.stride(0), z.stride(1), x.data_ptr())
            rows.logprob, rows.entropy, rows.status = lp.data_ptr(), H.data_ptr(), st.data_ptr()
            rows.workspace, rows.ws_bytes = ws.ptr, ws.bytes
            s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
            assert getattr(lib, f"adasd_test_logprob_{how}")(ctypes.byref(rows), s) == 0
            R.near(lp, o["lp"], R.tol_lp(o), "logprob")
            R.near(H, o["H"], R.tol_H(o), "entropy")
            assert not st.any()
            # (records that count as not there are formed from the logits again, which have to be whole then: not in place)
            for out in (g,) if how == "unarrived" else (g, z.clone()):
                if out is not g:
                    z2 = out
                    rows.logits = z2.data_ptr()
                rows.dlogits, rows.d_seq_stride, rows.d_pos_stride = out.data_ptr(), out.stride(0), out.stride(1)
                da, dh = a.cuda(), h.cuda()
                f = getattr(lib, f"adasd_test_logprob_grad_{how}")
                assert f(ctypes.byref(rows), ctypes.c_void_p(da.data_ptr()), ctypes.c_void_p(dh.data_ptr()), s) == 0
                torch.cuda.synchronize()
                R.near(out, *R.grad(o, a, h, dtype=dtype), "dlogits")
            rows.logits = z.data_ptr()
            assert torch.equal(am.token_logprob_grad(z, x, ws, a.cuda(), h.cuda()), am.token_logprob_grad(z, x, c.ws(am), a.cuda(), h.cuda()))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("layout", ["view", "in_place", "offset"])
def test_layouts_of_many_rows(am, layout, dtype):
    B, T, V = 31, 43, 1037
    c = Case(B, T, V, dtype, seed=26)
    if layout == "view":
        z, g = (torch.full((B, T + 1, V), 7.0, dtype=dtype, device="cuda")[:, :T] for _ in range(2))
    elif layout == "in_place":
        z = torch.full((T, B, V + 3), 7.0, dtype=dtype, device="cuda")[..., :V].transpose(0, 1)
        g = z
    else:
        z, g = (torch.full((B * T * V + 8,), 7.0, dtype=dtype, device="cuda")[k:k + B * T * V].view(B, T, V) for k in (1, 3))
    z.copy_(c.z)
    adv, old = c.n(B, T), c.old()
    o = am.policy_loss(z, c.x.cuda(), adv.cuda(), c.ws(am), weight=c.w.cuda(), old_logprob=old.cuda(), options=am.PolicyOptions(entropy_coef=0.01), dlogits=g)
    e = R.policy(c.z, c.x, adv, weight=c.w, old=old, ent=0.01)
    R.near(o.loss, e["loss"], e["loss_tol"], "loss")
    R.near(g, e["g"], e["g_tol"], "dlogits")
    total = g._base if g._base is not None else g
    inside = torch.zeros_like(total, dtype=torch.bool)
    inside.as_strided(g.shape, g.stride(), g.storage_offset()).fill_(True)
    assert (total[~inside] == 7.0).all()


def test_forms_without_gradient_or_coefficient(am):
    """No gradient wanted, or a reference whose KL is only reported, in every cut of the rows."""
    for B, T, V in ((2, 3, 40), (3, 5, 9001), (31, 43, 1037), (27, 48, 4009), (2, 600, 20011)):
        c = Case(B, T, V, BF, seed=27)
        _policy(am, c, "full", 0.1, need_grad=False)
        _policy(am, c, "full", 0.1, kl_coef=0.0)
        _policy(am, c, "none", need_grad=False)
        c = Case(B + B % 2, T, V, BF, seed=28)
        _preference(am, c, need_grad=False)


def test_workspace_of_a_shorter_vocabulary(am):
    """A workspace with less room for the slices' words than these rows take: the same results by another way."""
    c = Case(3, 400, 40009, BF, seed=29)
    small = am.LossWorkspace(3, 400, 50, BF)
    _policy(am, c, "full", 0.01, ws=small)
    c = Case(4, 300, 40009, BF, seed=30)
    _preference(am, c, ws=small)


def test_two_calls_at_once(am):
    """Two streams, each with its workspace and slices that wait for one another, over and over; each call against its result alone."""
    def make(shape, seed):
        c = Case(*shape, BF, seed=seed)
        d = dict(z=c.z.cuda(), x=c.x.cuda(), adv=c.n(c.B, c.T).cuda(), w=c.w.cuda(), ws=c.ws(am), zref=c.z.cuda().roll(1, 0))
        return d

    def call(d):
        o = am.policy_loss(d["z"], d["x"], d["adv"], d["ws"], weight=d["w"], ref_logits=d["zref"], options=am.PolicyOptions(kl_coef=0.1))
        p = am.preference_loss(d["z"], d["x"], d["ws"], weight=d["w"])
        return [o.loss, o.kl, o.dlogits, p.loss, p.dlogits]
    jobs = [make((2, 20, 70001), 31), make((4, 9, 128256), 32)]
    want = [[t.clone() for t in call(d)] for d in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(20):
        for k, (s, d) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[k].append(call(d))
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(want[k], r))


def test_two_graphs_on_one_workspace(am):
    c, e = Case(2, 10, 70001, BF, seed=33), Case(3, 200, 2003, F, seed=34)
    ws = am.LossWorkspace(3, 200, 70001, F)

    def step(c):
        z, x, adv, w = c.z.cuda(), c.x.cuda(), torch.ones(c.B, c.T, device="cuda"), c.w.cuda()
        torch.cuda.synchronize()

        def run():
            o = am.policy_loss(z, x, adv, ws, weight=w, options=am.PolicyOptions(entropy_coef=0.01))
            lp, H, _ = am.token_logprob(z, x, ws)
            return [o.loss, o.token_loss, o.dlogits, lp, H]
        want = [t.clone() for t in run()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        return graph, out, want, run           # (run keeps the inputs that the graph reads)
    steps = [step(c), step(e)]
    for k in range(6):
        graph, out, want, _ = steps[k % 2]
        for t in out:
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [100, 4003, 70001])
def test_gradients_that_are_no_numbers(am, V, dtype):
    """A derivative that is no number makes every element of its row one, tokens without mass among them, and no element of another row."""
    c = Case(2, 3, V, dtype, seed=41, masked=0.0)
    z = c.z.clone()
    z[..., ::3] = -math.inf
    x = torch.full((2, 3), 1, dtype=torch.int32)
    ws, one = c.ws(am), torch.ones(2, 3, device="cuda")

    def rows_of_nan(g, *rows):
        nan = torch.isnan(g.cpu().view(6, V))
        assert [bool(r.all()) for r in nan] == [i in rows for i in range(6)] and [bool(r.any()) for r in nan] == [i in rows for i in range(6)]

    nan = one.clone()
    nan[0, 1] = math.nan
    for a, h in ((nan, None), (one, nan), (nan, nan)):
        rows_of_nan(am.token_logprob_grad(z.cuda(), x.cuda(), ws, a, h), 1)
    inf = one.clone()
    inf[1, 2] = math.inf
    rows_of_nan(am.policy_loss(z.cuda(), x.cuda(), nan, ws, options=am.PolicyOptions(entropy_coef=0.1)).dlogits, 1)
    rows_of_nan(am.policy_loss(z.cuda(), x.cuda(), one, ws, weight=inf, options=am.PolicyOptions(entropy_coef=0.1)).dlogits, 5)
    zref = z.clone()
    zref[0, 2, 2] = -math.inf                                  # the reference has no mass where the row has
    for ent in (0.0, 0.1):
        o = am.policy_loss(z.cuda(), x.cuda(), one, ws, ref_logits=zref.cuda(), options=am.PolicyOptions(kl_coef=0.1, entropy_coef=ent))
        assert o.kl[0, 2].item() == math.inf
        rows_of_nan(o.dlogits, 2)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V", [100, 4003, 70001])
def test_mass_that_is_lost_in_the_type(am, V, dtype):
    """A probability below 2^-149 of the row's largest counts as 0, whatever the reference has there."""
    c = Case(1, 4, V, dtype, seed=42, masked=0.0)
    x = torch.full((1, 4), 1, dtype=torch.int32)
    z, zref = c.z.clone(), (c.z.float() + 0.25 * c.n(*c.z.shape)).to(dtype)
    z[..., 3::7] = -400.0
    zref[:, 0::2, 3::7] = -math.inf
    bare = z.clone()                                           # the same rows without those tokens
    bare[..., 3::7] = -math.inf
    opt = am.PolicyOptions(kl_coef=0.1, entropy_coef=0.1)
    ws, one = c.ws(am), torch.ones(1, 4, device="cuda")
    got, want = (am.policy_loss(a.cuda(), x.cuda(), one, ws, ref_logits=b.cuda(), options=opt) for a, b in ((z, zref), (bare, zref)))
    assert torch.isfinite(got.kl).all() and not got.dlogits[..., 3::7].any() and not got.status.any()
    for name in ("loss", "token_loss", "logprob", "entropy", "kl", "dlogits"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name


@pytest.mark.parametrize("dtype", [BF, F])
def test_the_largest_logits(am, dtype):
    """Rows whose largest logit is up to 2^26 in size are right; beyond that they are flagged, whatever the rounding of their sums."""
    B, T, V = 1, 16, 5000
    g = torch.Generator().manual_seed(43)
    noise, up = torch.randn(B, T, V, generator=g), 1.0 + 0.05 * torch.rand(B, T, generator=g)
    x = torch.full((B, T), 7, dtype=torch.int32)
    ws = am.LossWorkspace(B, T, V, dtype)
    for size in (6.2e7, -6.2e7, 1e8, 1e9, -1e9, 1e30, -1e30):
        z = noise.clone() if size > 0 else noise + size
        if size > 0:
            z[..., 7] = size * up
        z = z.to(dtype)
        lp, _, st = am.token_logprob(z.cuda(), x.cuda(), ws)
        if abs(size) < 2.0**26:
            # (equal logits, or one that takes all the mass: sums of up to 5000 equal terms, 13 roundings of half a unit)
            R.near(lp, torch.log_softmax(z.double(), -1)[..., 7], 13 * 2.0**-24 + 2.0**-24 * 9.0)
            assert not st.any()
        else:
            assert (st == 2).all() and torch.isnan(lp).all()
