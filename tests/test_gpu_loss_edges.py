"""Losses over vocabulary rows at the edges of their inputs: infinite terms, masks of any finite value, rows that do not count beside broken
ones, records that are not waited for.  Expected values are stated, or those of the 64-bit forms in loss_ref.py."""
import math

import pytest
import torch

import loss_ref as R
from test_gpu_losses import BF, F, Case, am, cu  # noqa: F401

pytestmark = pytest.mark.gpu

INF = math.inf

# positions: a workgroup's own rows, a row in slices, more than one launch adds up beside a gradient, more than any launch adds up
COUNTS = [(2, 3, 40), (2, 3, 32003), (4, 100, 9001), (20, 300, 40)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("shape", COUNTS)
def test_an_infinite_term_makes_the_loss_infinite(am, shape, dtype):  # noqa: F811
    """A KL of +inf (the reference has no mass where the row has) in the policy loss, however the terms are added up."""
    c = Case(*shape, dtype, seed=51, masked=0.0)
    zref = c.z.clone()
    zref[0, 1, 5] = -INF
    one = torch.ones(c.B, c.T, device="cuda")
    ws, opt = c.ws(am), am.PolicyOptions(kl_coef=0.1)
    for need_grad in (True, False):
        for sign in (1.0, -1.0):
            o = am.policy_loss(c.z.cuda(), c.x.cuda(), one, ws, weight=sign * one, ref_logits=zref.cuda(), options=opt, need_grad=need_grad)
            assert o.token_loss[0, 1].item() == INF and o.loss.item() == sign * INF
    w = one.clone()
    w[0, 1] = -1.0
    zref[1, 2, 5] = -INF
    o = am.policy_loss(c.z.cuda(), c.x.cuda(), one, ws, weight=w, ref_logits=zref.cuda(), options=opt)
    assert math.isnan(o.loss.item())                                               # inf - inf


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("side", ["chosen", "rejected"])
@pytest.mark.parametrize("shape", [(2, 3, 40), (4, 5, 32003), (4, 1030, 40), (4, 1030, 1037)])
def test_a_token_without_mass_in_a_pair(am, shape, side, dtype):  # noqa: F811
    """Log-probability -inf in the second pair: scores, losses and slopes as the formulas have them, below and above 4096 positions."""
    c = Case(*shape, dtype, seed=52, masked=0.0)
    B, T, V = shape
    P = B // 2
    b, t = (P - 1 if side == "chosen" else B - 1), T // 2
    z = c.z.clone()
    x = int(c.x[b, t])
    z[b, t, x] = -INF
    o = R.rows(z, c.x)
    beta, ws = 0.125, c.ws(am)
    for kind, e in (("logistic", 0.0), ("logistic", 0.25), ("hinge", 0.0), ("squared", 0.0)):
        r = am.preference_loss(z.cuda(), c.x.cuda(), ws, options=am.PreferenceOptions(kind=kind, beta=beta, label_smoothing=e))
        m = -INF if side == "chosen" else INF
        if kind == "squared":
            loss, slope = INF, 2.0 * m
        elif kind == "hinge":
            loss, slope = (INF, -beta) if side == "chosen" else (0.0, 0.0)
        else:
            loss = (INF if side == "chosen" or e > 0 else 0.0)
            slope = -beta * (1.0 - e) if side == "chosen" else beta * e
        assert r.logprob[b, t].item() == -INF and r.score[b].item() == -INF and torch.isfinite(r.score).sum().item() == B - 1
        assert r.margin[P - 1].item() == m and r.pair_loss[P - 1].item() == loss, (kind, r.margin, r.pair_loss)
        others = r.pair_loss.cpu()[:P - 1]
        assert torch.isfinite(others).all()
        assert r.loss.item() == INF if loss == INF else abs(r.loss.item() - others.double().sum().item() / P) <= 4 * R.H24 * others.double().sum().item()
        both = [P - 1, B - 1]
        if math.isinf(slope):
            assert not torch.isfinite(r.dlogits[b, t, x]).item()
            continue
        a = torch.zeros(B, T, dtype=torch.float64)
        a[P - 1], a[B - 1] = slope / P, -slope / P
        g, tol = R.grad({k: v[both] if torch.is_tensor(v) else v for k, v in o.items()}, a[both], dtype=dtype)
        R.near(r.dlogits[both], g, tol, f"dlogits {kind}")
        if slope == 0.0:
            assert not r.dlogits[both].any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind", ["logistic", "squared"])
def test_rows_that_do_not_count_in_a_broken_pair(am, kind, dtype):  # noqa: F811
    """Zeros, although the pair's slope is no number (a NaN row), or infinite (the squared loss of a token without mass)."""
    for B, T, V in ((2, 6, 40), (4, 5, 32003), (4, 1100, 40)):
        c = Case(B, T, V, dtype, seed=53, masked=0.5)
        w = (c.w != 0).float()
        w[0, 0], w[0, 1], w[B // 2, 2] = 1.0, 0.0, 0.0
        for broken in (math.nan, -INF):
            z = c.z.clone()
            z[0, 0, int(c.x[0, 0])] = broken
            z[w == 0] = math.nan
            o = am.preference_loss(z.cuda(), c.x.cuda(), c.ws(am), weight=w.cuda(), options=am.PreferenceOptions(kind=kind))
            assert not o.dlogits.cpu()[w == 0].any(), (B, T, V, broken)
            if math.isnan(broken):
                assert torch.isnan(o.dlogits.cpu()[0, 0]).all()


# Finite values that serve as masks, all far below the ordinary logits' 149 binary orders: the tokens have no mass, as with -inf.
MASKS = {BF: [-1e4, -1e9, -1.5e9, -1e10, -3e12, -1e30, -2.5e36, -5e36, -9e36, -2e37, -1e38, -2e38, torch.finfo(BF).min],
         F: [-1e4, -1e9, -1.5e9, -1e10, -3e12, -1e30, -5e36, -1e37, -1e38, -2e38, torch.finfo(F).min / 2, torch.finfo(F).min]}


@pytest.mark.parametrize("dtype, mask", [(d, m) for d in (BF, F) for m in MASKS[d]])
def test_masks_of_any_size(am, mask, dtype):  # noqa: F811
    """Whole stretches of the vocabulary masked with one value, longer than any lane's, wavefront's or slice's part, and single tokens: bit for bit
    what -inf gives, in every cut of the rows, in the forward pass and in the gradients, with a reference masked alike and without."""
    one = None
    for B, T, V in ((1, 1, 128256), (3, 5, 9001), (2, 2, 40), (31, 43, 1037), (2, 600, 20011)):
        c = Case(B, T, V, dtype, seed=54, masked=0.0)
        zref = (c.z.float() + 0.5 * c.n(B, T, V)).to(dtype)
        x = c.x.clone()

        def masked(value):
            z, q = c.z.clone(), zref.clone()
            for v in (z, q):
                keep = v.gather(-1, x.long()[..., None]).clone()
                v[..., V // 5:V // 5 + V // 2] = value
                v[..., 1::7] = value
                v.scatter_(-1, x.long()[..., None], keep)
            return z.cuda(), q.cuda()
        one = torch.ones(B, T, device="cuda")
        ws = c.ws(am)

        def call(value):
            z, q = masked(value)
            lp, H, st = am.token_logprob(z, x.cuda(), ws)
            g = am.token_logprob_grad(z, x.cuda(), ws, one, one)
            o = am.policy_loss(z, x.cuda(), one, ws, ref_logits=q, options=am.PolicyOptions(kl_coef=0.1, entropy_coef=0.1))
            r = [lp, H, st, g, o.loss, o.token_loss, o.kl, o.dlogits, o.status]
            if B % 2 == 0:
                p = am.preference_loss(z, x.cuda(), ws)
                r += [p.loss, p.score, p.dlogits]
            return r
        want, got = call(-INF), call(mask)
        assert not got[2].any() and not got[8].any(), (B, T, V)
        for k, (a, b) in enumerate(zip(got, want)):
            assert torch.isfinite(a).all() and torch.equal(a, b), (B, T, V, k)


def _kl_spread(z, zr, o):
    """What the terms of the KL cancel from, no token's difference by itself.  A term is t - tr, each logit about the largest of its own row (or part of
    it): |t| = |ln p + ln s|, |tr| = |ln q + ln sr| <= |D| + |ln p| + |ln sr|.  Weighted by p and rounded a few times each (tol_kl and grad allow
    more than 30 steps of it): KL-like sums, H, and the logarithms of the two rows' sums about their largest."""
    s, sr = (torch.logsumexp(v.double(), -1) - v.double().amax(-1) for v in (z, zr))
    return 2 * (o["p"] * o["D"].abs()).sum(-1) + o["H"] + s.abs() + sr.abs() + 1.0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("which", ["policy", "reference"])
@pytest.mark.parametrize("mask", [-1e4, -1e6, -1e9, -1e30])
def test_kl_where_the_token_itself_is_masked(am, mask, which, dtype):  # noqa: F811
    """The token's logit is a finite mask in one of the two rows: KL and gradient are those of the formula."""
    for B, T, V in ((2, 3, 40), (3, 5, 9001), (31, 43, 1037), (2, 3, 32003), (1, 1100, 5003)):
        c = Case(B, T, V, dtype, seed=55, masked=0.0)
        x = torch.where(c.x == V - 1, 0, c.x + 1).to(torch.int32)                  # (next to the peak, or anywhere)
        z, zref = c.z.clone(), (c.z.float() + 0.5 * c.n(B, T, V)).to(dtype)
        (z if which == "policy" else zref).scatter_(-1, x.long()[..., None], mask)
        o = R.rows(z, x, zref)
        o["spread"] = _kl_spread(z, zref, o)
        r = am.policy_loss(z.cuda(), x.cuda(), torch.zeros(B, T, device="cuda"), c.ws(am), ref_logits=zref.cuda(),
                           options=am.PolicyOptions(kl_coef=1.0))
        assert not r.status.any()
        R.near(r.kl, o["kl"], R.tol_kl(o), "kl")
        g, tol = R.grad(o, torch.zeros(B, T), k=torch.ones(B, T), dtype=dtype)
        R.near(r.dlogits, g, tol, "dlogits")


@pytest.mark.parametrize("dtype", [BF, F])
def test_kl_of_stretches_whose_mass_is_lost(am, dtype):  # noqa: F811
    """Stretches of tokens below 2^-149 of the row's largest, of which the reference has none: they count as 0, whoever adds them up."""
    for B, T, V in ((1, 2, 128256), (3, 5, 9001), (31, 43, 1037), (2, 600, 20011)):
        c = Case(B, T, V, dtype, seed=56, masked=0.0)
        x = torch.full((B, T), 1, dtype=torch.int32)
        z, zref = c.z.clone(), (c.z.float() + 0.25 * c.n(B, T, V)).to(dtype)
        at = slice(V // 5, V // 5 + V // 2)
        z[..., at], zref[..., at] = -400.0, -INF
        bare = z.clone()
        bare[..., at] = -INF
        opt, ws, one = am.PolicyOptions(kl_coef=0.1, entropy_coef=0.1), c.ws(am), torch.ones(B, T, device="cuda")
        got, want = (am.policy_loss(a.cuda(), x.cuda(), one, ws, ref_logits=zref.cuda(), options=opt) for a in (z, bare))
        assert torch.isfinite(got.kl).all() and torch.isfinite(got.dlogits).all() and not got.status.any()
        for name in ("loss", "token_loss", "logprob", "entropy", "kl", "dlogits"):
            assert torch.equal(getattr(got, name), getattr(want, name)), name


def _rows_of(am, c, z, x, ws, g):  # noqa: F811
    from test_losses import _Rows
    rows = _Rows(z.data_ptr(), int(c.dtype == BF), c.B, c.T, c.V, z.stride(0), z.stride(1), x.data_ptr())
    rows.workspace, rows.ws_bytes = ws.ptr, ws.bytes
    rows.dlogits, rows.d_seq_stride, rows.d_pos_stride = g.data_ptr(), g.stride(0), g.stride(1)
    return rows


@pytest.mark.parametrize("dtype", [BF, F])
def test_zero_rows_of_slices_that_gave_up(am, dtype):  # noqa: F811
    """A broken row with a derivative of 0 is written with zeros, also where a slice's part is done by another workgroup."""
    import ctypes
    lib = am.load_library()
    for B, T, V in ((1, 2, 128256), (3, 5, 32003), (1, 700, 20011)):
        c = Case(B, T, V, dtype, seed=57, masked=0.0)
        z, x, ws = c.z.clone(), c.x.cuda(), c.ws(am)
        z[:, 0::2, V // 3] = math.nan
        z = z.cuda()
        a = torch.ones(B, T, device="cuda")
        a[:, 0::2] = 0.0
        g = torch.full_like(z, 9.0)
        rows = _rows_of(am, c, z, x, ws, g)
        s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert lib.adasd_test_logprob_grad_given_up(ctypes.byref(rows), ctypes.c_void_p(a.data_ptr()), None, s) == 0
        torch.cuda.synchronize()
        assert not g[:, 0::2].any() and torch.isfinite(g).all()


@pytest.mark.parametrize("how", ["unarrived", "given_up"])
@pytest.mark.parametrize("dtype", [BF, F])
def test_policy_loss_whose_records_are_not_waited_for(am, how, dtype):  # noqa: F811
    """A reference's rows and an entropy bonus, where no slice waits for the others' sums, or all count as not there; the gradient
    in the logits' place too (but where records count as not there: they are formed from the logits again)."""
    import ctypes
    from test_losses import _PolicyArgs
    lib = am.load_library()
    for B, T, V in ((1, 2, 128256), (3, 5, 32003), (1, 700, 20011)):
        c = Case(B, T, V, dtype, seed=64)
        zref = (c.z.float() + 0.5 * c.n(B, T, V)).to(dtype)
        adv, old = c.n(B, T), c.old()
        e = R.policy(c.z, c.x, adv, weight=c.w, old=old, zref=zref, kl_coef=0.1, ent=0.01)
        x, ws, q = c.x.cuda(), c.ws(am), zref.cuda()
        d = [v.cuda() for v in (adv, old, c.w)]
        f = getattr(lib, f"adasd_test_policy_loss_{how}")
        for in_place in (False, True) if how == "given_up" else (False,):
            z = c.z.cuda()
            g = z if in_place else torch.full_like(z, 9.0)
            out = torch.full((2 * B * T + 1,), 9.0, device="cuda")
            rows = _rows_of(am, c, z, x, ws, g)
            rows.weight = d[2].data_ptr()
            p = _PolicyArgs(d[0].data_ptr(), 0, d[1].data_ptr(), None, q.data_ptr(), q.stride(0), q.stride(1), None, 0.2, 0.2, 0.1, 0.01,
                            out.data_ptr(), out[1:].data_ptr(), out[1 + B * T:].data_ptr())
            s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
            assert f(ctypes.byref(rows), ctypes.byref(p), s) == 0
            torch.cuda.synchronize()
            R.near(out[0], e["loss"], e["loss_tol"], "loss")
            R.near(out[1:1 + B * T].view(B, T), e["term"], e["term_tol"], "token_loss")
            R.near(out[1 + B * T:].view(B, T), e["kl"], e["kl_tol"], "kl")
            R.near(g, e["g"], e["g_tol"], "dlogits")


@pytest.mark.parametrize("dtype", [BF, F])
def test_gradient_of_a_token_outside_the_vocabulary(am, dtype):  # noqa: F811
    """Its log-probability is NaN, and so is a gradient row that hangs on it; the entropy's gradient needs no token."""
    for B, T, V in ((1, 6, 40), (2, 3, 32003), (31, 43, 1037)):
        c = Case(B, T, V, dtype, seed=58, masked=0.0)
        x = c.x.clone()
        x[0, 1], x[0, 2] = -100, V
        a, h = c.n(B, T), c.n(B, T)
        a[0, 2] = 0.0
        o = R.rows(c.z, c.x)
        for dH in (None, h):
            g = am.token_logprob_grad(c.z.cuda(), x.cuda(), c.ws(am), a.cuda(), cu(dH))
            assert torch.isnan(g[0, 1]).all()
            want, tol = R.grad(o, a, dH, dtype=dtype)
            g[0, 1] = want[0, 1].to(g)
            R.near(g, want, tol, "dlogits")


@pytest.mark.parametrize("dtype", [BF, F])
def test_sampled_kl_of_tokens_without_mass(am, dtype):  # noqa: F811
    """exp(d) - 1 - d is +inf at both ends: a token without mass in the row (d = +inf), or in the reference (d = -inf)."""
    for B, T, V in ((2, 3, 40), (2, 3, 32003), (31, 43, 1037)):
        c = Case(B, T, V, dtype, seed=59, masked=0.0)
        z, ref = c.z.clone(), c.lp.float().clone()
        z[0, 0, int(c.x[0, 0])] = -INF
        ref[0, 1] = -INF
        one = torch.ones(B, T, device="cuda")
        o = am.policy_loss(z.cuda(), c.x.cuda(), one, c.ws(am), ref_logprob=ref.cuda(), old_logprob=c.old().cuda(),
                           options=am.PolicyOptions(kl_coef=0.1))
        assert o.kl[0, 0].item() == INF and o.kl[0, 1].item() == INF and torch.isfinite(o.kl.cpu().view(-1)[2:]).all()
        assert o.token_loss[0, 0].item() == INF and o.token_loss[0, 1].item() == INF and o.loss.item() == INF
        assert torch.isfinite(o.dlogits[0, 1]).all() and not torch.isfinite(o.dlogits[0, 0, int(c.x[0, 0])]).item()


@pytest.mark.parametrize("margin", [0.0, 3.0, 17.0, 30.0, 34.0, 38.0, 60.0, 80.0])
def test_logistic_loss_of_large_margins(am, margin):  # noqa: F811
    """Loss and gradients of a pair that is far apart are small, and right to the last digits: float logits of two tokens, a margin set by the
    reference's log-probabilities.  m is formed in 64 bits from a float log-probability's sums (r of loss_ref for two scores, beta 1) and e^-m is off by
    that error relatively; loss and gradient are rounded twice more (4 steps of float are allowed)."""
    V = 8
    z = torch.randn(2, 1, V, generator=torch.Generator().manual_seed(60))
    x = torch.tensor([[1], [2]], dtype=torch.int32)
    lp = R.rows(z, x)["lp"]
    for sign in (1.0, -1.0):
        ref = (lp - torch.tensor([[sign * margin], [0.0]])).float()
        o = am.preference_loss(z.cuda(), x.cuda(), am.LossWorkspace(2, 1, V, F), ref_logprob=ref.cuda(), options=am.PreferenceOptions(beta=1.0))
        e = R.rows(z, x)
        m = (e["lp"] - ref.double())[0, 0] - (e["lp"] - ref.double())[1, 0]
        loss, slope = torch.log1p(torch.exp(-m.abs())) + (-m).clamp_min(0.0), -1.0 / (1.0 + torch.exp(m))
        rel = 2 * e["r"] + 4 * R.H24
        assert abs(o.pair_loss.item() - loss.item()) <= rel * loss.item()
        p = e["p"][:, 0]
        g = torch.stack([slope * ((torch.arange(V) == 1).double() - p[0]), -slope * ((torch.arange(V) == 2).double() - p[1])])
        # (1 - p of the token: both parts are rounded)
        tol = slope.abs() * (rel + e["r"] + 4 * R.H24) * (p + torch.stack([(torch.arange(V) == k).double() for k in (1, 2)]))
        R.near(o.dlogits[:, 0], g, tol, "dlogits")


def test_results_are_tensors_of_their_own(am):  # noqa: F811
    """Each result has its storage: it can be kept, saved and written to by itself."""
    import io
    c = Case(4, 3, 40, F, seed=61)
    z, x, ws, one = c.z.cuda(), c.x.cuda(), c.ws(am), torch.ones(4, 3, device="cuda")
    results = [am.token_logprob(z, x, ws), list(vars(am.policy_loss(z, x, one, ws)).values()), list(vars(am.preference_loss(z, x, ws)).values())]
    for r in results:
        assert len({t.untyped_storage().data_ptr() for t in r}) == len(r)
        for t in r:
            assert t.untyped_storage().nbytes() == t.numel() * t.element_size() and t.storage_offset() == 0 and t.is_contiguous()
        f = io.BytesIO()
        torch.save(list(r), f)
        f.seek(0)
        assert all(torch.equal(a.cpu(), b) for a, b in zip(r, torch.load(f, map_location="cpu", weights_only=True)))
    with torch.inference_mode():
        lp = am.token_logprob(z, x, ws)[0]
        assert lp.is_inference()
    empty = am.token_logprob(torch.empty(0, 40, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), ws)
    assert all(t.shape == (0,) for t in empty)


def test_tensors_written_to_are_known_to_torch(am):  # noqa: F811
    """A gradient in the place of logits that torch has saved for a backward pass is noticed there, as every write in place is."""
    c = Case(2, 3, 40, F, seed=62)
    ws, x, one = c.ws(am), c.x.cuda(), torch.ones(2, 3, device="cuda")
    h = c.z.cuda().requires_grad_(True)
    for call in (lambda v: am.token_logprob_grad(v, x, ws, one, dlogits=v), lambda v: am.policy_loss(v, x, one, ws, dlogits=v),
                 lambda v: am.preference_loss(v, x, ws, dlogits=v)):
        z = torch.tanh(h)                                    # (tanh's backward needs its result)
        before = z._version
        call(z)
        assert z._version == before + 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.sum().backward()
        z = h * 3.0                                          # (this one's does not)
        call(z)
        z.backward(z.detach())
    given = [torch.empty(2, 3, device="cuda"), torch.empty(2, 3, device="cuda"), torch.empty(2, 3, dtype=torch.int32, device="cuda")]
    z = c.z.cuda()
    am.token_logprob(z, x, ws, None, *given)
    assert [t._version for t in given] == [1, 1, 1] and z._version == 0
    am.policy_loss(z, x, one, ws)
    assert z._version == 0
    with torch.inference_mode():
        y = c.z.cuda()
        am.policy_loss(y, x, one, ws, dlogits=y)
    am.policy_loss(y, x, one, ws, dlogits=y)                 # (an inference tensor has no version)


def test_workspaces_of_the_other_kind_are_refused(am):  # noqa: F811
    """The scratch of verification and drafting, and that of the losses, are laid out differently."""
    B, K, V = 2, 3, 512
    c = Case(B, K, V, F, seed=63)
    z, x, one = c.z.cuda(), c.x.cuda(), torch.ones(B, K, device="cuda")
    ws, lws = am.Workspace(B, K, V, F), am.LossWorkspace(B, K, V, F)
    target = torch.randn(B, K + 1, V, device="cuda")
    for bad in (lambda: am.token_logprob(z, x, ws), lambda: am.token_logprob_grad(z, x, ws, one), lambda: am.policy_loss(z, x, one, ws),
                lambda: am.preference_loss(z, x, ws), lambda: am.token_logprob(z, x, None), lambda: am.draft_entropy(z[:, 0], lws),
                lambda: am.draft_step(z[:, 0], lws), lambda: am.verify(target, z, x, lws),
                lambda: am.verify_shard_stats(target, z, x, lws, am.Shard(1, 0, V, 0))):
        with pytest.raises(TypeError, match="orkspace"):
            bad()

    class Mine(am.LossWorkspace):
        pass
    assert am.token_logprob(z, x, Mine(B, K, V, F))[0].shape == (B, K)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("offset", [0.0, 300.0, 3e4, 3e6, 3e7])
def test_kl_of_rows_with_different_offsets(am, offset, dtype):  # noqa: F811
    """Softmax does not see a row's offset: KL and gradient have the accuracy of rows without one.  (The type's rounding of the shifted logits
    is part of the inputs.)"""
    for B, T, V in ((2, 3, 40), (3, 5, 9001), (31, 43, 1037), (2, 3, 32003), (1, 1100, 5003)):
        c = Case(B, T, V, dtype, seed=65, masked=0.0)
        if dtype == BF:                                                             # (differences that the type still has at that size)
            step = max(offset / 256, 1.0)
            z, zref = (c.z.float() * step / 3 + offset).to(dtype), (c.z.float() * step / 3 + step * c.n(B, T, V).round() - offset).to(dtype)
        else:
            z, zref = c.z + offset, c.z + 0.5 * c.n(B, T, V) - offset
        o = R.rows(z, c.x, zref)
        o["spread"] = _kl_spread(z, zref, o)
        r = am.policy_loss(z.cuda(), c.x.cuda(), torch.zeros(B, T, device="cuda"), c.ws(am), ref_logits=zref.cuda(),
                           options=am.PolicyOptions(kl_coef=1.0))
        assert not r.status.any()
        R.near(r.kl, o["kl"], R.tol_kl(o), "kl")
        g, tol = R.grad(o, torch.zeros(B, T), k=torch.ones(B, T), dtype=dtype)
        R.near(r.dlogits, g, tol, "dlogits")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n, V", [(4000, 2752), (4000, 9001), (2000, 32003), (64, 32003)])
def test_log_probabilities_have_no_bias(am, n, V, dtype):  # noqa: F811
    """The mean error of many rows, so that scores of long sequences do not drift: read off a sampled KL, which is formed from the log-probability
    before it is rounded, against a reference about 1 above.  Errors of single rows are within 7e-8 rms (of s: one rounding a term, five in the
    folds); their mean is within 4 of its standard deviations, and 2e-9 for factors of parts that are not counted."""
    def sums(seed):
        g = torch.Generator("cuda").manual_seed(seed)
        z = 3.0 * torch.randn(n, 1, V, device="cuda", generator=g)
        x = torch.randint(0, V, (n, 1, 1), device="cuda", generator=g)
        z = z.scatter_add_(-1, x, torch.full((n, 1, 1), 10.0, device="cuda")).to(dtype)
        lp = torch.cat([torch.log_softmax(r.double(), -1).gather(-1, k)[..., 0] for r, k in zip(z.split(256), x.split(256))])
        ref = (lp + 1.0).float()
        d = ref.double() - lp
        o = am.policy_loss(z, x[..., 0].to(torch.int32), torch.zeros(n, 1, device="cuda"), am.LossWorkspace(n, 1, V, dtype), ref_logprob=ref)
        # (kl is a float: half a step of 0.72 is 3e-8, over expm1(1) = 1.7)
        return -((o.kl.double() - (torch.expm1(d) - d)) / torch.expm1(d))
    e = torch.cat([sums(70 + k) for k in range(max(1, 2000 // n))])
    assert e.pow(2).mean().sqrt() < 7e-8
    assert e.mean().abs() < 4 * 7e-8 / math.sqrt(e.numel()) + 2e-9


@pytest.mark.parametrize("dtype", [BF, F])
def test_tokens_with_all_the_mass(am, dtype):  # noqa: F811
    """Log-probabilities are not above 0 (nor ratios and scores formed from them), and entropies not below, by no rounding."""
    for B, T, V in ((4, 64, 40), (4, 64, 5003), (2, 8, 128256), (40, 50, 1037)):
        c = Case(B, T, V, dtype, seed=66, masked=0.0)
        z = c.z.clone()
        z.scatter_(-1, c.x.long()[..., None], (60.0 + 30.0 * torch.rand(B, T, 1, generator=torch.Generator().manual_seed(67))).to(dtype))
        lp, H, _ = am.token_logprob(z.cuda(), c.x.cuda(), c.ws(am))
        assert (lp <= 0).all() and (lp > -1e-6).all() and (H >= 0).all() and (H < 1e-5).all()
        o = am.policy_loss(z.cuda(), c.x.cuda(), torch.ones(B, T, device="cuda"), c.ws(am), old_logprob=torch.zeros(B, T, device="cuda"))
        assert (o.token_loss >= -1).all()
        p = am.preference_loss(z.cuda(), c.x.cuda(), c.ws(am))
        assert (p.score <= 0).all()
#--END
