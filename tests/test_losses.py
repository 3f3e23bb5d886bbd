"""Losses over vocabulary rows without a GPU: the oracle of the GPU tests against differentiation and differences, and what the
entry points refuse before anything is enqueued."""
import ctypes as C

import pytest
import torch

import loss_ref as R


def _case(B=4, T=3, V=11, seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    z = 2 * n(B, T, V)
    x = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32)
    w = torch.rand(B, T, generator=g, dtype=torch.float64)
    w[1, 0] = 0.0
    lp = torch.log_softmax(z, -1).gather(-1, x.long()[..., None])[..., 0]
    return z, x, w, lp, n


R.HALF[torch.float64] = 0.0


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("ent", [0.0, 0.3])
def test_policy_oracle_is_the_formulas_derivative(kl, ent):
    z, x, w, lp, n = _case(seed=3)
    adv, old, ref, zref = n(4, 3), lp + 0.3 * n(4, 3), lp + 0.5 * n(4, 3), z + n(4, 3, 11)
    kw = dict(weight=w, old=old, kl_coef=0.0 if kl == "none" else 0.7, ent=ent, ref=ref if kl == "sampled" else None, zref=zref if kl == "full" else None)
    o = R.policy(z, x, adv, **kw)
    step = 1e-6
    for b, t, j in [(0, 0, 0), (1, 1, 5), (2, 2, 10), (3, 0, int(x[3, 0])), (1, 0, 2)]:
        up, dn = z.clone(), z.clone()
        up[b, t, j] += step
        dn[b, t, j] -= step
        diff = (R.policy(up, x, adv, **kw)["loss"] - R.policy(dn, x, adv, **kw)["loss"]) / (2 * step)
        assert abs(diff - o["g"][b, t, j]) < 1e-8, (b, t, j)
    v = z.clone().requires_grad_(True)
    l = torch.log_softmax(v, -1)
    p = l.gather(-1, x.long()[..., None])[..., 0]
    r = torch.exp(p - old)
    import numpy as np
    lo, hi = 1 - float(np.float32(0.2)), 1 + float(np.float32(0.2))
    term = -torch.minimum(r * adv, r.clamp(lo, hi) * adv)
    if kl == "sampled":
        term = term + 0.7 * (torch.exp(ref - p) - (ref - p) - 1)
    if kl == "full":
        term = term + 0.7 * (l.exp() * (l - torch.log_softmax(zref, -1))).sum(-1)
    term = term + ent * (l.exp() * l).sum(-1)
    loss = (w * term).sum()
    loss.backward()
    assert torch.allclose(loss, o["loss"], rtol=1e-12) and torch.allclose(v.grad, o["g"], rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("kind", ["logistic", "squared", "hinge"])
def test_preference_oracle_is_the_formulas_derivative(kind):
    z, x, w, lp, n = _case(seed=5)
    kw = dict(weight=w, ref=lp + 0.5 * n(4, 3), pair_weight=torch.tensor([0.25, 2.0]), kind=kind, beta=0.5, margin=0.125,
              smoothing=0.125 if kind == "logistic" else 0.0)
    o = R.preference(z, x, **kw)
    step = 1e-6
    for b, t, j in [(0, 0, 0), (1, 1, 5), (2, 2, 10), (3, 0, int(x[3, 0])), (1, 0, 2)]:
        up, dn = z.clone(), z.clone()
        up[b, t, j] += step
        dn[b, t, j] -= step
        diff = (R.preference(up, x, **kw)["loss"] - R.preference(dn, x, **kw)["loss"]) / (2 * step)
        assert abs(diff - o["g"][b, t, j]) < 1e-8, (b, t, j)


# ---- refusals

@pytest.fixture(scope="module")
def lib():
    import paper_2512_11280_amd as am
    from paper_2512_11280_amd import build as b
    b.build(force=False)
    L = am.load_library()
    L.adasd_token_logprob.argtypes = [C.POINTER(_Rows), C.c_void_p]
    L.adasd_token_logprob_grad.argtypes = [C.POINTER(_Rows), C.c_void_p, C.c_void_p, C.c_void_p]
    L.adasd_policy_loss.argtypes = [C.POINTER(_Rows), C.POINTER(_PolicyArgs), C.c_void_p]
    L.adasd_preference_loss.argtypes = [C.POINTER(_Rows), C.POINTER(_PreferenceArgs), C.c_void_p]
    return L


class _Rows(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("dt", C.c_int), ("B", C.c_int32), ("T", C.c_int32), ("V", C.c_int32),
                ("seq_stride", C.c_int64), ("pos_stride", C.c_int64), ("tokens", C.c_void_p), ("weight", C.c_void_p),
                ("active", C.c_void_p), ("logprob", C.c_void_p), ("entropy", C.c_void_p), ("status", C.c_void_p),
                ("dlogits", C.c_void_p), ("d_seq_stride", C.c_int64), ("d_pos_stride", C.c_int64),
                ("workspace", C.c_void_p), ("ws_bytes", C.c_size_t)]


class _PolicyArgs(C.Structure):
    _fields_ = [("advantage", C.c_void_p), ("adv_per_seq", C.c_int32), ("old_logprob", C.c_void_p),
                ("ref_logprob", C.c_void_p), ("ref_logits", C.c_void_p), ("r_seq_stride", C.c_int64),
                ("r_pos_stride", C.c_int64), ("grad_scale", C.c_void_p), ("clip_low", C.c_float), ("clip_high", C.c_float),
                ("kl_coef", C.c_float), ("entropy_coef", C.c_float), ("loss", C.c_void_p), ("token_loss", C.c_void_p),
                ("kl", C.c_void_p)]


class _PreferenceArgs(C.Structure):
    _fields_ = [("kind", C.c_int32), ("beta", C.c_float), ("margin", C.c_float), ("label_smoothing", C.c_float),
                ("ref_logprob", C.c_void_p), ("pair_weight", C.c_void_p), ("grad_scale", C.c_void_p), ("loss", C.c_void_p),
                ("pair_loss", C.c_void_p), ("pair_margin", C.c_void_p), ("score", C.c_void_p)]


P0 = 1 << 20            # addresses that are never followed: every call below is refused on the host


def _rows(**kw):
    a = _Rows(P0, 1, 2, 3, 100, 300, 100, P0 << 4)
    a.dlogits, a.d_seq_stride, a.d_pos_stride = P0 << 8, 300, 100
    a.workspace, a.ws_bytes = P0 << 10, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _policy(**kw):
    p = _PolicyArgs(P0 << 5, 0, P0 << 5)
    p.clip_low = p.clip_high = 0.2
    p.loss = P0 << 5
    p.r_seq_stride, p.r_pos_stride = 300, 100
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _preference(**kw):
    p = _PreferenceArgs(0, 0.1, 0.0, 0.0)
    p.loss = P0 << 5
    for k, v in kw.items():
        setattr(p, k, v)
    return p


ROWS = [
    (dict(B=-1), -1), (dict(V=0), -1), (dict(dt=7), -1), (dict(V=(1 << 24) + 1), -5), (dict(B=1 << 20, T=2), -5),
    (dict(logits=None), -1), (dict(tokens=None), -1),
    (dict(pos_stride=99), -1), (dict(seq_stride=299), -1), (dict(seq_stride=0), -1), (dict(pos_stride=-100), -1),
    (dict(seq_stride=1 << 60), -1),
    (dict(logits=P0 + 1), -2), (dict(tokens=(P0 << 4) + 2), -2), (dict(logprob=P0 + 2), -2), (dict(status=P0 + 1), -2),
    (dict(workspace=None), -4), (dict(workspace=(P0 << 10) + 64), -2), (dict(ws_bytes=4096), -4),
]


@pytest.mark.parametrize("change, code", ROWS)
def test_rows_are_checked_on_the_host(lib, change, code):
    a = _rows(**change)
    assert lib.adasd_token_logprob(C.byref(a), None) == code
    assert lib.adasd_token_logprob_grad(C.byref(a), P0, None, None) == code
    assert lib.adasd_policy_loss(C.byref(a), C.byref(_policy()), None) == code
    if change.get("B", 2) % 2 == 0:
        assert lib.adasd_preference_loss(C.byref(a), C.byref(_preference()), None) == code


@pytest.mark.parametrize("change, code", [
    (dict(d_pos_stride=99), -1), (dict(d_seq_stride=150), -1), (dict(dlogits=(P0 << 8) + 1), -2),
    (dict(dlogits=P0 + 2), -1),                                      # shifted by an element: overlaps
    (dict(dlogits=P0 + 1000), -1), (dict(dlogits=P0, d_pos_stride=101, d_seq_stride=400), -1),
])
def test_gradient_memory_is_checked_on_the_host(lib, change, code):
    a = _rows(**change)
    assert lib.adasd_token_logprob_grad(C.byref(a), P0, None, None) == code
    assert lib.adasd_policy_loss(C.byref(a), C.byref(_policy()), None) == code
    assert lib.adasd_preference_loss(C.byref(a), C.byref(_preference()), None) == code


def test_log_probability_calls_refuse(lib):
    assert lib.adasd_token_logprob(None, None) == -1
    assert lib.adasd_token_logprob(C.byref(_rows(weight=P0)), None) == -1       # weights belong to the losses
    assert lib.adasd_token_logprob_grad(C.byref(_rows()), None, None, None) == -1
    assert lib.adasd_token_logprob_grad(C.byref(_rows(dlogits=None)), P0, None, None) == -1
    assert lib.adasd_token_logprob_grad(C.byref(_rows()), P0 + 1, None, None) == -2
    assert lib.adasd_token_logprob(C.byref(_rows(B=0, logits=None, tokens=None)), None) == 0      # nothing to do
    n = C.c_size_t()
    assert lib.adasd_loss_workspace_bytes(2, 3, 100, 1, None) == -1
    assert lib.adasd_loss_workspace_bytes(2, -3, 100, 1, C.byref(n)) == -1
    assert lib.adasd_loss_workspace_bytes(1 << 11, 1 << 10, 100, 1, C.byref(n)) == -5
    assert lib.adasd_loss_workspace_bytes(4, 8, 100, 1, C.byref(n)) == 0
    small = n.value
    assert lib.adasd_loss_workspace_bytes(8, 8, 100, 1, C.byref(n)) == 0 and n.value > small > 0


@pytest.mark.parametrize("change, code", [
    (dict(ref_logprob=P0, ref_logits=P0), -1), (dict(adv_per_seq=2), -1), (dict(clip_low=-0.1), -1), (dict(clip_low=1.1), -1),
    (dict(clip_low=float("nan")), -1), (dict(clip_high=-0.1), -1), (dict(kl_coef=float("inf")), -1), (dict(entropy_coef=float("nan")), -1),
    (dict(loss=None), -1), (dict(advantage=None), -1), (dict(advantage=P0 + 1), -2), (dict(kl=P0 + 1), -2),
    (dict(ref_logits=P0 << 9, r_pos_stride=50), -1), (dict(ref_logits=(P0 << 9) + 1), -2),
    (dict(ref_logits=(P0 << 8) + 64), -1),                            # the gradient would overwrite the reference
])
def test_policy_loss_refuses(lib, change, code):
    assert lib.adasd_policy_loss(C.byref(_rows()), C.byref(_policy(**change)), None) == code
    assert lib.adasd_policy_loss(C.byref(_rows(active=P0)), C.byref(_policy()), None) == -1
    assert lib.adasd_policy_loss(None, C.byref(_policy()), None) == -1
    assert lib.adasd_policy_loss(C.byref(_rows()), None, None) == -1


@pytest.mark.parametrize("change, code", [
    (dict(kind=3), -1), (dict(beta=0.0), -1), (dict(beta=float("inf")), -1), (dict(margin=float("nan")), -1),
    (dict(label_smoothing=1.5), -1), (dict(kind=1, label_smoothing=0.1), -1), (dict(loss=None), -1), (dict(score=P0 + 2), -2),
])
def test_preference_loss_refuses(lib, change, code):
    assert lib.adasd_preference_loss(C.byref(_rows()), C.byref(_preference(**change)), None) == code
    assert lib.adasd_preference_loss(C.byref(_rows(B=3)), C.byref(_preference()), None) == -1
    assert lib.adasd_preference_loss(C.byref(_rows(T=0)), C.byref(_preference()), None) == -1
    assert lib.adasd_preference_loss(None, None, None) == -1


@pytest.mark.parametrize("call, error, text", [
    (lambda am, z, x: am.token_logprob(z, x, None), ValueError, "logits must be a CUDA tensor"),
    (lambda am, z, x: am.token_logprob_grad(z[0, 0], x, None, x), ValueError, "logits must be a CUDA tensor"),
    (lambda am, z, x: am.policy_loss(z, x, x, None), ValueError, "logits must be a CUDA tensor"),
    (lambda am, z, x: am.preference_loss(z[0], x, None), ValueError, r"\[2P, T, V\]"),
    (lambda am, z, x: am.preference_loss("z", x, None), ValueError, r"\[2P, T, V\]"),
])
def test_binding_checks_its_arguments(call, error, text):
    import paper_2512_11280_amd as am
    with pytest.raises(error, match=text):
        call(am, torch.zeros(2, 3, 8), torch.zeros(2, 3, dtype=torch.int32))
