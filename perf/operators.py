"""What the losses over vocabulary rows are timed on: log-probabilities of tokens, the clipped policy loss and the preference loss,
with their gradients, as a training step or a serving loop calls them through the package.

Each case is made as such a program has it in hand: logits [B, T, V] of a forward pass, the tokens, per-token weights (a mask divided
by what the mean is taken over), and what an earlier pass left (log-probabilities of the behaviour policy and of the reference).

The plain form computes every row in 32 bits with elementary operations and the few numbers per position in 64 (a ratio near its
clipping border, sums over a sequence).
"""
import math

import torch

own = False

# Vocabularies 32000 / 128256 / 152064 and the odd 32003 are those of the package's other cases; windows of 8 and 20 positions and
# batches of 1 to 32 as well.  Sequences of 100 to 1024 positions are what losses are computed over.
LISTED = [
    # log-probability of the token just emitted to a single stream: the smallest call there is
    dict(name="logprob_one", kind="logprob", B=1, T=1, V=128256, dtype="bf16", ragged=False, view=False),
    # log-probabilities of all tokens of a batch's verified windows
    dict(name="logprob_windows", kind="logprob", B=32, T=8, V=128256, dtype="bf16", ragged=True, view=False),
    # rescoring of whole rollouts (the old log-probabilities of a policy step), next-token view of the logits
    dict(name="logprob_rollouts", kind="logprob", B=4, T=1024, V=128256, dtype="bf16", ragged=True, view=True),
    # a loss of the caller's own: gradient of log-probabilities and entropies, odd vocabulary, float logits, ragged
    dict(name="logprob_grad_odd", kind="logprob_grad", B=3, T=101, V=32003, dtype="f32", ragged=True, view=False),
    # policy step over a handful of short answers of a small model, float logits
    dict(name="policy_small", kind="policy", B=4, T=20, V=32000, dtype="f32", ragged=False, view=False, kl="sampled", entropy=0.0),
    # ordinary policy step: ragged answers, KL from the reference's log-probabilities
    dict(name="policy_ragged", kind="policy", B=32, T=64, V=128256, dtype="bf16", ragged=True, view=False, kl="sampled", entropy=0.0),
    # KL over the whole vocabulary against the reference's logits, and an entropy bonus
    dict(name="policy_full_kl", kind="policy", B=8, T=128, V=152064, dtype="bf16", ragged=False, view=False, kl="full", entropy=0.01),
    # the same on an odd vocabulary in float, next-token views
    dict(name="policy_full_kl_odd", kind="policy", B=5, T=77, V=32003, dtype="f32", ragged=True, view=True, kl="full", entropy=0.0),
    # the largest step: a micro-batch of long answers, no reference
    dict(name="policy_large", kind="policy", B=16, T=512, V=128256, dtype="bf16", ragged=False, view=False, kl="none", entropy=0.0),
    # two short pairs of a small model, odd vocabulary
    dict(name="preference_small", kind="preference", B=4, T=33, V=32003, dtype="bf16", ragged=True, view=True, loss="logistic"),
    # ordinary step: sixteen answers of different lengths
    dict(name="preference_batch", kind="preference", B=16, T=128, V=128256, dtype="bf16", ragged=True, view=True, loss="logistic"),
    # float logits, length-averaged scores, squared loss
    dict(name="preference_f32", kind="preference", B=8, T=64, V=128256, dtype="f32", ragged=False, view=False, loss="squared"),
]
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_MOST = 16 * 512 * 128256 * 4            # bytes read and written by the largest listed case
CLIP_LOW, CLIP_HIGH, KL_COEF, BETA, SMOOTHING = 0.2, 0.28, 0.04, 0.1, 0.05


def listed():
    return [dict(c) for c in LISTED]


def _log_between(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["logprob", "logprob_grad", "policy", "policy", "preference", "preference"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = _log_between(rng, 2000, 152064)
    grain = rng.choice([64, 64, 8, 1])   # padded vocabularies mostly, and any size at all
    c = dict(kind=kind, B=_log_between(rng, 1, 64), T=_log_between(rng, 1, 1024), V=max(1, V // grain) * grain, dtype=dtype,
             ragged=rng.random() < 0.6, view=rng.random() < 0.4)
    if kind == "policy":
        c.update(kl=rng.choice(["none", "sampled", "full"]), entropy=rng.choice([0.0, 0.01]))
    if kind == "preference":
        c.update(loss=rng.choice(["logistic", "squared", "hinge"]), B=c["B"] + c["B"] % 2)
    per_row = _passes(c) * c["V"] * _SIZE[dtype]
    c["T"] = max(1, min(c["T"], _MOST // (per_row * c["B"])))
    return c


def _passes(c):                          # rows of logits that a position reads and writes
    return {"logprob": 1, "logprob_grad": 2, "preference": 2}.get(c["kind"]) or (3 if c["kl"] == "full" else 2)


def _span(c):
    """First and last position (exclusive) of each sequence that counts: a prompt before, padding behind."""
    B, T = c["B"], c["T"]
    if not c["ragged"]:
        return [(0, T)] * B
    spans = []
    for b in range(B):
        first = (b * 5 + 1) % 7 * T // 40
        spans.append((first, max(first + 1, T - (b * 11 % 13) * T // 24)))
    return spans


def _rows_counted(c):
    return sum(e - f for f, e in _span(c))


def _logits(c, gen, like=None, noise=0.0):
    """Rows of N(0, 3^2) with a peak at one index, or noisy copies of other rows; a view of a longer sequence's where the case says so."""
    B, T, V, dt = c["B"], c["T"], c["V"], _DTYPE[c["dtype"]]
    buf = torch.empty(B, T + 1 if c["view"] else T, V, dtype=dt, device="cuda")
    z = buf[:, :T]
    peak = torch.randint(0, V, (B, T), generator=gen, device="cuda")
    for b in range(B):
        r = torch.randn(T, V, generator=gen, device="cuda")
        if like is None:
            r *= 3.0
            r.scatter_add_(1, peak[b][:, None], torch.full((T, 1), 10.0, device="cuda"))
        else:
            r = r * noise + like[b].float()
        z[b] = r
    if c["view"]:
        buf[:, T] = 0
    return z, peak


def _logprob_now(z, x):
    """What an earlier pass of the same model would have left (to rounding): in slices, as large cases have many rows."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for b in range(x.shape[0]):
        r = z[b].float()
        out[b] = r.gather(1, x[b].long()[:, None])[:, 0].double() - torch.logsumexp(r, 1).double()
    return out


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, T, V = c["B"], c["T"], c["V"]
    f32 = dict(dtype=torch.float32, device="cuda")
    z, peak = _logits(c, gen)
    other = torch.randint(0, V, (B, T), generator=gen, device="cuda")
    x = torch.where(torch.rand(B, T, generator=gen, device="cuda") < 0.7, peak, other).to(torch.int32)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    mask = torch.zeros(B, T, **f32)
    for b, (f, e) in enumerate(_span(c)):
        mask[b, f:e] = 1.0
    s = dict(case=c, z=z, x=x)
    if own:
        import paper_2512_11280_amd as am
        s["ws"] = am.LossWorkspace(B, T, V, z.dtype)
    if c["kind"] == "logprob":
        s.update(active=mask.to(torch.uint8) if c["ragged"] else None)
        return s
    if c["kind"] == "logprob_grad":
        s.update(active=mask.to(torch.uint8) if c["ragged"] else None, dlp=normal(B, T), dH=0.1 * normal(B, T))
        return s
    lp = _logprob_now(z, x)
    if c["kind"] == "policy":
        # Ratios spread about 1.  One next to a border of the clipping may fall on either side of it by rounding alone, and has its
        # gradient there or has none: such positions are moved off it.
        d = 0.15 * normal(B, T).double()
        for border in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH), 0.0):
            d = torch.where((d - border).abs() < 1e-3, d + 3e-3, d)
        s.update(weight=mask / mask.sum(), old=(lp - d).float(), adv=normal(B, T) if c["T"] <= 64 else normal(B),
                 ref=(lp + 0.3 * normal(B, T).double()).float() if c["kl"] == "sampled" else None,
                 zref=_logits(c, gen, like=z, noise=0.5)[0] if c["kl"] == "full" else None,
                 scale=torch.full((1,), 8.0, **f32) if c["kl"] == "sampled" else None)
        return s
    w = mask / mask.sum(1, keepdim=True) if c["loss"] == "squared" else mask
    s.update(weight=w, ref=(lp + 0.2 * normal(B, T).double()).float())
    if c["loss"] == "hinge":             # margins next to the hinge's corner: moved off it, as above
        P, ref = B // 2, s["ref"]
        score = (w.double() * (lp - ref.double())).sum(1)
        near = (BETA * (score[:P] - score[P:]) - 1.0).abs() < 1e-3
        ref[:P] += torch.where(near, 0.2, 0.0).float()[:, None]
    return s


# ---- the plain form ------------------------------------------------------------------------------------------------------------

def _rows(z, x):
    """exp(z - max) [.., V], its sum, z - max (masked logits at a finite value), log-probability and entropy (64 bits per position)."""
    z = z.float()
    d = z - z.amax(-1, keepdim=True)
    e = torch.exp(d)
    s = e.sum(-1)
    d = d.clamp_min(-200.0)
    lns = torch.log(s.double())
    lp = d.gather(-1, x.long()[..., None])[..., 0].double() - lns
    H = lns - (d * e).sum(-1).double() / s.double()
    return e, s, d, lns, lp, H


def _gradient(z, x, e, s, a, bracket):
    """a (1[j = x] - p) + p bracket, for a [.., 1] and a bracket that broadcasts over the row."""
    a = a.float()[..., None]
    g = (bracket - a) * (e / s[..., None])
    g.scatter_add_(-1, x.long()[..., None], a)
    return g.to(z.dtype)


def _plain_logprob(st):
    z, x, active = st["z"], st["x"], st["active"]
    e, s, d, lns, lp, H = _rows(z, x)
    on = torch.ones_like(lp) if active is None else active.double()
    out = [(lp * on).float(), (H * on).float(), torch.zeros_like(x)]
    if st["case"]["kind"] == "logprob_grad":
        a, c = st["dlp"].double() * on, st["dH"].double() * on
        lnp = d - lns.float()[..., None]
        out.append(_gradient(z, x, e, s, a, -c.float()[..., None] * (lnp + H.float()[..., None])))
    return out


def _plain_policy(st):
    c, z, x, w = st["case"], st["z"], st["x"], st["weight"].double()
    e, s, d, lns, lp, H = _rows(z, x)
    A = st["adv"].double()
    A = A[:, None].expand_as(lp) if A.dim() == 1 else A
    r = torch.exp(lp - st["old"].double())
    free, held = r * A, r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * A
    loss = -torch.minimum(free, held)
    a = torch.where(free <= held, -A * r, 0.0)
    kl = torch.zeros_like(lp)
    bracket = torch.zeros((), device=z.device)
    if c["kl"] == "sampled":
        delta = st["ref"].double() - lp
        kl = torch.expm1(delta) - delta
        a = a - KL_COEF * torch.expm1(delta)
    if c["kl"] == "full":
        q = st["zref"].float()
        dq = q - q.amax(-1, keepdim=True)
        D = (d - dq) - (lns - torch.log(torch.exp(dq).sum(-1).double())).float()[..., None]
        kl = (e * D).sum(-1).double() / s.double()
        bracket = KL_COEF * (D - kl.float()[..., None])
    if c["entropy"]:
        bracket = bracket + c["entropy"] * ((d - lns.float()[..., None]) + H.float()[..., None])
    on = (w != 0).double()
    loss = (loss + KL_COEF * kl - c["entropy"] * H) * on
    W = w if st["scale"] is None else w * st["scale"].double()
    g = _gradient(z, x, e, s, a * W, bracket * W.float()[..., None])
    return [(w * loss).sum().float(), loss.float(), (lp * on).float(), (H * on).float(), (kl * on).float(), torch.zeros_like(x), g]


def _plain_preference(st):
    c, z, x, w = st["case"], st["z"], st["x"], st["weight"].double()
    P = c["B"] // 2
    e, s, d, lns, lp, H = _rows(z, x)
    score = (w * (lp - st["ref"].double())).sum(1)
    m = score[:P] - score[P:]
    if c["loss"] == "squared":
        pair, slope = (m - 0.5 / BETA).square(), 2.0 * (m - 0.5 / BETA)
    else:
        m = BETA * m
        if c["loss"] == "hinge":
            pair, slope = (1.0 - m).clamp_min(0.0), torch.where(m < 1.0, -BETA, 0.0).double()
        else:
            soft = lambda v: torch.log1p(torch.exp(-v.abs())) + v.clamp_min(0.0)  # noqa: E731
            pair = (1.0 - SMOOTHING) * soft(-m) + SMOOTHING * soft(m)
            slope = BETA * (SMOOTHING / (1.0 + torch.exp(-m)) - (1.0 - SMOOTHING) / (1.0 + torch.exp(m)))
    a = torch.cat([slope, -slope])[:, None] * w / P
    on = (w != 0).double()
    return [pair.mean().float(), pair.float(), m.float(), score.float(), (lp * on).float(), torch.zeros_like(x),
            _gradient(z, x, e, s, a, torch.zeros((), device=z.device))]


def run(state):
    st, c = state, state["case"]
    if not own:
        return {"policy": _plain_policy, "preference": _plain_preference}.get(c["kind"], _plain_logprob)(st)
    import paper_2512_11280_amd as am
    if c["kind"] in ("logprob", "logprob_grad"):
        lp, H, status = am.token_logprob(st["z"], st["x"], st["ws"], active=st["active"])
        if c["kind"] == "logprob":
            return [lp, H, status]
        return [lp, H, status, am.token_logprob_grad(st["z"], st["x"], st["ws"], st["dlp"], st["dH"], active=st["active"])]
    if c["kind"] == "policy":
        o = am.policy_loss(st["z"], st["x"], st["adv"], st["ws"], weight=st["weight"], old_logprob=st["old"], ref_logprob=st["ref"],
                           ref_logits=st["zref"], grad_scale=st["scale"],
                           options=am.PolicyOptions(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, entropy_coef=c["entropy"],
                                                    kl_coef=0.0 if c["kl"] == "none" else KL_COEF))
        return [o.loss, o.token_loss, o.logprob, o.entropy, o.kl, o.status, o.dlogits]
    o = am.preference_loss(st["z"], st["x"], st["ws"], weight=st["weight"], ref_logprob=st["ref"],
                           options=am.PreferenceOptions(kind=c["loss"], beta=BETA,
                                                        label_smoothing=SMOOTHING if c["loss"] == "logistic" else 0.0))
    return [o.loss, o.pair_loss, o.margin, o.score, o.logprob, o.status, o.dlogits]


def work(case):
    """Rows that count are read once; every row of a gradient is written once (zeros where a position does not count)."""
    c = case
    row, n, rows = c["V"] * _SIZE[c["dtype"]], _rows_counted(c), c["B"] * c["T"]
    full = c["kind"] == "policy" and c["kl"] == "full"
    if c["kind"] == "logprob":
        return {"bytes": n * row + 17.0 * rows, "flops": 8.0 * n * c["V"]}
    # forward: scale and shift, exponential, two sums (maximum aside); backward: scale and shift, exponential, product and what is added
    return {"bytes": (2 if full else 1) * n * row + rows * row + 40.0 * rows, "flops": (26.0 if full else 13.0) * n * c["V"]}


# ---- in 64 bits, by differentiation ----------------------------------------------------------------------------------------------

def exact(case, seed):
    c, st = case, prepare(case, seed)
    z, x = st["z"], st["x"].long()
    B, T, V = z.shape
    f64 = dict(dtype=torch.float64, device=z.device)
    step = max(1, (1 << 26) // V)

    def chunks():
        for b in range(B):
            for t in range(0, T, step):
                yield b, slice(t, min(T, t + step))

    def logs(b, t, grad=False):
        r = z[b, t].double().requires_grad_(grad)
        return r, torch.log_softmax(r, -1)

    def entropy(l):
        return -(l.exp() * l.clamp_min(-1e5)).sum(-1)

    pick = lambda l, b, t: l.gather(1, x[b, t][:, None])[:, 0]  # noqa: E731
    if c["kind"] in ("logprob", "logprob_grad"):
        on = torch.ones(B, T, **f64) if st["active"] is None else st["active"].double()
        lp, H, g = torch.zeros(B, T, **f64), torch.zeros(B, T, **f64), None
        grad = c["kind"] == "logprob_grad"
        if grad:
            g = torch.zeros(B, T, V, **f64)
        for b, t in chunks():
            r, l = logs(b, t, grad)
            p, h = pick(l, b, t), entropy(l)
            if grad:
                (on[b, t] * (st["dlp"][b, t].double() * p + st["dH"][b, t].double() * h)).sum().backward()
                g[b, t] = r.grad
            lp[b, t], H[b, t] = p.detach() * on[b, t], h.detach() * on[b, t]
        return [lp, H, None] + ([g] if grad else [])
    w = st["weight"].double()
    on = (w != 0).double()
    g, lp = torch.zeros(B, T, V, **f64), torch.zeros(B, T, **f64)
    if c["kind"] == "policy":
        A = st["adv"].double()
        A = A[:, None].expand(B, T) if A.dim() == 1 else A
        scale = 1.0 if st["scale"] is None else st["scale"].double()
        tok, H, KL = (torch.zeros(B, T, **f64) for _ in range(3))
        for b, t in chunks():
            r, l = logs(b, t, True)
            p, h = pick(l, b, t), entropy(l)
            ratio = torch.exp(p - st["old"][b, t].double())
            L = -torch.minimum(ratio * A[b, t], torch.clamp(ratio, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * A[b, t])
            k = torch.zeros_like(p)
            if c["kl"] == "sampled":
                delta = st["ref"][b, t].double() - p
                k = torch.expm1(delta) - delta
            if c["kl"] == "full":
                k = (l.exp() * (l - torch.log_softmax(st["zref"][b, t].double(), -1))).sum(-1)
            L = L + KL_COEF * k - c["entropy"] * h
            (scale * w[b, t] * L).sum().backward()
            g[b, t] = r.grad
            tok[b, t], lp[b, t], H[b, t], KL[b, t] = (v.detach() * on[b, t] for v in (L, p, h, k))
        return [(w * tok).sum(), tok, lp, H, KL, None, g]
    P = B // 2
    for b, t in chunks():
        lp[b, t] = pick(logs(b, t)[1], b, t)
    score = (w * (lp - st["ref"].double())).sum(1).requires_grad_(True)
    m = score[:P] - score[P:]
    if c["loss"] == "squared":
        pair = (m - 0.5 / BETA) ** 2
    elif c["loss"] == "hinge":
        m = BETA * m
        pair = torch.relu(1.0 - m)
    else:
        m = BETA * m
        ls = torch.nn.functional.logsigmoid
        pair = -(1.0 - SMOOTHING) * ls(m) - SMOOTHING * ls(-m)
    pair.mean().backward()
    for b, t in chunks():
        r, l = logs(b, t, True)
        (score.grad[b] * w[b, t] * pick(l, b, t)).sum().backward()
        g[b, t] = r.grad
    return [pair.mean().detach(), pair.detach(), m.detach(), score.detach(), lp * on, None, g]
