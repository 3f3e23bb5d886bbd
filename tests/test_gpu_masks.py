"""Rows masked with finite values in the drafting and verification calls: whole stretches of the vocabulary at one value give, bit for bit, what
-inf gives there."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
MASKS = {BF: [-1e4, -5e8, -8e8, -1e9, -1.2e9, -1e10, -3e12, -1e30, -2.5e36, -5e36, -9e36, -2e37, -1e38, -2e38, torch.finfo(BF).min],
         F: [-1e4, -5e8, -8e8, -1e9, -1.2e9, -1e10, -3e12, -1e30, -1e37, -1e38, -2e38, torch.finfo(F).min]}


@pytest.fixture(scope="module")
def am():
    import paper_2512_11280_amd as am
    am.load_library()
    return am


def _rows(B, K, V, dtype, seed):
    """Draft and target logits, and the stretch that is masked in all of them."""
    g = torch.Generator().manual_seed(seed)
    q = 3.0 * torch.randn(B, K, V, generator=g)
    p = torch.cat([q + 0.7 * torch.randn(B, K, V, generator=g), 3.0 * torch.randn(B, 1, V, generator=g)], 1)
    at = torch.zeros(V, dtype=torch.bool)
    at[V // 5:V // 5 + V // 2] = True
    at[1::7] = True
    return p.to(dtype), q.to(dtype), at


@pytest.mark.parametrize("stats_path", [0, 1, 2])
@pytest.mark.parametrize("dtype, mask", [(d, m) for d in (BF, F) for m in MASKS[d]])
def test_masks_of_any_size(am, mask, dtype, stats_path):
    for B, K, V in ((1, 8, 128256), (3, 5, 9001), (32, 8, 4003), (2, 2, 64)):
        p, q, at = _rows(B, K, V, dtype, 5)

        def call(value):
            z, d = p.clone(), q.clone()
            z[..., at] = value
            d[..., at] = value
            z, d = z.cuda(), d.cuda()
            ws, state = am.Workspace(B, K, V, dtype), am.State(B, 64)
            out = list(am.draft_entropy(d[:, 0], ws))
            steps = [am.draft_step(d[:, i], ws, step=i, k_max=20, seed=7) for i in range(K)]
            out += [t for s in steps for t in s]
            x = torch.stack([s[2] for s in steps], 1).contiguous()
            r = am.verify(z, d, x, ws, state=state, seed=7, options=am.Options(stats_path=stats_path, apply_update=1))
            return out + [r.n_accept, r.next_token, r.H_p, r.H_q, r.d_js, r.accept_mask, r.status, state.ent_sum, state.nA, state.nR]
        want, got = call(-math.inf), call(mask)
        for k, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (B, K, V, k, a.flatten()[:4].tolist(), b.flatten()[:4].tolist())


@pytest.mark.parametrize("stats_path", [0, 1, 2])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("value", [-1e4, -1e6, -1e9])
def test_rows_that_are_masked_throughout(am, value, dtype, stats_path):
    """Every logit the same, however low: a flat row.  The entropy is ln V to 1e-5 of it, and so is the normaliser above the logits.  Rows that start
    elsewhere in a vector are added up in another order, so that two normalisers may differ by delta, |delta| <= 2e-5 ln V / ln 2 in units of log2; the
    distance that follows is sqrt(delta^2 / 4) (the terms' series, stats_device.h), no more than half of that."""
    for B, K, V in ((1, 8, 128256), (3, 5, 9001), (2, 2, 64)):
        z, d = torch.full((B, K + 1, V), value, dtype=dtype, device="cuda"), torch.full((B, K, V), value, dtype=dtype, device="cuda")
        ws = am.Workspace(B, K, V, dtype)
        H, _, x, status = am.draft_step(d[:, 0], ws, step=0, k_max=20, seed=7)
        assert (H - math.log(V)).abs().max() < 1e-5 * math.log(V) and not (status & 2).any()
        x = x[:, None].expand(B, K).contiguous()
        r = am.verify(z, d, x, ws, seed=7, options=am.Options(stats_path=stats_path))
        assert (r.H_p - math.log(V)).abs().max() < 1e-5 * math.log(V) and not (r.status & 2).any()
        assert (r.d_js >= 0).all() and r.d_js.max() <= 1e-5 * math.log(V) / math.log(2)


@pytest.mark.parametrize("dtype, mask", [(d, m) for d in (BF, F) for m in MASKS[d]])
def test_column_shards_that_are_masked(am, mask, dtype):
    """The same where whole column slices hold nothing but masked logits: the statistics of every position (what is accepted may differ: a drafted
    token masked in both rows has the ratio 0 / 0 with -inf and that of two numbers otherwise), and no row is broken."""
    from paper_2512_11280_amd import workloads as wl
    from test_gpu_parity import _sharded_decisions, _sharded_tokens
    got = []
    for value in (-math.inf, mask):
        batch = wl.config_batched(B=3, k=4, V=9000, dtype=dtype, seed=11, cap=96)
        batch.target[..., 2000:7000] = value
        batch.draft[..., 2000:7000] = value
        ctx = _sharded_decisions(am, batch, 5, options=am.Options(apply_update=1))
        _sharded_tokens(am, batch, ctx, ctx[0])
        got.append(ctx[0])
    for a, b in zip(*got):
        assert all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("H_p", "H_q", "d_js"))
        assert not (b.status & 2).any() and (b.next_token >= 0).all()
