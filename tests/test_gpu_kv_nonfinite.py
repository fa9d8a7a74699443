"""Numbers that are not finite in the paged cache, in every kind of layer: they reach the heads and requests that see them, and
no others; scores of minus infinity weigh nothing."""
import math

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

LENS = [40, 700, 300, 200, 5]


def batch(qs, kind, dtype):
    if kind == "latent":
        return ref.Batch(qs, LENS, 20, 1, 192, 128, page=16, latent=True, dtype=dtype, seed=4)
    return ref.Batch(qs, LENS, 12, 2, 64, page=16, dtype=dtype, e4m3=kind == "e4m3", seed=4)


def others_stand(b, hit):
    """o and lse of all rows but those that `hit` names (request, first head, end) are within their bounds."""
    o, lse, do, dl = b.expect()
    got, gl = b.o.double().cpu(), b.lse.double().cpu()
    keep = torch.ones(got.shape[:2], dtype=torch.bool)
    for r, h0, h1 in hit:
        keep[r, h0:h1] = False
    assert bool(((got - o).abs() <= 2 * do)[keep].all()) and bool(((gl - lse).abs() <= dl)[keep].all())


@pytest.mark.parametrize("kind,dtype", [("heads", "bf16"), ("heads", "f16"), ("e4m3", "bf16"), ("latent", "bf16"), ("latent", "f16")])
def test_what_is_not_finite_stays_where_it_is_seen(qs, kind, dtype):
    b = batch(qs, kind, dtype)
    at = lambda r, t: (b.table[r][t // 16], slice(None) if kind == "latent" else 1, t % 16)  # noqa: E731
    whole = 20 if kind == "latent" else 12
    first = 0 if kind == "latent" else 6
    for r, t in ((0, 3), (1, 0), (2, 299)):   # keys: a whole head's scores
        if kind == "e4m3":
            b.cache.k_exp[at(r, t)] = 255
        else:
            b.k[at(r, t) + (b.cfg.dk - 1,)] = float("nan" if r else "inf")
    if kind == "e4m3":
        b.cache.v_exp[at(3, 100)] = 255
    elif kind == "heads":
        b.v[at(3, 100)] = float("nan")
    b.run(qs)
    qs.qstate_check()
    hit = [(0, first, whole), (1, first, whole), (2, first, whole)] + ([] if kind == "latent" else [(3, first, whole)])
    o = b.o.float().cpu()
    for r, h0, h1 in hit[1:]:
        assert bool(torch.isnan(o[r, h0:h1]).all())
    # infinity times the sign of q: a head whose score is +inf has no answer, one whose score is -inf loses a token
    if kind != "e4m3":
        up = b.qval[0, first:whole, -1] > 0
        assert bool(torch.isnan(o[0, first:whole][up]).all()) and bool(torch.isfinite(o[0, first:whole, : b.cfg.dv - 1][~up]).all())
    others_stand(b, hit)


@pytest.mark.parametrize("kind,dtype", [("heads", "bf16"), ("heads", "f16"), ("latent", "f16")])
@pytest.mark.parametrize("place", ["all", "first", "last"])
def test_scores_of_minus_infinity_weigh_nothing(qs, kind, dtype, place):
    """A key entry of minus infinity against queries over zero there: its token is as if it were not in the cache."""
    b = batch(qs, kind, dtype)
    at = b.cfg.dk - 1   # no value of a latent
    b.qval[..., at] = 1.0
    b.q.copy_(b.qval)
    for r, n in enumerate(LENS):
        gone = {"all": range(n), "first": range(n - n // 3), "last": range(n // 3, n)}[place]
        for t in gone:
            b.k[b.table[r][t // 16], :, t % 16, at] = -math.inf
            b.kval[b.table[r][t // 16], :, t % 16, at] = -1e6
    if kind == "latent":
        b.vval = b.kval[..., : b.cfg.dv]
    b.run(qs)
    qs.qstate_check()
    if place == "all":
        assert not bool(b.o.any()) and bool((b.lse == -math.inf).all())
        return
    others_stand(b, [(4, 0, 20)])   # five tokens: a third of them leaves one
    assert bool(torch.isfinite(b.o.float()).all())
