"""Attention over the paged cache where most of a row's weight lies on tokens whose values are zero (the first token of
many models): what is left of o comes from weights that are tiny beside the largest one, and has to be as exact as any
other o."""
import math

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

FAR = 2.0 ** -16


def scored(qs, kind, dtype, lens, score, Hq=8, Hkv=2, d=64, value=1.0, page=32, seed=0):
    """A batch whose scores are score(r, n) and whose values are `value` (1 + noise / 4), zero where the score is above 4."""
    e4m3, latent = kind == "e4m3", kind == "latent"
    if latent:
        b = ref.Batch(qs, lens, Hq, 1, 192, 128, page=page, latent=True, dtype=dtype, scale=1.0, seed=seed)
    else:
        b = ref.Batch(qs, lens, Hq, Hkv, d, page=page, dtype=dtype, e4m3=e4m3, scale=1.0, seed=seed)
    at = b.cfg.dk - 1   # the entry that makes the score; no value of a latent
    b.qval.zero_()
    b.qval[..., at] = 1.0
    b.q.copy_(b.qval)
    g = torch.Generator().manual_seed(seed + 1)
    k, kv = b.k.float().cpu(), b.kval.clone()
    v, vv = (k, kv) if latent else (b.v.float().cpu(), b.vval.clone())
    kx, vx = (b.cache.k_exp.cpu(), b.cache.v_exp.cpu()) if e4m3 else (None, None)
    for r, n in enumerate(lens):
        t = torch.arange(n)
        ids, row = torch.tensor(b.table[r], dtype=torch.long)[t // page], t % page
        x = score(r, n)
        val = value * (1 + 0.25 * torch.randn(n, b.cfg.Hkv, b.cfg.dv, generator=g))
        val[x > 4] = 0
        key = torch.zeros(n, b.cfg.Hkv, b.cfg.dk)
        key[..., at] = x[:, None]
        if latent:
            key[..., : b.cfg.dv] = val
        if e4m3:
            for y, codes, exps, out in ((key, k, kx, kv), (val, v, vx, vv)):
                c, e = ref.quantise(y.to(torch.bfloat16))
                codes[ids, :, row], exps[ids, :, row] = c.float(), e
                out[ids, :, row] = c * torch.exp2(e.double() - 127)[..., None]
        else:
            for y, codes, out in ((key, k, kv), (val, v, vv)) if not latent else ((key, k, kv),):
                codes[ids, :, row] = y
                out[ids, :, row] = y.to(b.t).double()
    b.k.copy_(k.to(b.k.dtype))
    if not latent:
        b.v.copy_(v.to(b.v.dtype))
    if e4m3:
        b.cache.k_exp.copy_(kx), b.cache.v_exp.copy_(vx)
    b.kval, b.vval = kv, vv[..., : b.cfg.dv]
    return b


def check(qs, b, kind, dtype):
    """Bounds, first order.  Output: half a unit in the last place.  A weight: rounded to 16 bits twice with its normalisation
    (f16, or bf16 for latents of that type), its exponential and rescalings (2^-17), the sums of n.  f16 ends 2^-25 under
    1; the reference stays near the largest weight of the 16 (latents: 64) tokens that are worked together, so that a
    weight loses at most 2^-16 of that largest one, and never more than itself."""
    qs.qstate_check()
    c, blk = b.cfg, 64 if kind == "latent" else 16
    u_out = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    u_p = 2.0 ** -8 if kind == "latent" and dtype == "bf16" else 2.0 ** -11
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -120
    got, gl = b.o.double().cpu(), b.lse.double().cpu()
    for r, n in enumerate(b.lens):
        t = torch.arange(n)
        ids = torch.tensor(b.table[r], dtype=torch.long)[t // c.page]
        K, V = b.kval[ids, :, t % c.page], b.vval[ids, :, t % c.page]
        z = torch.einsum("hgd,nhd->hgn", b.qval[r].double().view(c.Hkv, -1, c.dk), K)
        lse = torch.logsumexp(z, -1, keepdim=True)
        w = torch.exp(z - lse)
        o = torch.einsum("hgn,nhd->hgd", w, V)
        # the powers of values count towards the largest weight of an e4m3 cache; zero vectors do not
        size = V.abs().amax(-1).T[:, None] if kind == "e4m3" else torch.ones(1, 1, n, dtype=torch.float64)
        top = torch.nn.functional.pad(w * size, (0, -n % blk)).view(*w.shape[:2], -1, blk).amax(-1).repeat_interleave(blk, -1)[..., :n]
        far = torch.minimum(w, FAR * 2 * top / size.clamp(min=1e-300))
        loss = torch.einsum("hgn,nhd->hgd", w * (2 * u_p + 2.0 ** -17 + n * 2.0 ** -24) + far, V.abs())
        bound = (u_out * o.abs() + loss + tiny).flatten(0, 1)
        err = (got[r] - o.flatten(0, 1)).abs()
        assert bool((err <= bound).all()), f"request {r} of {n}: {float((err / bound).max()):.3g} bounds, o {float(o.abs().max()):.3g}"
        lse = lse.reshape(-1)
        assert bool(((gl[r] - lse).abs() <= 2.0 ** -19 + n * 2.0 ** -24 + lse.abs() * 2.0 ** -22).all())


KINDS = [("heads", "bf16"), ("heads", "f16"), ("e4m3", "bf16"), ("latent", "bf16"), ("latent", "f16")]
LENS = [6000 - 37 * r for r in range(40)]   # some tens of tiles a CTA


def sink(place, above):
    def score(r, n):
        x = 0.5 * torch.sin(torch.arange(n) * 1.7 + r)
        x[{"first": 0, "middle": n // 2, "last": n - 1}[place]] = above
        return x
    return score


@pytest.mark.parametrize("above", [9.0, 17.0, 17.375, 24.0, 36.0])
@pytest.mark.parametrize("place", ["first", "middle", "last"])
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_a_sink_without_a_value(qs, kind, dtype, place, above):
    # f16 holds o itself down to 2^-24: its values are larger where little of them is left
    value = 1.0 if dtype == "bf16" or above < 20 else 8192.0
    b = scored(qs, kind, dtype, LENS, sink(place, above), value=value, seed=int(above))
    b.run(qs)
    check(qs, b, kind, dtype)


@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (10, 1, 128), (16, 1, 256), (40, 2, 64)])
@pytest.mark.parametrize("kind,dtype", [("heads", "f16"), ("e4m3", "bf16")])
def test_a_sink_without_a_value_for_other_heads(qs, kind, dtype, Hq, Hkv, d):
    b = scored(qs, kind, dtype, LENS[:20] + [70, 33, 2], sink("first", 19.0), Hq=Hq, Hkv=Hkv, d=d, seed=d)
    b.run(qs)
    check(qs, b, kind, dtype)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_scores_that_fall_by_hundreds_after_a_sink(qs, kind, dtype):
    """A row whose weights fall without end: the reference does not follow for ever, and nothing overflows."""
    def score(r, n):
        x = -torch.arange(n) * (0.0625 * (1 + r % 3))
        x[0] = 30.0
        return x.clamp(min=-440.0)
    b = scored(qs, kind, dtype, LENS, score, value=64.0)
    b.run(qs)
    check(qs, b, kind, dtype)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_many_sinks_without_values(qs, kind, dtype):
    """Every 200th token: the reference goes up and down all along a row."""
    def score(r, n):
        x = 0.5 * torch.sin(torch.arange(n) * 1.7 + r)
        x[r % 200::200] = 20.0
        return x
    b = scored(qs, kind, dtype, LENS, score, value=1.0 if dtype == "bf16" else 512.0)
    b.run(qs)
    check(qs, b, kind, dtype)


@pytest.mark.parametrize("value", [2.0 ** -60, 2.0 ** -20, 2.0 ** -9, 180.0])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 64, 32), (10, 1, 128, 8), (4, 2, 256, 64), (24, 2, 128, 1)])
def test_vectors_of_zeros_among_values_of_any_size(qs, Hq, Hkv, d, page, value):
    """A vector of zeros has the power 2^0 in an e4m3 cache, however small the others' are."""
    def score(r, n):
        x = 0.5 * torch.sin(torch.arange(n) * 1.7 + r)
        x[r % 7::7] = 4.5
        return x
    b = scored(qs, "e4m3", "bf16", [900 - 11 * r for r in range(30)] + [1, 2, 33], score, Hq=Hq, Hkv=Hkv, d=d, page=page, value=value)
    b.run(qs)
    check(qs, b, "e4m3", "bf16")
