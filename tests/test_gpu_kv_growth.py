"""Attention over the paged cache where scores outgrow the running reference while a CTA is under way: in every kind of
tile of a row (the last one among them), with rows of two to five tiles taken whole and with long shares of split rows.
Against plain attention in 64 bits, and bit for bit from run to run."""
import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu


def set_scores(qs, b, score):
    """Makes score(r, n), a tensor of n scores of request r, the scores of b (scale 1) up to what the random rest of keys and
    queries adds (nothing in e4m3)."""
    e4m3 = b.cfg.store == qs.KV_E4M3
    b.qval[..., 1:] *= 0.0 if e4m3 else 0.02
    b.qval[..., 0] = 1.0
    b.q.copy_(b.qval)
    k = b.k.float().cpu()
    if e4m3:
        b.cache.k_exp.fill_(127)
    for r, n in enumerate(b.lens):
        if n:
            t = torch.arange(n)
            ids = torch.tensor(b.table[r], dtype=torch.long)[t // b.cfg.page]
            k[ids, :, t % b.cfg.page, 0] = score(r, n)[:, None]
    b.k.copy_(k.to(b.k.dtype))
    b.kval = b.k.float().cpu().double()
    if b.v is None:
        b.vval = b.kval[..., : b.cfg.dv]


def spike(where):
    """Scores about 0 and one that is 6.5 above (2^9.4), in the row's last tile or in one of its tiles."""
    def score(r, n):
        x = 0.25 * ((torch.arange(n) * 7 + r) % 5).float()
        first = (n - 1) // 64 * 64 if where == "last" else r % ((n + 63) // 64) * 64
        x[first + (5 * r) % min(64, n - first)] = 6.5
        return x
    return score


def stairs(r, n):
    """Seven more from tile to tile, up to 224."""
    return 7.0 * ((torch.arange(n) // 64).clamp(max=32)).float()


SCORES = {"last": spike("last"), "any": spike("any"), "stairs": stairs}


def check(qs, b):
    """Twice the bound of o that the reference gives: half a unit in the last place is up to 2^-8 of a bf16 value
    and 2^-11 of an f16 one, where it counts half of that, and a few equal scores may all be rounded the same way."""
    qs.qstate_check()
    o, lse, do, dl = b.expect()
    assert bool(((b.o.double().cpu() - o).abs() <= 2 * do).all())
    assert bool(((b.lse.double().cpu() - lse).abs() <= dl).all())


def repeated(qs, b, times=5):
    b.run(qs)
    check(qs, b)
    o, lse = b.o.clone(), b.lse.clone()
    for _ in range(times):
        b.o.fill_(9.0)
        b.run(qs)
        assert torch.equal(b.o.view(torch.int16), o.view(torch.int16)) and torch.equal(b.lse, lse)


@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (320, 256), (576, 512)])
@pytest.mark.parametrize("Hq", [5, 16, 32, 64])
def test_latents_of_rows_taken_whole(qs, Hq, dk, dv, dtype, scores):
    lens = [65 + (37 * r) % 176 for r in range(170)]
    b = ref.Batch(qs, lens, Hq, 1, dk, dv, page=16, latent=True, dtype=dtype, scale=1.0, seed=Hq)
    set_scores(qs, b, SCORES[scores])
    repeated(qs, b)


@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("f16", 32)])
@pytest.mark.parametrize("Hq,dk,dv", [(16, 128, 128), (64, 192, 128), (64, 320, 256), (30, 512, 512)])
def test_latents_of_long_shares(qs, Hq, dk, dv, dtype, page, scores):
    lens = [200 + (911 * r) % 2600 for r in range(60)]   # some four tiles a CTA
    b = ref.Batch(qs, lens, Hq, 1, dk, dv, page=page, latent=True, dtype=dtype, scale=1.0, seed=Hq)
    set_scores(qs, b, SCORES[scores])
    repeated(qs, b)


@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(6, 2), (20, 2)])
def test_heads_of_rows_taken_whole(qs, Hq, Hkv, d, dtype, e4m3, scores):
    lens = [65 + (37 * r) % 176 for r in range(170)]
    b = ref.Batch(qs, lens, Hq, Hkv, d, page=16, dtype=dtype, e4m3=e4m3, scale=1.0, seed=d)
    set_scores(qs, b, SCORES[scores])
    repeated(qs, b)


@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads_of_long_shares(qs, d, dtype, e4m3, scores):
    lens = [200 + (911 * r) % 2600 for r in range(60)]
    b = ref.Batch(qs, lens, 16, 4, d, page=32, dtype=dtype, e4m3=e4m3, scale=1.0, seed=d)
    set_scores(qs, b, SCORES[scores])
    repeated(qs, b)
