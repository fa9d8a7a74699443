"""Keys, values and weights at the ends of their types' ranges among the tokens that a group shares, against plain attention in 64 bits."""
import pytest
import torch

import kv_reference as ref
import kv_share_reference as share

pytestmark = pytest.mark.gpu

LENS = [300, 300, 311, 302]
COMMON = 290
TOP = 255.0 * 2.0 ** 120   # the largest bf16; e4m3 rounds it to 2^128


@pytest.fixture(autouse=True)
def share_everything(qs):
    """Groups share whatever it costs: the cases here are small."""
    qs.qstate_set_shared_gain(0)
    yield
    qs.qstate_set_shared_gain(-1)


def codes_batch(qs, K, V, q, d, scale):
    """A batch of e4m3 whose token t has keys K[t] and values V[t] (64 bits, rounded to bf16 by their maker) in every request, and
    whose queries are all q."""
    b = share.Batch(qs, LENS, [(0, len(LENS), COMMON)], 4, 1, d, e4m3=True, scale=scale, seed=1)
    at = [(b.table[r][t // 16], t % 16, t) for r, n in enumerate(LENS) for t in range(n)]
    page, place, token = (torch.tensor(x) for x in zip(*at))
    for x, codes, exps, val in ((K, b.k, b.cache.k_exp, b.kval), (V, b.v, b.cache.v_exp, b.vval)):
        y, e = ref.quantise(x)
        raw, many = codes.view(torch.uint8).cpu(), exps.cpu()
        raw[page, 0, place] = y.float().to(torch.float8_e4m3fn).view(torch.uint8)[token]
        many[page, 0, place] = e[token]
        codes.view(torch.uint8).copy_(raw)
        exps.copy_(many)
        val[page, 0, place] = (y * torch.ldexp(torch.ones_like(y), e[:, None].int() - 127))[token]
    b.qval[:] = q.to(torch.bfloat16)
    b.q.copy_(b.qval)
    return b


def compare(qs, b, o_more, lse_more):
    """Within the bounds of ordinary numbers and these beside them."""
    b.run(qs)
    qs.qstate_check()
    o, lse, do, dl = b.expect()
    got, gl = b.o.double().cpu(), b.lse.double().cpu()
    assert bool(((got - o).abs() <= do + o_more).all()), float((got - o).abs().max())
    assert bool(((gl - lse).abs() <= dl + lse_more).all()), float((gl - lse).abs().max())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_largest_keys_of_e4m3(qs, d):
    """2^128 is no bf16: shared keys there are 2^-8 less, so scores of up to 2 are off by 2^-7, weights by twice that."""
    g = torch.Generator().manual_seed(d)
    K = torch.zeros(max(LENS), d, dtype=torch.float64)
    sign = torch.randint(0, 2, (max(LENS),), generator=g) * 2 - 1
    K[:, 0] = torch.where(torch.rand(max(LENS), generator=g) < 0.5, TOP, 2.0 ** 127) * sign
    V = torch.randn(max(LENS), d, generator=g, dtype=torch.float64).to(torch.bfloat16).double()
    q = torch.zeros(d)
    q[0] = 2.0 ** -125
    b = codes_batch(qs, K, V, q, d, 0.25)
    assert bool((b.cache.k_exp[b.table[0][0]] == 247).any())
    w_most = float(V.abs().max())
    compare(qs, b, 2.0 ** -6 * w_most, 2.0 ** -7)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_largest_values_of_e4m3(qs, d):
    """A token of small weight with the largest values: its product is finite, and 2^-8 less where values are 2^128."""
    g = torch.Generator().manual_seed(d)
    K = torch.zeros(max(LENS), d, dtype=torch.float64)
    far = 77
    K[far, 0] = -20.0
    V = torch.randn(max(LENS), d, generator=g, dtype=torch.float64).to(torch.bfloat16).double()
    V[far] = TOP * (torch.randint(0, 2, (d,), generator=g) * 2 - 1)
    q = torch.zeros(d)
    q[0] = 1.0
    b = codes_batch(qs, K, V, q, d, 1.0)
    assert int(b.cache.v_exp[b.table[0][far // 16], 0, far % 16]) == 247
    # the token's weight, under e^-20 / 290, times 2^128 times 2^-8
    compare(qs, b, 2.0 ** 128 * 2.0 ** -28.8 / 290 * 2.0 ** -8, 0.0)


def test_the_smallest_keys_of_e4m3(qs):
    """At the lowest power, 2^-126, codes under 2^-7 are no multiples of bf16's last step, 2^-133: a key's entry is off by up to 2^-134,
    four of them times queries of 2^126 a score by 2^-6, and a weight by twice that."""
    d = 128
    g = torch.Generator().manual_seed(2)
    K = torch.zeros(max(LENS), d, dtype=torch.float64)
    K[:, :4] = (torch.randn(max(LENS), 4, generator=g, dtype=torch.float64) * 2.0 ** -126).to(torch.bfloat16).double()
    V = torch.randn(max(LENS), d, generator=g, dtype=torch.float64).to(torch.bfloat16).double()
    q = torch.zeros(d)
    q[:4] = 2.0 ** 126
    b = codes_batch(qs, K, V, q, d, 1.0)
    assert bool((b.cache.k_exp[b.table[0][0]] == 1).all())
    compare(qs, b, 2.0 ** -5 * float(V.abs().max()), 2.0 ** -6)


@pytest.mark.parametrize("power", [-100, -126])
def test_the_smallest_values_of_e4m3(qs, power):
    """Products of weights and values are FP32, under whose normal numbers a result may be taken as nothing: each of n products
    and of n sums of them loses up to 2^-126, against weights p = 2^(z - m) of which the largest is 1 or more, so o loses up to
    2 n 2^-126 / sum_t e^(z_t - max z).  At 2^-100 that is nothing beside the rounding of o; at 2^-126, where a value has half a step of
    2^-133 less beside it, it is more than o, which has to be finite and no larger."""
    d = 128
    g = torch.Generator().manual_seed(3)
    K = torch.randn(max(LENS), d, generator=g, dtype=torch.float64).to(torch.bfloat16).double()
    V = (torch.randn(max(LENS), d, generator=g, dtype=torch.float64) * 2.0 ** power).to(torch.bfloat16).double()
    b = codes_batch(qs, K, V, torch.randn(d, generator=g), d, d ** -0.5)
    b.run(qs)
    qs.qstate_check()
    b.vval = b.vval * 2.0 ** -power   # the bound's steps are those of numbers about one
    o, lse, do, dl = b.expect()
    lost = torch.zeros(len(LENS), 4, 1, dtype=torch.float64)
    for r, n in enumerate(LENS):
        y, e = ref.quantise(K[:n])
        z = y * torch.exp2(e.double() - 127)[:, None] @ b.qval[r].double().cpu().T * d ** -0.5
        lost[r, :, 0] = 2 * n * 2.0 ** (-126 - power) / torch.exp(z - z.amax(0)).sum(0)
    assert bool(((b.o.double().cpu() * 2.0 ** -power - o).abs() <= do + lost + 2.0 ** (-133 - power)).all())
    assert bool(((b.lse.double().cpu() - lse).abs() <= dl).all())


@pytest.mark.parametrize("first", [0, 5, 69, 3839])
def test_small_weights_behind_and_before_large_ones_in_f16(qs, first):
    """Every 60th tile has a token whose score is 20.58 above all others' and whose value is zero: the answer is what the others make
    of it, 0.03 or so.  Beside the large one, whose weight is 2^7, theirs are 2.48 steps of 2^-24, the last that f16 has.  In a tile with a
    large one they are off by up to half a step, a fifth of them; in all others the reference is theirs, and they are off by 2^-11 at
    most.  (Were it the large one's, they would be 2 steps, a fifth less, in a fourth of all tiles or more: a worker goes through about 60
    tiles, in two streams; against 2^7 less they would be nothing.)"""
    n, Hkv, d, gap = 60 * 64 * 9 + 1920, 16, 64, 20.578125
    b = share.Batch(qs, [n, n + 9], [(0, 2, n)], Hkv, Hkv, d, page=64, dtype="f16", scale=1.0, seed=4)
    b.qval.zero_()
    b.qval[..., 0] = 1.0
    b.q.copy_(b.qval)
    large = list(range(first, n, 60 * 64))
    for k, v in ((b.k, b.v), (b.kval, b.vval)):
        k[..., 0] = 0.0
        v.abs_().mul_(2.0 ** 13)
        for r in range(2):
            for t in large:
                k[b.table[r][t // 64], :, t % 64, 0] = gap
                v[b.table[r][t // 64], :, t % 64] = 0.0
    b.run(qs)
    qs.qstate_check()
    o, lse, _, dl = b.expect()
    tiles = {t // 64 for t in large}
    small = torch.exp(torch.tensor(-gap, dtype=torch.float64)) / len(large)   # a weight, but for 1e-4 of it
    for r in range(2):
        pages = torch.tensor(b.table[r][: -(-n // 64)])
        V = torch.nan_to_num(b.vval[pages])                                  # (tiles, Hkv, 64, d); places behind the last token are NaN
        beside = small * V[sorted(tiles)].sum((0, 2)).cpu()
        # half a step; a weight's rounding, the sum's and o's, 2^-11 each; scores of 30 in base 2 and sums of 570 parts in FP32
        bound = beside * (0.5 / 2.48) + o[r] * (3 * 2.0 ** -11 + 2.0 ** -17) + 2.0 ** -25
        assert bool((o[r] > 0.01).all()) and bool((bound < 0.02 * o[r]).all())
        assert bool(((b.o[r].double().cpu() - o[r]).abs() <= bound).all()), float(((b.o[r].double().cpu() - o[r]) / o[r]).abs().max())
    assert bool(((b.lse.double().cpu() - lse).abs() <= dl).all())
