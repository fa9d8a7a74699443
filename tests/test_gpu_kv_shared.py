"""Attention over tokens that groups of requests share, against plain attention in 64 bits."""
import math

import pytest
import torch

import kv_share_reference as share

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def share_everything(qs):
    """Groups share whatever it costs: the cases here are small."""
    qs.qstate_set_shared_gain(0)
    yield
    qs.qstate_set_shared_gain(-1)

# groups of three and nine (one empty, one that lacks a common token), one request by itself before, between and behind
LENS = [70, 200, 205, 333, 1, 129, 128, 0, 400, 131, 129, 300, 900, 130, 55]
GROUPS = [(1, 4, 200), (5, 14, 129)]


def check(qs, b):
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
def test_types_and_widths(qs, d, kind):
    check(qs, share.Batch(qs, LENS, GROUPS, 12, 2, d, dtype="f16" if kind == "f16" else "bf16", e4m3=kind == "e4m3", seed=d))


@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 128, 1024])
def test_pages(qs, page):
    check(qs, share.Batch(qs, LENS, GROUPS, 8, 2, 128, page=page, seed=page))
    check(qs, share.Batch(qs, LENS, GROUPS, 4, 1, 64, page=page, e4m3=True, seed=page))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (7, 1), (12, 4), (40, 2), (64, 1), (130, 1)])
def test_head_layouts(qs, Hq, Hkv):
    check(qs, share.Batch(qs, LENS, GROUPS, Hq, Hkv, 64, seed=Hq))


@pytest.mark.parametrize("members,Hq,Hkv,d", [(2, 1, 1, 64), (16, 8, 1, 128), (17, 8, 1, 128), (32, 8, 1, 64), (33, 8, 1, 64), (90, 12, 2, 128),
                                            (16, 8, 1, 256), (17, 8, 1, 256), (50, 16, 2, 256)])
def test_blocks_of_rows(qs, members, Hq, Hkv, d):
    """Rows about the ends of blocks and of their halves."""
    check(qs, share.Batch(qs, [300 + 7 * i for i in range(members)], [(0, members, 290)], Hq, Hkv, d, seed=members))


@pytest.mark.parametrize("common", [1, 63, 64, 127, 128, 129, 255, 257, 1000])
@pytest.mark.parametrize("d", [128, 256])
def test_common_tokens_about_tiles(qs, common, d):
    check(qs, share.Batch(qs, [common + n for n in (0, 1, 2, 65, 130)], [(0, 5, common)], 4, 2, d, seed=common))


@pytest.mark.parametrize("d,members,Hq,Hkv", [(64, 19, 64, 4), (128, 19, 64, 4), (128, 33, 32, 8), (256, 21, 16, 2), (256, 16, 16, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "e4m3"])
def test_many_tiles_a_worker(qs, d, members, Hq, Hkv, dtype):
    """Workers that go through blocks of one half and of two, tile after tile."""
    lens, groups = [], []
    for common in (5000, 129, 7001):
        groups.append((len(lens), len(lens) + members, common))
        lens += [common + i for i in range(members)]
    check(qs, share.Batch(qs, lens, groups, Hq, Hkv, d, page=64, dtype="f16" if dtype == "f16" else "bf16", e4m3=dtype == "e4m3", seed=d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "e4m3"])
def test_one_long_group_in_many_parts(qs, dtype):
    check(qs, share.Batch(qs, [30000, 30011, 30500], [(0, 3, 30000)], 6, 1, 128, page=64, dtype="f16" if dtype == "f16" else "bf16",
                        e4m3=dtype == "e4m3", seed=1))


def test_many_small_groups(qs):
    lens, groups = [], []
    for g in range(300):
        groups.append((len(lens), len(lens) + 2, 40 + g % 100))
        lens += [40 + g % 100 + g % 3, 45 + g % 100]
    check(qs, share.Batch(qs, lens, groups, 4, 2, 64, page=8, seed=2))


@pytest.mark.parametrize("window", [1, 100, 200, 250, 10000])
def test_windows(qs, window):
    """Requests whose window begins behind token 0 read by themselves, beside others that share."""
    check(qs, share.Batch(qs, LENS, GROUPS, 8, 2, 64, window=window, seed=window))


def test_groups_of_which_one_or_nobody_shares(qs):
    check(qs, share.Batch(qs, [50, 40, 0, 0, 0, 70], [(0, 2, 45), (2, 5, 10), (5, 6, 70)], 4, 2, 64, seed=3))
    check(qs, share.Batch(qs, [0, 0, 0], [(0, 3, 5)], 4, 2, 64, seed=3))
    check(qs, share.Batch(qs, [33, 20], [], 4, 2, 64, seed=3))


def test_narrow_tables(qs):
    """Tables of so few tiles that a request's own tokens are never split."""
    check(qs, share.Batch(qs, [20, 25, 31, 22], [(0, 4, 19)], 4, 2, 128, seed=4))


def test_a_negative_scale_and_a_zero_one(qs):
    for scale in (-0.1, 0.0):
        check(qs, share.Batch(qs, LENS, GROUPS, 8, 2, 64, scale=scale, seed=5))
        check(qs, share.Batch(qs, LENS, GROUPS, 8, 2, 64, scale=scale, dtype="f16", seed=5))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_scores(qs, dtype):
    """The reference follows maxima that come late, in both kinds of tile order."""
    check(qs, share.Batch(qs, LENS, GROUPS, 8, 2, 64, spread=12.0, dtype=dtype, seed=6))


def test_queries_with_strides_and_off_16_bytes(qs):
    for d in (64, 256):
        b = share.Batch(qs, LENS, GROUPS, 6, 2, d, seed=7)
        wide = torch.zeros(len(LENS), 3, 6, d + 9, dtype=b.t, device="cuda")
        wide[:, 1, :, 3:3 + d] = b.q
        b.q = wide[:, 1, :, 3:3 + d]
        check(qs, b)


def test_the_same_answer_every_time(qs):
    b = share.Batch(qs, [5000, 5100, 5003, 5200], [(0, 4, 5000)], 8, 2, 128, seed=8)
    b.run(qs)
    first, lse = b.o.clone(), b.lse.clone()
    for _ in range(5):
        b.o.fill_(3)
        b.run(qs)
        assert torch.equal(b.o, first) and torch.equal(b.lse, lse)
    b.check(qs)


def test_without_lse(qs):
    b = share.Batch(qs, LENS, GROUPS, 8, 2, 128, seed=9)
    b.run(qs)
    want = b.o.clone()
    b.o.fill_(5)
    qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, b.d_groups, b.o, None, b.work)
    assert torch.equal(b.o, want)
    qs.qstate_check()


def test_groups_outside_their_bounds(qs):
    """Reported, and nothing is shared: the answers stand."""
    b = share.Batch(qs, LENS, GROUPS, 8, 2, 64, seed=10)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for start, common in ((i32(0, 9, 4), i32(50, 50)), (i32(-1, 4), i32(10)), (i32(0, 16), i32(10)),
                          (i32(1, 4), i32(-2)), (i32(1, 4), i32(2 ** 30))):
        b.start, b.common = start, common
        b.o.fill_(9)
        b.run(qs)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_EDEVICE
        b.check(qs)


def test_pages_outside_the_pool_among_the_common_tokens(qs):
    """Reported, and as if their tokens were not there, for every request that shares them."""
    b = share.Batch(qs, [300, 310, 305], [(0, 3, 256)], 4, 2, 64, seed=11)
    b.d_table[0, 3] = b.cfg.n_pages
    b.d_table[0, 8] = -1
    b.run(qs)
    with pytest.raises(qs.QstateError):
        qs.qstate_check()
    for r in range(3):
        b.table[r] = [x for c, x in enumerate(b.table[r]) if c not in (3, 8)]
    b.lens = [n - 32 for n in b.lens]
    b.check(qs)


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
def test_what_is_not_finite_stays_where_it_is_seen(qs, kind):
    lens = [300, 310, 305, 290, 80]
    b = share.Batch(qs, lens, [(0, 4, 280)], 12, 2, 64, dtype="f16" if kind == "f16" else "bf16", e4m3=kind == "e4m3", seed=12)
    at = lambda r, t, h: (b.table[r][t // 16], h, t % 16)  # noqa: E731
    if kind == "e4m3":
        b.cache.k_exp[at(0, 100, 1)] = 255
        b.cache.v_exp[at(2, 300, 0)] = 255
    else:
        b.k[at(0, 100, 1) + (7,)] = float("nan")
        b.v[at(2, 300, 0)] = float("nan")
    b.q[3, 2] = float("nan")   # one head of one request
    b.run(qs)
    qs.qstate_check()
    o, lse, do, dl = b.expect()
    got, gl = b.o.double().cpu(), b.lse.double().cpu()
    hit = torch.zeros(got.shape[:2], dtype=torch.bool)
    hit[:4, 6:] = True
    hit[2, :6] = True
    hit[3, 2] = True
    assert bool(torch.isnan(got[:4, 6:]).all()) and bool(torch.isnan(got[2, :6]).all()) and bool(torch.isnan(got[3, 2]).all())
    assert bool(((got - o).abs() <= do)[~hit].all())
    hit[2, :6] = False   # a value is no part of lse
    assert bool(((gl - lse).abs() <= dl)[~hit].all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("place", ["common", "own", "all", "half"])
def test_scores_of_minus_infinity_weigh_nothing(qs, dtype, place):
    lens = [300, 310, 305]
    b = share.Batch(qs, lens, [(0, 3, 280)], 6, 2, 64, dtype=dtype, seed=13)
    b.qval[..., -1] = 1.0
    b.q.copy_(b.qval)
    for r, n in enumerate(lens):
        for t in {"common": range(280), "own": range(280, n), "all": range(n), "half": range(140)}[place]:
            b.k[b.table[r][t // 16], :, t % 16, -1] = -math.inf
            b.kval[b.table[r][t // 16], :, t % 16, -1] = -1e6
    b.run(qs)
    if place == "all":
        qs.qstate_check()
        assert not bool(b.o.any()) and bool((b.lse == -math.inf).all())
        return
    if place == "common":   # a request whose own tokens are none
        assert bool(torch.isfinite(b.o.float()).all())
    b.check(qs)


def test_weights_far_under_the_largest_are_not_lost_in_f16(qs):
    """One token with a score 30 above the others' and a value of zero: the answer is what the others make of it."""
    for where in (0, 150, 299):
        b = share.Batch(qs, [300, 300], [(0, 2, 300)], 4, 1, 64, dtype="f16", scale=1.0, seed=14)
        b.qval.zero_()
        b.qval[..., 0] = 1.0
        b.q.copy_(b.qval)
        for t in (b.k, b.kval):
            t[..., 0] = 0.0
        page, at = b.table[0][where // 16], where % 16
        for r in range(2):
            page = b.table[r][where // 16]
            for t, y in ((b.k, 30.0), (b.kval, 30.0)):
                t[page, 0, at, 0] = y
            for t in (b.v, b.vval):
                t[page, 0, at] = 0.0
        for t in (b.v, b.vval):
            t.mul_(2.0 ** 14)
        b.run(qs)
        qs.qstate_check()
        o, lse, _, dl = b.expect()
        # weights of e^-30 each: within 2^-8 of the sum's magnitude, which an f16 answer of some 2^-26 cannot show; so by lse, and
        # by the answer's size where it is scaled up to f16's range
        assert bool(((b.lse.double().cpu() - lse).abs() <= dl).all())
        want = o.abs().amax()
        if float(want) > 2.0 ** -20:
            assert float((b.o.double().cpu() - o).abs().amax()) <= 2.0 ** -24 + 2.0 ** -8 * float(want)


def test_a_wait_that_gives_up(qs):
    b = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 128, seed=15)
    b.run(qs)
    qs.qstate_check()
    want = b.o.clone()
    qs.qstate_set_wait_limit(0)
    try:
        b.run(qs)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_ETIMEOUT
    finally:
        qs.qstate_set_wait_limit(-1)
    b.run(qs)
    qs.qstate_check()
    assert torch.equal(b.o, want)


def test_groups_made_for_other_requests_are_reported(qs):
    b = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 64, seed=16)
    other = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 8, 2, 64, seed=16)
    other.group(qs)
    groups = qs.KvGroups(other.d_groups.data, 3)
    qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, groups, b.o, b.lse, b.work)
    with pytest.raises(qs.QstateError):
        qs.qstate_check()


def test_captured_and_replayed_while_lengths_and_groups_change(qs):
    b = share.Batch(qs, [300, 310, 305, 281, 340], [(0, 5, 280)], 8, 2, 64, seed=17)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    b.run(qs)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        b.run(qs)
    for lens, common in (([300, 310, 305, 280, 340], 280), ([290, 0, 305, 281, 340], 256), ([5, 310, 6, 7, 8], 4), ([0] * 5, 100),
                         ([300, 310, 305, 280, 340], 0)):
        b.lens = lens
        b.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.common.fill_(common)
        graph.replay()
        b.check(qs)


def test_two_streams_with_work_spaces_of_their_own(qs):
    batches = [share.Batch(qs, [900 + 10 * i for i in range(9)], [(0, 9, 880)], 8, 2, 128, seed=s) for s in (18, 19)]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(batches, streams):
            b.run(qs, stream=s)
    torch.cuda.synchronize()
    for b in batches:
        b.check(qs)


def test_across_32_bit_offsets(qs):
    """Pages whose entries lie behind 2^31 entries (4 GB and more) of the pool."""
    page, Hkv, d = 1024, 4, 256
    n_pages = 2 ** 31 // (page * Hkv * d) + 40
    small = share.Batch(qs, [2500, 2200, 2100], [(0, 3, 2050)], 8, Hkv, d, page=page, spare=1)
    cfg = qs.KvConfig(Hq=8, Hkv=Hkv, dk=d, dv=d, page=page, n_pages=n_pages, max_pages=3, scale=d ** -0.5)
    cache = qs.new_kv_cache(cfg)
    shift = n_pages - small.cfg.n_pages
    cache.k[shift:], cache.v[shift:] = small.k, small.v
    table = torch.where(small.d_table >= 0, small.d_table + shift, -1)[:, :3].contiguous()
    small.group(qs)
    groups = qs.KvGroups(small.d_groups.data, 3)
    qs.qstate_kv_attend_shared(cfg, cache, small.q, table, small.d_lens, groups, small.o, small.lse, small.work)
    small.check(qs)
    # and a copy there
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    qs.qstate_kv_copy(cfg, cache, qs.KvMoves(i32(n_pages - 1, 3), i32(2, n_pages - 2)))
    qs.qstate_check()
    assert torch.equal(cache.k[2], cache.k[n_pages - 1]) and not bool(cache.v[n_pages - 2].any())


def test_groups_of_another_layer_are_refused(qs):
    b = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 64, seed=20)
    other = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 256, seed=20)
    other.group(qs)
    b.group(qs)
    with pytest.raises(ValueError):
        qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, other.d_groups, b.o, b.lse, b.work)
    # through the C interface: reported on the device, and what is wrong stays inside the buffers
    groups = qs.KvGroups(torch.zeros_like(other.d_groups.data), 3)
    groups.data.copy_(other.d_groups.data)
    qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, groups, b.o, b.lse, b.work)
    with pytest.raises(qs.QstateError):
        qs.qstate_check()
    b.run(qs)
    b.check(qs)


def test_groups_of_another_store_are_refused(qs):
    b = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 128, seed=22)
    codes = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 128, e4m3=True, seed=22)
    codes.group(qs)
    with pytest.raises(ValueError):
        qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, codes.d_groups, b.o, b.lse, b.work)
    groups = qs.KvGroups(torch.zeros_like(codes.d_groups.data), 3)   # through the C interface: reported on the device
    groups.data.copy_(codes.d_groups.data)
    qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, groups, b.o, b.lse, b.work)
    with pytest.raises(qs.QstateError):
        qs.qstate_check()
    check(qs, b)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_few_units_for_many_workers(qs, dtype):
    """Blocks of one and of two halves with so few tiles that not every worker has one."""
    lens, groups = [], []
    for members, common in ((2, 1), (33, 64), (9, 65), (40, 130), (3, 200)):
        groups.append((len(lens), len(lens) + members, common))
        lens += [common + i % 3 for i in range(members)]
    check(qs, share.Batch(qs, lens, groups, 8, 1, 128, e4m3=dtype == "e4m3", seed=23))
    check(qs, share.Batch(qs, lens, groups[:1], 8, 1, 64, e4m3=dtype == "e4m3", seed=24))


def test_the_work_space_serves_the_other_attention_too(qs):
    b = share.Batch(qs, LENS, GROUPS, 8, 2, 128, seed=21)
    check(qs, b)
    b.o.fill_(3)
    qs.qstate_kv_attend(b.cfg, b.cache, b.q, b.d_table, b.d_lens, b.o, b.lse, b.work)
    b.check(qs)


def test_groups_share_where_it_gains(qs):
    """By default a few requests read for themselves; the answers are the same within both bounds, and a request that shares nothing
    has the other attention's to the bit."""
    few = share.Batch(qs, [300, 310, 305], [(0, 3, 280)], 4, 2, 64, seed=22)
    many = share.Batch(qs, [3000] * 200, [(0, 200, 2990)], 8, 8, 128, page=64, seed=23)
    for b, shares in ((few, False), (many, True)):
        for ns in (0, -1):
            qs.qstate_set_shared_gain(ns)
            b.group(qs)
            assert bool(b.d_groups.data[:4].view(torch.int32).item()) == (shares or ns == 0)
            b.o.fill_(7)
            b.attend(qs)
            b.check(qs)
        if not shares:
            got, lse = b.o.clone(), b.lse.clone()
            qs.qstate_kv_attend(b.cfg, b.cache, b.q, b.d_table, b.d_lens, b.o, b.lse, b.work)
            assert torch.equal(b.o, got) and torch.equal(b.lse, lse)
