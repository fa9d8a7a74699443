"""The paged cache of attention layers on the GPU, against plain implementations in 64 bits."""
import math

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200]


# ---- plan --------------------------------------------------------------------------------------------------


def run_plan(qs, lens, n_new, page, spare, T, max_pages, seed=0, in_place=False):
    g = torch.Generator().manual_seed(seed)
    R = len(lens)
    used = sum(ref.pages_of(n, page) for n in lens)
    n_pages = max(1, used + spare)
    perm = torch.randperm(n_pages, generator=g).tolist()
    table = [[-1] * max_pages for _ in lens]
    for r, n in enumerate(lens):
        for c in range(ref.pages_of(n, page)):
            table[r][c] = perm.pop()
    free = list(perm)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cfg = qs.KvConfig(page=page, n_pages=n_pages, max_pages=max_pages)
    pages = qs.KvPages(i32(table).reshape(R, max_pages), i32(lens), i32(free + [-5] * (n_pages - len(free))), i32([len(free)]))
    slots = qs.new_kv_slots(R, T)
    for t in (slots.cu, slots.slot, slots.pos, slots.req):
        t.fill_(-99)
    work = qs.new_kv_work(cfg)
    lens_out, free_out = (pages.lens, pages.free_count) if in_place else (torch.full_like(pages.lens, -99), i32([-99]))
    qs.qstate_kv_plan(cfg, pages, i32(n_new), slots, work, None if in_place else lens_out, None if in_place else free_out)
    qs.qstate_check()
    before = list(free)
    want = ref.plan(lens, n_new, table, free, page, T, max_pages)
    assert slots.cu.tolist() == want["cu"]
    assert slots.ok.tolist() == want["ok"]
    assert lens_out.tolist() == want["lens"]
    assert slots.slot.tolist() == want["slot"]
    assert slots.pos.tolist() == want["pos"]
    assert slots.req.tolist() == want["req"]
    assert pages.table.reshape(R, max_pages).tolist() == table
    assert free_out.tolist() == [len(want["stack"])]
    got = pages.free_list.tolist()
    assert got[: len(want["stack"])] == want["stack"]
    assert got[len(before):] == (want["whole"][len(before):len(want["stack"])] + [-5] * n_pages)[: n_pages - len(before)]
    assert not bool(work.view(torch.int32)[:1024].any())
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R,page,T", [(1, 16, 1), (3, 1, 7), (257, 16, 400), (1025, 64, 9000), (8192, 8, 20000)])
def test_plan_of_a_mixed_step(qs, R, page, T, in_place):
    g = torch.Generator().manual_seed(R)
    pick = lambda lo, hi: torch.randint(lo, hi, (R,), generator=g).tolist()  # noqa: E731
    lens, kind, more = pick(0, 300), pick(0, 10), pick(1, 40)
    n_new = [-1 if k == 0 else 0 if k == 1 else m if k == 2 else 1 for k, m in zip(kind, more)]
    run_plan(qs, lens, n_new, page, spare=R, T=T, max_pages=400, seed=R, in_place=in_place)


@pytest.mark.parametrize("spare", [0, 1, 5, 1000])
def test_plan_refuses_what_the_pool_lacks(qs, spare):
    lens = [16, 15, 0, 40, 16, 3, 0, 32]
    n_new = [1, 1, 100, 1, 16, 0, -1, 1]
    want = run_plan(qs, lens, n_new, 16, spare, 256, 12)
    if spare in (0, 5):
        assert 0 in want["ok"] and 1 in want["ok"]


def test_plan_takes_the_pages_that_come_back(qs):
    want = run_plan(qs, [64, 0, 48, 0], [-1, 40, -3, 70], 16, 0, 110, 8)
    assert want["ok"] == [1, 1, 1, 0]
    want = run_plan(qs, [64, 0, 48, 0], [-1, 40, -3, 50], 16, 0, 90, 8)
    assert want["ok"] == [1, 1, 1, 1]


def test_plan_refuses_rows_and_columns_that_are_not_there(qs):
    assert run_plan(qs, [10, 10, 10], [5, 5, 5], 16, 9, 12, 4)["ok"] == [1, 1, 0]
    assert run_plan(qs, [10, 60, 10], [5, 5, 5], 16, 9, 20, 4)["ok"] == [1, 0, 1]
    assert run_plan(qs, [10], [2 ** 31 - 1], 16, 9, 20, 4)["ok"] == [0]
    want = run_plan(qs, [0] * 3, [2 ** 31 - 1, 2 ** 31 - 1, 1], 16, 9, 20, 4)
    assert want["ok"] == [0, 0, 0]


def test_plan_without_requests_or_rows(qs):
    cfg = qs.KvConfig(page=16, n_pages=4, max_pages=2)
    pages, slots, work = qs.new_kv_pages(cfg, 0), qs.new_kv_slots(0, 5), qs.new_kv_work(cfg)
    qs.qstate_kv_plan(cfg, pages, torch.empty(0, dtype=torch.int32, device="cuda"), slots, work)
    qs.qstate_check()
    assert slots.cu.tolist() == [0] and slots.slot.tolist() == [-1] * 5 and pages.free_count.tolist() == [4]
    run_plan(qs, [5, 7], [-1, 0], 16, 1, 0, 2)


def test_plan_reports_an_inconsistent_pool(qs):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cfg = qs.KvConfig(page=16, n_pages=4, max_pages=2)
    work = qs.new_kv_work(cfg)
    for lens, n_new, table, free, count in (([40], [1], [[0, 1]], [2, 3, 0, 0], 2), ([-3], [1], [[0, 1]], [2, 3, 0, 0], 2),
                                            ([16], [1], [[0, -1]], [2, 9, 0, 0], 2), ([3], [1], [[77, -1]], [2, 3, 0, 0], 2),
                                            ([3], [1], [[0, -1]], [2, 3, 0, 0], 9), ([3], [-1], [[1 << 20, -1]], [2, 3, 0, 0], 2)):
        pages, slots = qs.KvPages(i32(table), i32(lens), i32(free), i32([count])), qs.new_kv_slots(1, 4)
        qs.qstate_kv_plan(cfg, pages, i32(n_new), slots, work)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_EDEVICE and "cache" in str(e.value)
        assert max(slots.slot.tolist()) < 64
    qs.qstate_check()


# ---- append ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("e4m3,dtype", [(False, "bf16"), (False, "f16"), (True, "bf16")])
@pytest.mark.parametrize("T,Hkv,d,page,view", [(1, 1, 64, 1, "dense"), (37, 3, 128, 16, "fused"), (130, 5, 256, 8, "odd"),
                                               (5, 2, 64, 1024, "heads first"), (700, 8, 128, 32, "fused")])
def test_append(qs, T, Hkv, d, page, view, e4m3, dtype):
    g = torch.Generator().manual_seed(T + d)
    n_pages = -(-T // page) + 2
    cfg = qs.KvConfig(Hq=Hkv, Hkv=Hkv, dk=d, dv=d, page=page, n_pages=n_pages, max_pages=n_pages,
                      dtype=qs.KV_F16 if dtype == "f16" else qs.KV_BF16, store=qs.KV_E4M3 if e4m3 else qs.KV_16)
    t = cfg.torch_dtype
    x = torch.randn(2, T, Hkv, d, generator=g) * torch.exp2(torch.randint(-12, 12, (2, T, Hkv, 1), generator=g).float())
    x = x.to(t)
    x[0, 0, 0] = 0
    if T > 30:
        x[1, 3, 0, 5], x[0, 4, 1, 7], x[0, 5, 1, 0] = float("nan"), float("inf"), -float("inf")
        x[1, 6, 0], x[1, 7, 0, 0], x[1, 8, 0, 0] = 448.0, 3.5, 3.515625
        x[0, 9, 0] = 0
        x[0, 9, 0, 1] = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -24
        x[0, 10, 0, 2] = torch.finfo(t).max
    if view == "fused":
        wide = torch.zeros(T, 3 * Hkv, d, dtype=t, device="cuda")
        wide[:, Hkv:2 * Hkv], wide[:, 2 * Hkv:] = x[0].cuda(), x[1].cuda()
        k, v = wide[:, Hkv:2 * Hkv], wide[:, 2 * Hkv:]
    elif view == "odd":   # rows that start on no 16 bytes
        flat = torch.zeros(2, T * (Hkv * d + 3) + 1, dtype=t, device="cuda")
        k, v = (flat[i, 1:].as_strided((T, Hkv, d), (Hkv * d + 3, d, 1), i * flat.shape[1] + 1) for i in range(2))
        k.copy_(x[0]), v.copy_(x[1])
    elif view == "heads first":
        k, v = (x[i].cuda().transpose(0, 1).contiguous().transpose(0, 1) for i in range(2))
    else:
        k, v = x[0].cuda(), x[1].cuda()
    slot = torch.randperm(n_pages * page, generator=g)[:T].int()
    slot[T // 2] = -1 if T > 1 else slot[T // 2]
    cache = qs.new_kv_cache(cfg)
    qs.qstate_kv_append(cfg, cache, k, v, slot.cuda())
    qs.qstate_check()
    keep = slot >= 0
    at, row = slot[keep].long() // page, slot[keep].long() % page
    for got, exps, y in ((cache.k, cache.k_exp, x[0]), (cache.v, cache.v_exp, x[1])):
        want = torch.zeros(n_pages, Hkv, page, d, dtype=torch.float64)
        if e4m3:
            codes, byte = ref.quantise(y[keep])
            wexp = torch.full((n_pages, Hkv, page), 127, dtype=torch.uint8)
            want[at, :, row], wexp[at, :, row] = codes, byte
            assert torch.equal(exps.cpu(), wexp)
            assert torch.equal(got.float().cpu().double(), want)
        else:
            raw = torch.zeros(n_pages, Hkv, page, d, dtype=t)
            raw[at, :, row] = y[keep]
            assert torch.equal(got.cpu().view(torch.int16), raw.view(torch.int16))


@pytest.mark.parametrize("dk,dv", [(128, 128), (288, 256), (576, 512)])
def test_append_latents(qs, dk, dv):
    cfg = qs.KvConfig(kind=qs.KV_LATENT, Hq=4, Hkv=1, dk=dk, dv=dv, page=32, n_pages=5, max_pages=5)
    x = torch.randn(41, 1, dk).to(torch.bfloat16)
    slot = torch.randperm(160)[:41].int()
    cache = qs.new_kv_cache(cfg)
    qs.qstate_kv_append(cfg, cache, x.cuda(), None, slot.cuda())
    qs.qstate_check()
    want = torch.zeros(160, dk, dtype=torch.bfloat16)
    want[slot.long()] = x[:, 0]
    assert torch.equal(cache.k.cpu().view(160, dk), want)


def test_append_reports_a_slot_outside_the_pool(qs):
    for e4m3 in (False, True):
        cfg = qs.KvConfig(Hq=1, Hkv=1, dk=64, dv=64, page=16, n_pages=2, max_pages=2, store=qs.KV_E4M3 if e4m3 else qs.KV_16)
        x = torch.randn(3, 1, 64, device="cuda").to(torch.bfloat16)
        cache = qs.new_kv_cache(cfg)
        qs.qstate_kv_append(cfg, cache, x, x, torch.tensor([5, 32, -9], dtype=torch.int32, device="cuda"))
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_EDEVICE
        assert bool(cache.k[0, 0, 5].float().any()) and not bool(cache.k.view(-1, 64)[6:].float().any())


# ---- attend ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,page", [(1, 1, 16), (6, 2, 8), (20, 4, 64), (16, 1, 1), (40, 2, 32), (24, 8, 1024)])
def test_attend(qs, Hq, Hkv, page, d, dtype, e4m3):
    b = ref.Batch(qs, EDGES, Hq, Hkv, d, page=page, dtype=dtype, e4m3=e4m3, seed=Hq + d, spread=2.0)
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (160, 128), (320, 256), (512, 512), (544, 512), (576, 512)])
@pytest.mark.parametrize("Hq,page", [(1, 16), (7, 64), (16, 1), (33, 32), (64, 8), (100, 128), (130, 16)])
def test_attend_latents(qs, Hq, page, dk, dv, dtype):
    b = ref.Batch(qs, EDGES, Hq, 1, dk, dv, page=page, latent=True, dtype=dtype, seed=Hq + dk, spread=2.0)
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("window", [1, 7, 16, 64, 100, 5000])
@pytest.mark.parametrize("kind", ["heads", "e4m3", "latent"])
def test_attend_through_a_window(qs, kind, window):
    lens = EDGES + [1000, 777]
    b = (ref.Batch(qs, lens, 12, 1, 320, 256, page=16, latent=True, window=window, seed=window) if kind == "latent" else
         ref.Batch(qs, lens, 12, 3, 128, page=16, e4m3=kind == "e4m3", window=window, seed=window))
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("lens", [[4097], [9000, 1], [1, 9000, 0, 333], [30011], [0], [1], [0, 0, 0, 5]])
@pytest.mark.parametrize("kind", ["heads", "e4m3", "latent"])
def test_attend_splits_long_rows(qs, kind, lens):
    b = (ref.Batch(qs, lens, 24, 1, 192, 128, page=32, latent=True, seed=1) if kind == "latent" else
         ref.Batch(qs, lens, 8, 2, 64, page=32, e4m3=kind == "e4m3", seed=2))
    b.run(qs)
    b.check(qs)
    first = b.o.clone(), b.lse.clone()
    for _ in range(3):   # the same sums in the same order each time
        b.o.fill_(9.0)
        b.run(qs)
        assert torch.equal(b.o.view(torch.int16), first[0].view(torch.int16)) and torch.equal(b.lse, first[1])


@pytest.mark.parametrize("R", [300, 2000])
@pytest.mark.parametrize("kind", ["heads", "latent"])
def test_attend_many_short_rows(qs, kind, R):
    lens = [(7 * r) % 41 for r in range(R)]
    b = (ref.Batch(qs, lens, 3, 1, 128, 128, page=8, latent=True) if kind == "latent" else
         ref.Batch(qs, lens, 4, 2, 64, page=8, dtype="f16"))
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("kind", ["heads", "e4m3", "latent"])
def test_attend_with_scores_that_grow_and_fall(qs, kind):
    """Scores that rise by hundreds along the row, fall, or are all as large as the type allows without
    overflow: the running maximum has to follow them."""
    for sign in (1.0, -1.0):
        kw = dict(page=16, scale=1.0, seed=3)
        b = (ref.Batch(qs, [700, 64], 4, 1, 128, 128, latent=True, **kw) if kind == "latent" else
             ref.Batch(qs, [700, 64], 4, 2, 64, e4m3=kind == "e4m3", **kw))
        if kind == "e4m3":
            b.cache.k_exp.fill_(127)
        b.q[:, :, 1:] = 0
        b.q[:, :, 0] = 1
        b.qval.copy_(b.q.cpu())
        for r, n in enumerate(b.lens):
            for t in range(n):
                b.k[b.table[r][t // 16], :, t % 16, 0] = (torch.tensor(t * 0.5 * sign).to(b.t) if kind != "e4m3" else
                                                          torch.tensor(float((t // 16) * 8 * sign)).to(b.k.dtype))
        val = b.k.float().cpu().double()
        if kind == "e4m3":
            val = val * torch.exp2(b.cache.k_exp.cpu().double() - 127)[..., None]
        b.kval = val
        if kind == "latent":
            b.vval = val[..., :128]
        b.run(qs)
        b.check(qs)


def test_attend_strided_queries_without_lse_on_another_stream(qs):
    b = ref.Batch(qs, EDGES, 12, 4, 128, page=16)
    wide = torch.full((len(EDGES), 20, 131), 3.0, dtype=b.t, device="cuda")
    wide[:, 4:16, 1:129] = b.q
    q = wide[:, 4:16, 1:129]   # heads apart by an odd number of entries, on no 16 bytes
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    qs.qstate_kv_attend(b.cfg, b.cache, q, b.d_table, b.d_lens, b.o, b.lse, b.work, stream=s)
    o = b.o
    b.o = torch.empty_like(o)
    qs.qstate_kv_attend(b.cfg, b.cache, q, b.d_table, b.d_lens, b.o, None, b.work, stream=s)
    s.synchronize()
    assert torch.equal(o, b.o)
    b.check(qs)


@pytest.mark.parametrize("latent", [False, True])
def test_attend_across_32_bit_offsets(qs, latent):
    """Pages whose entries lie behind 2^31 entries (4 GB and more) of the pool."""
    Hkv, dk, dv = (1, 576, 512) if latent else (4, 256, 256)
    page = 1024
    n_pages = 2 ** 31 // (page * Hkv * dk) + 40
    cfg = qs.KvConfig(kind=qs.KV_LATENT if latent else qs.KV_HEADS, Hq=8, Hkv=Hkv, dk=dk, dv=dv, page=page, n_pages=n_pages,
                      max_pages=3, scale=dk ** -0.5)
    cache = qs.new_kv_cache(cfg)
    small = ref.Batch(qs, [2500, 1100], 8, Hkv, dk, dv, page=page, latent=latent, spare=1)
    shift = n_pages - small.cfg.n_pages
    cache.k[shift:] = small.k
    if not latent:
        cache.v[shift:] = small.v
    table = torch.where(small.d_table >= 0, small.d_table + shift, -1)[:, :3].contiguous()
    qs.qstate_kv_attend(cfg, cache, small.q, table, small.d_lens, small.o, small.lse, small.work)
    small.check(qs)
    # and the write
    x = torch.randn(5, Hkv, dk, device="cuda").to(torch.bfloat16)
    slot = torch.arange(n_pages * page - 5, n_pages * page, dtype=torch.int32, device="cuda")
    qs.qstate_kv_append(cfg, cache, x, None if latent else x, slot)
    qs.qstate_check()
    assert torch.equal(cache.k[-1, :, -5:].transpose(0, 1), x)


@pytest.mark.parametrize("latent", [False, True])
def test_attend_reports_lengths_and_pages_outside(qs, latent):
    make = lambda: (ref.Batch(qs, [40, 70, 20], 4, 1, 128, 128, latent=True) if latent else  # noqa: E731
                    ref.Batch(qs, [40, 70, 20], 4, 2, 64))
    for change in ("long", "negative", "page", "no page"):
        b = make()
        if change == "long":
            b.d_lens[0] = b.cfg.max_pages * b.cfg.page + 1
            b.d_table[0] = 0
        elif change == "negative":
            b.d_lens[0] = -1
        else:
            b.d_table[0, 1] = b.cfg.n_pages if change == "page" else -1
        b.run(qs)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_EDEVICE and "cache" in str(e.value)
        o, lse, do, _ = b.expect()   # the other requests are not touched by it
        assert bool(((b.o.double().cpu() - o).abs() <= do)[1:].all())


def test_attend_passes_on_what_is_not_finite(qs):
    b = ref.Batch(qs, [40, 70, 20], 4, 2, 64)
    b.v[b.table[0][0], 0, 3, 5] = float("nan")
    b.k[b.table[1][1], 1, 3, 5] = float("nan")
    b.run(qs)
    qs.qstate_check()
    o, lse, do, _ = b.expect()
    got = b.o.double().cpu()
    assert bool(torch.isnan(got[0, :2, 5]).all()) and bool(torch.isnan(got[1, 2:]).all()) and bool(torch.isnan(b.lse[1, 2:]).all())
    bad = torch.isnan(got)
    bad[0, :2, 5] = False
    bad[1, 2:] = False
    assert not bool(bad.any())
    fine = ~torch.isnan(got)
    assert bool(((got - o).abs() <= do)[fine].all())


@pytest.mark.parametrize("dk,dv,page", [(128, 128, 16), (576, 512, 32), (320, 256, 1)])
def test_latent_waits_that_run_out_are_reported(qs, dk, dv, page):
    """With no polls allowed the call gives up and says so; the next one is unaffected."""
    b = ref.Batch(qs, [700, 90, 0, 64], 20, 1, dk, dv, page=page, latent=True)
    qs.qstate_set_wait_limit(0)
    try:
        b.run(qs)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_ETIMEOUT
    finally:
        qs.qstate_set_wait_limit(-1)
    b.run(qs)
    b.check(qs)


def test_a_step_in_a_captured_graph(qs):
    """plan, append and attend captured once and replayed token by token give what a growing cache gives."""
    R, Hq, Hkv, d, page, steps = 5, 8, 2, 64, 16, 40
    cfg = qs.KvConfig(Hq=Hq, Hkv=Hkv, dk=d, dv=d, page=page, n_pages=R * 4, max_pages=4, scale=d ** -0.5)
    cache, pages, slots, work = qs.new_kv_cache(cfg), qs.new_kv_pages(cfg, R), qs.new_kv_slots(R, R), qs.new_kv_work(cfg)
    n_new = torch.ones(R, dtype=torch.int32, device="cuda")
    x = torch.zeros(R, Hq + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.zeros(R, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(R, Hq, device="cuda")

    def step():
        qs.qstate_kv_plan(cfg, pages, n_new, slots, work)
        qs.qstate_kv_append(cfg, cache, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots.slot)
        qs.qstate_kv_attend(cfg, cache, x[:, :Hq], pages.table, pages.lens, o, lse, work)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):   # first calls: the library looks its status word up
        step()
    s.synchronize()
    pages.lens.zero_()
    pages.free_count.fill_(cfg.n_pages)
    pages.free_list.copy_(torch.arange(cfg.n_pages - 1, -1, -1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    xs = torch.randn(steps, R, Hq + 2 * Hkv, d, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    for t in range(steps):
        x.copy_(xs[t])
        graph.replay()
    qs.qstate_check()
    assert pages.lens.tolist() == [steps] * R and pages.free_count.tolist() == [cfg.n_pages - 3 * R]
    z = xs.double()
    K, V = z[:, :, Hq:Hq + Hkv], z[:, :, Hq + Hkv:]
    q = z[-1, :, :Hq].view(R, Hkv, Hq // Hkv, d)
    w = torch.softmax(torch.einsum("rhgd,trhd->rhgt", q, K) * d ** -0.5, -1)
    want = torch.einsum("rhgt,trhd->rhgd", w, V).reshape(R, Hq, d)
    mag = torch.einsum("rhgt,trhd->rhgd", w, V.abs()).reshape(R, Hq, d)
    assert bool(((o.double().cpu() - want).abs() <= 2.0 ** -9 * want.abs() + (2.0 ** -8 + 2.0 ** -13) * mag).all())
    assert math.isfinite(float(lse.sum()))


@pytest.mark.parametrize("window", [0, 45])
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_codes_over_pages_shorter_than_a_chunk(qs, d, page, window):
    b = ref.Batch(qs, EDGES, 10, 2, d, page=page, e4m3=True, window=window, seed=page + d, spread=2.0)
    b.run(qs)
    b.check(qs)
