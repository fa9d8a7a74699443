"""Fork, compact and copy of pages that requests hold together: every number against plain loops, over chains of steps."""
import random

import pytest
import torch

import kv_reference as ref
import kv_share_reference as share

pytestmark = pytest.mark.gpu


def random_step(pool, rng):
    """Parents and tokens to keep: most requests go on, some end, start from another, or go back."""
    R = pool.R
    parent, keep = [], []
    for r in range(R):
        kind = rng.random()
        parent.append(-1 if kind < 0.1 else rng.randrange(R) if kind < 0.5 else r)
        n = pool.lens[parent[-1]] if parent[-1] >= 0 else 0
        keep.append(-1 if rng.random() < 0.5 else rng.choice([0, n, n + 3, rng.randrange(n + 1), n // pool.page * pool.page]))
    return parent, keep


@pytest.mark.parametrize("R,page,n_pages,max_pages,seed", [
    (1, 1, 5, 4, 0), (3, 4, 40, 30, 1), (7, 16, 60, 20, 2), (20, 8, 90, 40, 3), (33, 2, 700, 300, 4), (64, 1, 1500, 130, 5),
    (5, 1024, 12, 6, 6), (2, 4, 900, 700, 7)])
def test_chains_of_steps(qs, R, page, n_pages, max_pages, seed):
    pool = share.Pool(qs, R, page, n_pages, max_pages, seed)
    rng = random.Random(seed)
    most = max_pages * page
    for step in range(12):
        pool.grow([rng.randrange(min(most, max(2, n_pages * page // (2 * R)))) if rng.random() < 0.7 else 0 for _ in range(R)])
        pool.fork(*random_step(pool, rng), spare_moves=step % 3)
        pool.sound()
        if step % 3 == 2:
            limit = rng.choice([n_pages, max(1, n_pages // 2), 1, rng.randrange(1, n_pages + 1)])
            pool.compact(limit, rng.choice([0, 1, n_pages]), apart=step % 2 == 0)
            pool.compact(n_pages, 3)   # every page that nobody holds is on the list again
            pool.sound()
    qs.qstate_check()


def test_more_requests_than_a_thread_each(qs):
    R, page = 1500, 4
    pool = share.Pool(qs, R, page, 9000, 12, 1)
    rng = random.Random(8)
    pool.grow([rng.randrange(20) for _ in range(R)])
    for _ in range(2):
        parent, keep = random_step(pool, rng)
        pool.fork([r // 3 * 3 if p != r and p >= 0 else p for r, p in enumerate(parent)], keep)
        pool.sound()
    qs.qstate_check()


def test_long_tables_in_parts(qs):
    """Tables above what one cluster works on, with parts that end inside a request's pages."""
    R, page, width = 40, 1, 20000
    pool = share.Pool(qs, R, page, 60000, width, 2)
    pool.grow([900 * r % 3001 for r in range(R)])
    rng = random.Random(3)
    for _ in range(2):
        pool.fork(*random_step(pool, rng))
        pool.sound()
    pool.compact(30000, 60000)
    qs.qstate_check()


@pytest.mark.parametrize("R,n_pages,max_pages", [
    (12, 30000, 1000), (12, 70000, 1000),   # one cluster with several spans of the pool, more spans than it has CTAs
    (33, 9000, 500), (31, 9000, 500),       # compact by steps and fork by the cluster, both by the cluster
    (256, 20000, 128), (257, 20000, 100)])  # fork by the cluster, fork by steps
def test_both_forms_of_the_launch(qs, R, n_pages, max_pages):
    pool = share.Pool(qs, R, 2, n_pages, max_pages, R)
    rng = random.Random(n_pages)
    pool.grow([rng.randrange(min(2 * max_pages, 2 * n_pages // (2 * R))) for _ in range(R)])
    for _ in range(3):
        pool.fork(*random_step(pool, rng))
        pool.sound()
    pool.compact(n_pages // 3, n_pages)
    pool.compact(n_pages, 0)
    pool.sound()
    qs.qstate_check()


def test_families_whose_members_take_over_from_each_other(qs):
    """Prefixes that are held before and after: their holders stay, whoever changes places and whoever leaves."""
    R = 24
    pool = share.Pool(qs, R, 4, 900, 60, 9)
    pool.grow([150 if r % 8 == 0 else 0 for r in range(R)])
    pool.fork([r // 8 * 8 for r in range(R)])          # three families of eight
    rng = random.Random(10)
    for step in range(6):
        pool.grow([rng.randrange(9) for _ in range(R)])
        parent = [r // 8 * 8 + rng.randrange(8) for r in range(R)]
        if step % 2:
            parent[8:16] = [-1] * 8 if step == 3 else [0] * 8   # a family ends, or goes over to another
        pool.fork(parent, [rng.choice([-1, 120, 151]) for _ in range(R)])
        pool.sound()
    qs.qstate_check()


def test_holders_counted_one_short(qs):
    """The formula's numbers, whatever the counts say: a page that requests take over again can come back too."""
    R = 12
    pool = share.Pool(qs, R, 4, 200, 30, 11)
    pool.grow([50 if r % 6 == 0 else 0 for r in range(R)])
    pool.fork([r // 6 * 6 for r in range(R)])
    pool.others = [h - (h > 0 and x % 3 == 0) for x, h in enumerate(pool.others)]
    pool.d_others.copy_(pool.i32(pool.others))
    before = pool.free
    pool.fork([(r // 6 * 6 + (r + 1) % 6) if r not in (4, 9) else -1 for r in range(R)], [37] * R)
    pool.fork([r // 6 * 6 for r in range(R)])
    for _ in range(4):
        pool.others = [max(h - 1, 0) for h in pool.others]
        pool.d_others.copy_(pool.i32(pool.others))
        pool.fork([r // 6 * 6 + (r + 2) % 6 for r in range(R)])
    assert pool.free > before
    qs.qstate_check()


def test_holders_counted_two_short(qs):
    """A count under none is none, and the page is not on the list."""
    R = 6
    pool = share.Pool(qs, R, 4, 100, 30, 12)
    pool.grow([50, 0, 0, 0, 0, 9])
    pool.fork([0, 0, 0, 0, 0, 5])
    pool.others = [max(h - 2, 0) for h in pool.others]
    pool.d_others.copy_(pool.i32(pool.others))
    pool.fork([-1, -1, -1, -1, -1, 5])   # five held them, three are known
    assert min(pool.others) == 0
    qs.qstate_check()


@pytest.mark.parametrize("n_pages", [100, 40000])   # one cluster, and by steps
def test_lengths_of_before_with_tables_of_after(qs, n_pages):
    """A call made again on the lengths it has replaced: counts, list and tables by the formula, though they do not agree."""
    R = 12
    pool = share.Pool(qs, R, 4, n_pages, 30, 13)
    pool.grow([20 + 3 * r for r in range(R)] if n_pages > 100 else [5 + r for r in range(R)])
    lens = list(pool.lens)
    pool.others[pool.free_list[0]] = 3   # of a page that nobody holds
    pool.d_others.copy_(pool.i32(pool.others))
    for k in range(3):
        pool.fork([r // 4 * 4 + (r * (k + 2) + 1) % 4 if r % 5 else -1 for r in range(R)])
        pool.lens = list(lens)
        pool.pages.lens.copy_(pool.i32(lens))
    qs.qstate_check()


def test_beams_that_change_places(qs):
    pool = share.Pool(qs, 8, 16, 200, 20, 3)
    pool.grow([100] * 8)
    rng = random.Random(4)
    for step in range(10):
        pool.fork([r // 4 * 4 + rng.randrange(4) for r in range(8)])
        pool.sound()
        pool.grow([1 + step % 3] * 8)
    assert max(pool.others) > 0
    qs.qstate_check()


def test_refusals_for_want_of_pages(qs):
    pool = share.Pool(qs, 6, 8, 10, 10, 5)
    pool.grow([20, 0, 0, 0, 0, 0])           # 3 pages, the last cut; 7 on the list
    pool.grow([0, 32, 0, 0, 0, 0])           # 3 left
    moves, got = pool.fork([0, 1, 0, 0, 0, 0])
    assert got["ok"] == [1, 1, 1, 1, 1, 0] and pool.lens[5] == 0
    pool.sound()
    qs.qstate_check()


def test_everyone_ends(qs):
    pool = share.Pool(qs, 9, 4, 80, 12, 6)
    pool.grow([0, 3, 4, 5, 8, 9, 20, 21, 40])
    pool.fork([8, 8, 8, 6, 6, 7, 6, 7, 8])
    pool.fork([-1] * 9)
    assert pool.free == 80 and not any(pool.others)
    pool.sound()
    qs.qstate_check()


def test_no_requests(qs):
    cfg = qs.KvConfig(page=4, n_pages=6, max_pages=2)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pages = qs.KvPages(i32(), i32(), i32(3, 1, 2, 0, 4, 5), i32(4))
    others, out, left = torch.zeros(6, dtype=torch.int32, device="cuda"), i32(-1), i32(-1)
    moves, work = qs.new_kv_moves(2), qs.new_kv_pages_work(cfg, 0)
    moves.src.fill_(7)
    qs.qstate_kv_fork(cfg, pages, others, i32(), None, moves, torch.zeros(0, dtype=torch.uint8, device="cuda"), work, free_out=out)
    assert out.tolist() == [4] and moves.src.tolist() == [-1, -1]
    qs.qstate_kv_compact(cfg, pages, None, 5, moves, left, work)
    assert pages.free_list.tolist() == [4, 3, 2, 1, 0, 5] and pages.free_count.tolist() == [5] and left.tolist() == [0]
    qs.qstate_check()


def test_a_work_space_serves_fewer_requests_too(qs):
    """What must be zero between calls lies at the same place whatever the number of requests."""
    cfg = qs.KvConfig(page=4, n_pages=300, max_pages=50)
    work = qs.new_kv_pages_work(cfg, 30)
    for R in (30, 3, 17, 30):
        pool = share.Pool(qs, R, 4, 300, 50, R)
        pool.work = work
        rng = random.Random(R)
        pool.grow([rng.randrange(30) for _ in range(R)])
        pool.fork(*random_step(pool, rng))
        pool.compact(100, 300)
        pool.compact(300, 0)   # pages behind the limit go back on the list
        pool.sound()
    qs.qstate_check()


def test_pages_outside_the_pool_are_reported(qs):
    for table, lens, parent in (([[0, 99, 2], [3, 4, 5]], [10, 12], [0, 0]), ([[0, 1, -3], [3, 4, 5]], [11, 1], [-1, 0]),
                                ([[0, 1, 77], [3, 4, 5]], [9, 12], [1, 0]), ([[0, 1, 2], [3, 4, 5]], [13, -1], [0, 1]),
                                ([[0, 1, 2], [3, 4, 5]], [5, 5], [2, 1])):
        cfg = qs.KvConfig(page=4, n_pages=12, max_pages=3)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        pages = qs.KvPages(i32(table), i32(lens), i32(list(range(6, 12)) + [-1] * 6), i32([6]))
        work, moves, others = qs.new_kv_pages_work(cfg, 2), qs.new_kv_moves(2), torch.zeros(12, dtype=torch.int32, device="cuda")
        qs.qstate_kv_fork(cfg, pages, others, i32(parent), None, moves, torch.zeros(2, dtype=torch.uint8, device="cuda"), work)
        with pytest.raises(qs.QstateError) as e:
            qs.qstate_check()
        assert e.value.code == qs.QSTATE_EDEVICE
    pages = qs.KvPages(i32([[0, 50, 2]]), i32([12]), i32([-1] * 12), i32([0]))
    qs.qstate_kv_compact(cfg, pages, None, 12, moves, None, work)
    with pytest.raises(qs.QstateError):
        qs.qstate_check()


@pytest.mark.parametrize("kind,page", [("heads", 16), ("heads", 1), ("e4m3", 32), ("e4m3", 1), ("e4m3", 2), ("latent", 64)])
def test_copies_of_whole_pages(qs, kind, page):
    n_pages = 23
    layer = dict(kind=qs.KV_LATENT, Hq=4, Hkv=1, dk=160, dv=128) if kind == "latent" else dict(Hq=6, Hkv=3, dk=64, dv=64)
    cfg = qs.KvConfig(page=page, n_pages=n_pages, max_pages=4, store=qs.KV_E4M3 if kind == "e4m3" else qs.KV_16, **layer)
    cache = qs.new_kv_cache(cfg)
    g = torch.Generator().manual_seed(3)
    held = [t for t in (cache.k, cache.v, cache.k_exp, cache.v_exp) if t is not None]
    for t in held:   # any bits
        raw = t.view(torch.uint8)
        raw.copy_(torch.randint(0, 256, raw.shape, generator=g).to(torch.uint8))
    want = [t.view(torch.uint8).clone() for t in held]
    src, dst = [0, -1, 5, 7, 22, 9], [1, -1, 6, 8, 3, 21]
    for w in want:
        for a, b in zip(src, dst):
            if a >= 0:
                w[b] = w[a]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    qs.qstate_kv_copy(cfg, cache, qs.KvMoves(i32(src), i32(dst)))
    qs.qstate_check()
    for t, w in zip(held, want):
        assert torch.equal(t.view(torch.uint8), w)
    qs.qstate_kv_copy(cfg, cache, qs.KvMoves(i32([]), i32([])))
    qs.qstate_kv_copy(cfg, cache, qs.KvMoves(i32([4, 4, 0]), i32([n_pages, -1, 1])))
    with pytest.raises(qs.QstateError):
        qs.qstate_check()
    for t, w in zip(held, want):
        assert torch.equal(t.view(torch.uint8), w)


def test_a_captured_step_replayed(qs):
    """plan and fork in a graph: each replay goes on from where the last one left the tables."""
    pool = share.Pool(qs, 12, 4, 400, 60, 9)
    pool.grow([17] * 12)
    parent, new = [0, 0, 2, 2, 5, 4, -1, 7, 8, 8, 11, 10], [2] * 12
    d_parent, d_new = pool.i32(parent), pool.i32(new)
    slots, moves = qs.new_kv_slots(12, 24), qs.new_kv_moves(12)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        qs.qstate_kv_fork(pool.cfg, pool.pages, pool.d_others, d_parent, None, moves, pool.ok, pool.work)
        qs.qstate_kv_plan(pool.cfg, pool.pages, d_new, slots, pool.plan_work)
    for _ in range(4):
        graph.replay()
        got = share.fork(pool.lens, pool.table, pool.free_list, pool.free, pool.others, parent, None, 4)
        stack = pool.free_list[: got["free"]]
        plan = ref.plan(got["lens"], new, pool.table, stack, 4, 24, 60)
        pool.lens, pool.free = plan["lens"], len(stack)
        assert moves.src.tolist() == got["src"] and slots.slot.tolist() == plan["slot"]
        pool.same()
    pool.sound()
    qs.qstate_check()
