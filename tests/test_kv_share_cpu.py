"""Refusals and sizes of the calls on shared pages, on the CPU: placeholder device addresses, which every call here refuses
before anything could read them; and the plain loops that the GPU is compared with."""
import ctypes as ct
import os
import random
import re

import pytest
import torch

import kv_reference as ref
import kv_share_reference as share
from test_kv_cpu import A, config, copies

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_30950_gb300", "csrc")


@pytest.fixture(scope="module")
def q():
    from paper_2609_30950_gb300 import build
    import paper_2609_30950_gb300 as q
    build.build()
    q.load()
    return q


def test_calls_refuse_what_cannot_be(q):
    L, r = q._lib, ct.byref
    c, lat, e4 = config(q), config(q, kind=1, Hkv=1, dk=192, dv=128), config(q, store=1)
    good = q._KvCache(A, A, None, None)

    def fork(c=c, table=A, lens=A, lens_out=A, fl=A, fc=A, fo=A, others=A, parent=A, R=1, src=A, dst=A, n=1, ok=A, work=A):
        return L.qstate_kv_fork(r(c._c), r(q._KvPages(table, lens, lens_out, fl, fc, fo)), others, parent, None, R,
                                r(q._KvMoves(src, dst, n)), ok, work, None)

    def compact(c=c, table=A, lens=A, fl=A, fo=A, R=1, limit=5, src=A, dst=A, n=1, out=A, left=None, work=A):
        return L.qstate_kv_compact(r(c._c), r(q._KvPages(table, lens, None, fl, None, fo)), None, R, limit, r(q._KvMoves(src, dst, n)),
                                   left, out, work, None)

    def copy(c=c, cache=good, src=A, dst=A, n=1):
        return L.qstate_kv_copy(r(c._c), r(cache), r(q._KvMoves(src, dst, n)), None)

    def group(c=c, lens=A, R=4, start=A, common=A, N=2, groups=A):
        return L.qstate_kv_group(r(c._c), lens, R, start, common, N, groups, None)

    def attend(c=c, cache=good, qp=A, table=A, lens=A, R=1, groups=A, o=A, lse=A, work=A):
        return L.qstate_kv_attend_shared(r(c._c), r(cache), qp, 1024, 128, table, lens, R, groups, o, lse, work, None)

    calls = [lambda k=k, f=f: f(**{k: None}) for f, names in (
        (fork, ("table", "lens", "lens_out", "fl", "fc", "fo", "others", "parent", "src", "dst", "ok", "work")),
        (compact, ("table", "lens", "fl", "fo", "src", "dst", "out", "work")), (copy, ("src", "dst")),
        (group, ("lens", "start", "common", "groups")), (attend, ("qp", "table", "lens", "groups", "o", "work"))) for k in names]
    calls += [lambda k=k, f=f: f(**{k: A + 2}) for f, names in (   # arrays of words
        (fork, ("table", "lens", "lens_out", "fl", "fc", "fo", "others", "parent", "src", "dst")),
        (compact, ("table", "lens", "fl", "fo", "src", "dst", "out", "left")), (copy, ("src", "dst")),
        (group, ("lens", "start", "common")), (attend, ("table", "lens", "lse"))) for k in names]
    calls += [lambda f=f, R=R: f(R=R) for f in (fork, compact, group, attend) for R in (-1, 8193)]
    calls += [lambda: fork(n=0), lambda: fork(R=2), lambda: fork(n=-1), lambda: compact(n=-1), lambda: copy(n=-1),
              lambda: compact(limit=0), lambda: compact(limit=11), lambda: fork(work=A + 64), lambda: compact(work=A + 64),
              lambda: attend(work=A + 64), lambda: attend(groups=A + 8), lambda: group(groups=A + 8), lambda: group(N=-1), lambda: group(N=5),
              lambda: attend(c=lat, cache=q._KvCache(A, None, None, None)), lambda: group(c=lat), lambda: attend(c=e4), lambda: copy(c=e4),
              lambda: copy(cache=q._KvCache(None, A, None, None)), lambda: copy(cache=q._KvCache(A + 8, A, None, None)),
              lambda: attend(o=A + 8), lambda: attend(qp=A + 1), lambda: fork(c=config(q, page=3)), lambda: compact(c=config(q, page=3))]
    for call in calls:
        assert call() == q.QSTATE_EINVAL
        assert L.qstate_last_error()
    assert L.qstate_kv_copy(r(c._c), r(good), None, None) == q.QSTATE_EINVAL
    assert L.qstate_kv_fork(None, None, A, A, None, 1, None, A, A, None) == q.QSTATE_EINVAL
    # nothing to do, and nothing launched
    assert copy(n=0) == attend(R=0) == q.QSTATE_OK


def test_sizes(q):
    c, L, r = config(q), q._lib, ct.byref
    lat = config(q, kind=1, Hkv=1, dk=192, dv=128)
    for name in ("qstate_kv_pages_work_bytes", "qstate_kv_group_bytes", "qstate_kv_shared_work_bytes"):
        f = getattr(L, name)
        small, large = f(r(c._c), 1), f(r(c._c), 100)
        assert 0 < small < large and f(r(c._c), 0) > 0
        assert f(r(c._c), -1) == f(r(c._c), 8193) == f(r(config(q, page=3)._c), 4) == 0
        if "pages" not in name:
            assert f(r(lat._c), 4) == 0
    # what the other attention needs of a work space lies in front
    assert L.qstate_kv_shared_work_bytes(r(c._c), 1) > L.qstate_kv_work_bytes(r(c._c))
    pool = q._KvCfg(page=16, n_pages=10, max_pages=4)
    assert L.qstate_kv_pages_work_bytes(r(pool), 4) > 0
    with pytest.raises(q.QstateError):
        q.new_kv_groups(lat, 4, device="cpu")


def test_binding_refuses_what_does_not_fit(q, monkeypatch):
    monkeypatch.setattr(q, "_ptr", lambda t: t.data_ptr())   # host tensors stand for device ones
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    moves = q.KvMoves(i32(3), i32(3))
    for d in copies(moves):
        assert d._at == ct.addressof(d._c) != moves._at and d._c.src == d.src.data_ptr() and d._c.n == d.n == 3
    with pytest.raises(ValueError):
        q.KvMoves(i32(3), i32(4))
    with pytest.raises(ValueError):
        q.KvMoves(torch.zeros(3, dtype=torch.int64), i32(3))
    c = config(q)
    groups = q.new_kv_groups(c, 5, device="cpu")
    groups._check(c)
    with pytest.raises(ValueError):
        q.KvGroups(torch.zeros(100, dtype=torch.uint8), 5)._check(c)
    with pytest.raises(ValueError):   # no device tensor
        q.qstate_kv_group(c, i32(5), i32(3), i32(2), groups)
    pages = q.KvPages(i32(3, 4), i32(3), i32(10), i32(1))
    work = q.new_kv_pages_work(c, 3, device="cpu")
    with pytest.raises(ValueError):
        q.qstate_kv_fork(c, pages, i32(10), i32(3), None, q.KvMoves(i32(2), i32(2)), torch.zeros(3, dtype=torch.uint8), work)
    with pytest.raises(ValueError):
        q.qstate_kv_compact(c, pages, None, 5, moves, None, torch.zeros(16, dtype=torch.uint8), free_out=i32(1))


@pytest.mark.parametrize("seed", range(30))
def test_the_plain_loops_keep_tables_sound(seed):
    """Pages are held as often as `others` says or once on the list, a page that is not full has one holder, and every token stays
    what it was: tokens are labels, written where a request's next one goes and copied as the moves say."""
    rng = random.Random(seed)
    R, page, n_pages, width = rng.randrange(1, 9), rng.choice([1, 2, 4]), rng.randrange(4, 60), rng.randrange(2, 20)
    lens, table, others = [0] * R, [[-5] * width for _ in range(R)], [0] * n_pages
    free_list, free = list(range(n_pages)), n_pages
    place, text, label = {}, [[] for _ in range(R)], 0   # (page, place) -> label; each request's labels
    for step in range(8):
        new, stack = [rng.randrange(8) for _ in range(R)], free_list[:free]
        before, got = lens, ref.plan(lens, new, table, stack, page, sum(new), width)
        lens, free = got["lens"], len(stack)
        for r in range(R):
            for t in range(before[r], lens[r]):
                place[table[r][t // page], t % page] = label
                text[r].append(label)
                label += 1
        parent = [-1 if rng.random() < .1 else rng.randrange(R) if rng.random() < .5 else r for r in range(R)]
        keep = [rng.choice([-1, 0, rng.randrange(20)]) for _ in range(R)]
        got = share.fork(lens, table, free_list, free, others, parent, keep, page)
        lens, free = got["lens"], got["free"]
        moves = list(zip(got["src"], got["dst"]))
        old = text
        text = [old[p][:n] if p >= 0 else [] for p, n in zip(parent, lens)]
        if step % 3 == 2:
            copied = dict(place)
            for a, b in moves:
                for i in range(page):
                    place[b, i] = copied.get((a, i))
            got = share.compact(lens, table, table, free_list, others, rng.randrange(1, n_pages + 1), rng.choice([1, n_pages]), page)
            moves, free = list(zip(got["src"], got["dst"])), got["free"]
            copied = dict(place)
            for a, b in moves:
                for i in range(page):
                    place[b, i] = copied.get((a, i))
            free = share.compact(lens, table, table, free_list, others, n_pages, 0, page)["free"]
        else:
            copied = dict(place)
            for a, b in moves:
                for i in range(page):
                    place[b, i] = copied.get((a, i))
        held = [0] * n_pages
        for r, n in enumerate(lens):
            assert [place[table[r][t // page], t % page] for t in range(n)] == text[r]
            for x in table[r][: ref.pages_of(n, page)]:
                held[x] += 1
        assert others == [max(h - 1, 0) for h in held]
        assert sorted(free_list[:free]) == [x for x, h in enumerate(held) if h == 0]
        for r, n in enumerate(lens):
            assert n % page == 0 or held[table[r][n // page]] == 1


def test_tensor_memory_of_shared_tokens_is_taken_between_wait_and_release():
    """A kernel that is let in before this one holds its tensor memory could take it first and then wait for this one."""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "qs_kv_shared.cuh")).read())
    body = src[src.index("kv_shared_kernel(const KvAttendParams p"):src.index("cudaError_t launch_shared(")]
    at = [body.index(s) for s in ("chain_enter();", "tmem_alloc(", "tmem_relinquish();", "chain_release();", "__syncthreads();")]
    assert at == sorted(at)
    assert body.count("chain_") == 2 and "chain_wait" not in src


def test_a_refused_call_makes_no_groups(q, monkeypatch):
    """What groups were made for is what the last call that was accepted said."""
    monkeypatch.setattr(q, "_ptr", lambda t: t.data_ptr())   # host tensors stand for device ones
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    c, other = config(q), config(q, window=7)
    groups = q.new_kv_groups(c, 5, device="cpu")
    q._keep(groups, _made=c)   # as an accepted call leaves it
    with pytest.raises(ValueError):   # no device tensors
        q.qstate_kv_group(other, i32(5), i32(3), i32(2), groups)
    assert groups._made is c
