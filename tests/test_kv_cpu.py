"""Refusals and sizes of the paged cache's calls, on the CPU: placeholder device addresses, which every call
here refuses before anything could read them."""
import copy
import ctypes as ct
import io

import pytest
import torch

import kv_reference as ref

A = 1 << 20


@pytest.fixture(scope="module")
def q():
    from paper_2609_30950_gb300 import build
    import paper_2609_30950_gb300 as q
    build.build()
    q.load()
    return q


def config(q, **kw):
    base = dict(page=16, n_pages=10, max_pages=4, Hq=8, Hkv=2, dk=128, dv=128)
    base.update(kw)
    return q.KvConfig(**base)


@pytest.mark.parametrize("kw", [
    dict(page=0), dict(page=24), dict(page=2048), dict(n_pages=0), dict(n_pages=1 << 28), dict(max_pages=0),
    dict(max_pages=1 << 28), dict(Hq=0), dict(Hq=9), dict(Hq=2048, Hkv=1), dict(Hkv=0), dict(dk=96, dv=96), dict(dv=64),
    dict(kind=2), dict(dtype=2), dict(store=2), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(store=1, dtype=1), dict(kind=1), dict(kind=1, Hkv=1, dk=144, dv=128), dict(kind=1, Hkv=1, dk=192, dv=192),
    dict(kind=1, Hkv=1, dk=192, dv=128, store=1)])
def test_configurations_that_are_refused(q, kw):
    with pytest.raises(q.QstateError) as e:
        q.kv_validate(config(q, **kw))
    assert e.value.code == q.QSTATE_EINVAL
    assert q._lib.qstate_kv_work_bytes(ct.byref(config(q, **kw)._c)) == 0


@pytest.mark.parametrize("kw", [
    dict(), dict(page=1), dict(page=1024), dict(dk=64, dv=64), dict(dk=256, dv=256), dict(store=1), dict(dtype=1),
    dict(kind=1, Hkv=1, dk=576, dv=512), dict(kind=1, Hkv=1, dk=128, dv=128, Hq=1, dtype=1), dict(window=1), dict(scale=-1.0)])
def test_configurations_that_are_taken(q, kw):
    c = config(q, **kw)
    q.kv_validate(c)
    per = c.n_pages * c.page * c.Hkv * (1 if c.store else 2)
    assert q._lib.qstate_kv_cache_bytes(ct.byref(c._c), 0) == per * c.dk
    assert q._lib.qstate_kv_cache_bytes(ct.byref(c._c), 1) == (0 if c.kind else per * c.dv)
    assert q._lib.qstate_kv_work_bytes(ct.byref(c._c)) >= 4096


def test_calls_refuse_missing_and_unaligned_pointers(q):
    L, c, r = q._lib, config(q), ct.byref
    lat = config(q, kind=1, Hkv=1, dk=192, dv=128)
    e4 = config(q, store=1)
    good = q._KvCache(A, A, None, None)

    def attend(c=c, cache=good, qp=A, table=A, lens=A, R=1, o=A, work=A):
        return L.qstate_kv_attend(r(c._c), r(cache), qp, 1024, 128, table, lens, R, o, None, work, None)

    def append(c=c, cache=good, k=A, v=A, slot=A, T=1):
        return L.qstate_kv_append(r(c._c), r(cache), k, 256, 128, v, 256, 128, slot, T, None)

    def plan(c=c, table=A, lens=A, lens_out=A, fl=A, fc=A, fo=A, n_new=A, R=1, cu=A, slot=A, ok=A, T=1, work=A):
        return L.qstate_kv_plan(r(c._c), r(q._KvPages(table, lens, lens_out, fl, fc, fo)), n_new, R,
                                r(q._KvSlots(cu, slot, None, None, ok, T)), work, None)

    bad_cache = [q._KvCache(None, A, None, None), q._KvCache(A, None, None, None), q._KvCache(A + 8, A, None, None),
                 q._KvCache(A, A + 2, None, None), q._KvCache(A, A, A, A)]
    calls = [lambda b=b: attend(cache=b) for b in bad_cache] + [lambda b=b: append(cache=b) for b in bad_cache]
    calls += [lambda: attend(c=lat), lambda: attend(c=e4), lambda: append(c=e4),
              lambda: append(c=lat, cache=q._KvCache(A, None, None, None)),   # values beside a latent
              lambda: attend(R=-1), lambda: attend(R=8193), lambda: append(T=-1), lambda: plan(R=-1), lambda: plan(R=8193),
              lambda: plan(T=-1), lambda: plan(slot=None), lambda: plan(work=A + 64), lambda: plan(work=None),
              lambda: plan(c=config(q, page=3))]
    for call in calls:
        assert call() == q.QSTATE_EINVAL
        assert L.qstate_last_error()
    assert L.qstate_kv_plan(r(c._c), None, A, 1, None, A, None) == q.QSTATE_EINVAL
    assert L.qstate_kv_attend(None, r(good), A, 0, 0, A, A, 1, A, None, A, None) == q.QSTATE_EINVAL
    assert L.qstate_kv_append(None, r(good), A, 0, 0, A, 0, 0, A, 1, None) == q.QSTATE_EINVAL


def test_binding_refuses_host_tensors_and_changed_fields(q):
    c = config(q)
    with pytest.raises(ValueError):
        q.KvCache(torch.zeros(4, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        q.KvPages(*(torch.zeros(4, dtype=torch.int64) for _ in range(4)))
    with pytest.raises(Exception):
        c.page = 8


def test_reference_codes_are_the_nearest():
    """The reference's quantiser against a search over all codes of the type."""
    raw = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double()
    raw = raw[torch.isfinite(raw)].unique()
    x = torch.cat([torch.randn(20, 64, generator=torch.Generator().manual_seed(1)), torch.zeros(1, 64),
                   torch.full((1, 64), 448.0), torch.full((1, 64), 449.0)]).to(torch.bfloat16)
    codes, byte = ref.quantise(x)
    y = x.double() / torch.exp2(byte.double() - 127)[:, None]
    assert float(y.abs().max()) <= 448
    assert torch.equal((codes - y).abs(), (y[..., None] - raw).abs().amin(-1))
    big = y.abs().amax(-1)
    assert bool(((big > 224) | (big == 0)).all())   # one power lower would not do


def test_exponents_that_are_not_aligned_are_refused(q):
    """The attention reads exponents four at a time."""
    L, c, r = q._lib, config(q, store=q.KV_E4M3), ct.byref
    for cache in (q._KvCache(A, A, A + 2, A), q._KvCache(A, A, A, A + 1)):
        assert L.qstate_kv_attend(r(c._c), r(cache), A, 1024, 128, A, A, 1, A, None, A, None) == q.QSTATE_EINVAL
        assert b"exponents" in L.qstate_last_error()
        assert L.qstate_kv_append(r(c._c), r(cache), A, 256, 128, A, 256, 128, A, 1, None) == q.QSTATE_EINVAL


def copies(x):
    yield copy.copy(x)
    yield copy.deepcopy(x)
    file = io.BytesIO()
    torch.save(x, file)   # pickles, tensors of every type among it
    file.seek(0)
    yield torch.load(file, weights_only=False)


def test_copies_of_a_description_stand_by_themselves(q):
    """The calls pass a description's address on: a copy has to have one of its own."""
    c = config(q, window=7)
    for d in copies(c):
        assert d == c and d._at != c._at and d._at == ct.addressof(d._c)
        seen = q._KvCfg.from_address(d._at)
        assert [getattr(seen, n) for n, _ in q._KvCfg._fields_] == [getattr(c._c, n) for n, _ in q._KvCfg._fields_]
        q.kv_validate(d)


def test_copies_of_tensors_holders_point_to_their_own_tensors(q, monkeypatch):
    monkeypatch.setattr(q, "_ptr", lambda t: t.data_ptr())   # host tensors stand for device ones
    c = config(q, store=q.KV_E4M3)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    fp8 = lambda: torch.zeros(10, 2, 16, 128).to(torch.float8_e4m3fn)  # noqa: E731
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8)  # noqa: E731
    cache = q.KvCache(fp8(), fp8(), u8(10, 2, 16), u8(10, 2, 16))
    cache._check(c)
    pages, slots = q.KvPages(i32(3, 4), i32(3), i32(10), i32(1)), q.KvSlots(i32(4), i32(5), i32(5), None, u8(3))
    for d in copies(pages):
        assert d._args == [t.data_ptr() for t in (d.table, d.lens, d.free_list, d.free_count)] and d.R == 3
    for x, names in ((cache, ("k", "v", "k_exp", "v_exp")), (slots, ("cu", "slot", "pos", "req", "ok"))):
        for d in copies(x):
            assert d._at == ct.addressof(d._c) != x._at
            for n in names:
                t = getattr(d, n)
                assert getattr(d._c, n) == (None if t is None else t.data_ptr())
    deep = copy.deepcopy(pages)
    deep.lens.fill_(5)
    assert not bool(pages.lens.any()) and deep._args[1] == deep.lens.data_ptr() != pages._args[1]


def test_a_pool_alone_has_the_plans_work_space(q):
    """The plan takes a description of which page, n_pages and max_pages alone are set, and so does its work space."""
    bytes_of = lambda **kw: q._lib.qstate_kv_work_bytes(ct.byref(q._KvCfg(**kw)))  # noqa: E731
    layer = q._lib.qstate_kv_work_bytes(ct.byref(config(q)._c))
    assert 4096 <= bytes_of(page=16, n_pages=10, max_pages=4) <= layer
    assert bytes_of(page=16, n_pages=10) == bytes_of(page=3, n_pages=10, max_pages=4) == 0
    assert bytes_of(page=16, n_pages=10, max_pages=4, dk=128) == 0   # an unfinished layer
    pool = q.KvConfig(page=16, n_pages=10, max_pages=4, Hq=0, Hkv=0, dk=0, dv=0)
    assert q.new_kv_work(pool, device="cpu").numel() >= 4096
    with pytest.raises(q.QstateError):
        q.new_kv_work(q.KvConfig(page=3, n_pages=10, max_pages=4, Hq=0, Hkv=0, dk=0, dv=0), device="cpu")


def test_arrays_of_words_that_are_not_aligned_are_refused(q):
    L, c, r = q._lib, config(q), ct.byref
    cache = q._KvCache(A, A, None, None)
    for i in range(3):
        at = [A + 2 * (i == j) for j in range(3)]   # table, lens, lse
        assert L.qstate_kv_attend(r(c._c), r(cache), A, 1024, 128, at[0], at[1], 1, A, at[2], A, None) == q.QSTATE_EINVAL
        assert b"4-byte" in L.qstate_last_error()
    assert L.qstate_kv_append(r(c._c), r(cache), A, 256, 128, A, 256, 128, A + 1, 1, None) == q.QSTATE_EINVAL
    assert b"4-byte" in L.qstate_last_error()
    for i in range(11):
        at = [A + 2 * (i == j) for j in range(11)]
        pages, slots = q._KvPages(*at[:6]), q._KvSlots(*at[6:10], A, 1)
        assert L.qstate_kv_plan(r(c._c), r(pages), at[10], 1, r(slots), A, None) == q.QSTATE_EINVAL
        assert b"4-byte" in L.qstate_last_error()


def test_the_last_tile_of_the_longest_request_ends_within_32_bits(q):
    """Tiles have up to 128 tokens: with 2^31 - 1 tokens the places behind the last one would be negative numbers."""
    for page, columns in ((1, 2 ** 31 - 1), (1, 2 ** 31 - 1023), (64, 2 ** 25 - 15), (64, 2 ** 25 - 1)):
        with pytest.raises(q.QstateError):
            q.kv_validate(config(q, page=page, max_pages=columns))
    for page, columns in ((1, 2 ** 31 - 1024), (64, 2 ** 25 - 16), (1024, 2 ** 21 - 1)):
        q.kv_validate(config(q, page=page, max_pages=columns))
