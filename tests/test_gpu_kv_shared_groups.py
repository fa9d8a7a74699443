"""Attention over shared tokens with groups that were made for something else, and in work spaces that served other calls: every request
is answered in full, and what does not fit is reported."""
import pytest
import torch

import kv_share_reference as share

pytestmark = pytest.mark.gpu

# requests that have no token of their own (as right after a fork), some with, one that is empty, one by itself
LENS = [280, 280, 305, 0, 280, 90]
GROUPS = [(0, 5, 280)]


@pytest.fixture(autouse=True)
def share_everything(qs):
    """Groups share whatever it costs: the cases here are small."""
    qs.qstate_set_shared_gain(0)
    yield
    qs.qstate_set_shared_gain(-1)


def litter(b, seed):
    """What an earlier call may have left behind the counters: any bits, those of floats among them."""
    g = torch.Generator().manual_seed(seed)
    words = b.work.view(torch.int32)[1024:]
    words.copy_(torch.randint(0, 2 ** 31 - 1, words.shape, generator=g, dtype=torch.int32))


def raw(qs, groups, R):
    """The same bytes, as a caller of the C interface has them: nothing on the host knows what they were made for."""
    return qs.KvGroups(groups.data.clone(), R)


def attend(qs, b, groups):
    b.o.fill_(9.0)
    b.lse.fill_(9.0)
    qs.qstate_kv_attend_shared(b.cfg, b.cache, b.q, b.d_table, b.d_lens, groups, b.o, b.lse, b.work)


def reported(qs, b, groups):
    """The status is set, and the answers are those of requests that share nothing."""
    attend(qs, b, groups)
    with pytest.raises(qs.QstateError) as e:
        qs.qstate_check()
    assert e.value.code == qs.QSTATE_EDEVICE
    b.check(qs)


@pytest.mark.parametrize("kind,d", [("bf16", 64), ("bf16", 128), ("f16", 128), ("e4m3", 64), ("bf16", 256), ("e4m3", 256)])
@pytest.mark.parametrize("lens", [LENS, [40, 40, 44, 0, 40, 7]], ids=["split", "whole"])
def test_groups_of_other_heads_count_as_none(qs, kind, d, lens):
    """A request whose tokens are all shared has no work of its own; where the groups are none it reads them all."""
    groups = [(0, 5, lens[0])]
    make = lambda Hq: share.Batch(qs, lens, groups, Hq, 2, d, dtype="f16" if kind == "f16" else "bf16", e4m3=kind == "e4m3",  # noqa: E731
                                  seed=d)
    b, other = make(4), make(8)
    other.group(qs)
    for seed in range(3):
        litter(b, seed)
        reported(qs, b, raw(qs, other.d_groups, len(lens)))
    litter(b, 9)
    b.run(qs)
    b.check(qs)


def test_groups_of_fewer_requests_count_as_none(qs):
    b = share.Batch(qs, LENS, GROUPS, 4, 2, 64, seed=3)
    few = share.Batch(qs, LENS[:3], [(0, 3, 280)], 4, 2, 64, seed=3)
    few.group(qs)
    data = torch.zeros_like(b.d_groups.data)
    data[: few.d_groups.data.numel()] = few.d_groups.data
    litter(b, 1)
    reported(qs, b, qs.KvGroups(data, len(LENS)))


def test_a_work_space_of_more_requests_and_other_heads(qs):
    """A large call leaves sums, references and places all over; a small one of another layout reads only what it wrote itself."""
    large = share.Batch(qs, [300 + 5 * i for i in range(20)], [(0, 20, 290)], 32, 8, 128, seed=4)
    for kind in ("bf16", "e4m3"):
        b = share.Batch(qs, LENS, GROUPS, 8, 2, 128, e4m3=kind == "e4m3", seed=5)
        other = share.Batch(qs, LENS, GROUPS, 16, 2, 128, e4m3=kind == "e4m3", seed=5)
        other.group(qs)
        large.run(qs)
        b.work = large.work
        reported(qs, b, raw(qs, other.d_groups, len(LENS)))
        large.run(qs)
        b.run(qs)
        b.check(qs)
    large.run(qs)
    large.check(qs)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_wait_that_gives_up_at_once_reads_no_part_that_nobody_wrote(qs, kind):
    """A limit of 0: reported, and the tokens are read as if nothing were shared."""
    large = share.Batch(qs, [300 + 5 * i for i in range(20)], [(0, 20, 290)], 32, 8, 128, seed=6)
    b = share.Batch(qs, LENS, GROUPS, 32, 8, 128, e4m3=kind == "e4m3", seed=7)
    b.group(qs)

    def gives_up():
        qs.qstate_set_wait_limit(0)
        try:
            attend(qs, b, b.d_groups)
            with pytest.raises(qs.QstateError) as e:
                qs.qstate_check()
            assert e.value.code == qs.QSTATE_ETIMEOUT
        finally:
            qs.qstate_set_wait_limit(-1)
        b.check(qs)

    for seed in range(3):
        litter(b, seed)
        gives_up()
    large.run(qs)
    b.work = large.work
    gives_up()
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("made,used", [(0, 200), (200, 0), (100, 250), (10000, 0)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_groups_of_another_window_count_as_none(qs, made, used, kind):
    """Layers with a window and without one stand beside each other: groups of one are not the other's, though nothing else differs."""
    lens = [200, 230, 305, 0, 280, 90]
    make = lambda w: share.Batch(qs, lens, [(0, 5, 180)], 8, 2, 64, window=w, e4m3=kind == "e4m3", seed=8)  # noqa: E731
    b, other = make(used), make(made)
    other.group(qs)
    with pytest.raises(ValueError):   # the binding knows what they were made for
        attend(qs, b, other.d_groups)
    if int(other.d_groups.data[:4].view(torch.int32).item()) == 0:   # nothing is shared, whoever looks at it
        attend(qs, b, raw(qs, other.d_groups, len(lens)))
    else:
        reported(qs, b, raw(qs, other.d_groups, len(lens)))
    b.run(qs)
    b.check(qs)


@pytest.mark.parametrize("made,used", [(64, 128), (128, 64), (256, 128)])
def test_groups_of_another_width_count_as_none(qs, made, used):
    b, other = (share.Batch(qs, LENS, GROUPS, 8, 2, d, seed=9) for d in (used, made))
    other.group(qs)
    reported(qs, b, raw(qs, other.d_groups, len(LENS)))


def test_groups_serve_layers_of_other_pages(qs):
    """What is shared is counted in tokens: tables of other pages may be read with the same groups."""
    made = share.Batch(qs, LENS, GROUPS, 8, 2, 128, page=16, seed=10)
    made.group(qs)
    for page in (1, 64, 256):
        b = share.Batch(qs, LENS, GROUPS, 8, 2, 128, page=page, seed=page)
        for groups in (made.d_groups, raw(qs, made.d_groups, len(LENS))):
            attend(qs, b, groups)
            b.check(qs)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_common_tokens_behind_the_table_count_as_none(qs, kind):
    """Groups with more in common than a row of this layer's table holds: nothing is looked up behind it."""
    made = share.Batch(qs, LENS, GROUPS, 8, 2, 64, page=16, e4m3=kind == "e4m3", seed=11)
    b = share.Batch(qs, [40, 40, 44, 0, 40, 7], [(0, 5, 40)], 8, 2, 64, page=16, e4m3=kind == "e4m3", seed=12)
    assert b.cfg.max_pages * 16 < 280
    made.group(qs)
    for groups in (made.d_groups, raw(qs, made.d_groups, len(LENS))):
        reported(qs, b, groups)
    b.run(qs)
    b.check(qs)
