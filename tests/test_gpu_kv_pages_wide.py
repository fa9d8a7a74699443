"""Fork and compact over the widest table that a description allows: its last columns lie just below 2^31."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


def same_as_range(x, first):
    """x[i] = first + i, looked at in pieces."""
    step = 1 << 28
    return all(torch.equal(x[i:i + step], torch.arange(first + i, first + min(i + step, x.numel()), dtype=torch.int32, device="cuda"))
               for i in range(0, x.numel(), step))


def test_the_last_columns_of_the_widest_table(qs):
    """One request that holds a page of one token in every column.  Parts of the columns, 2^18 each, end at 2^31."""
    if torch.cuda.mem_get_info()[0] < 70e9:
        pytest.skip("needs 60 GB")
    width, n_pages = 2 ** 31 - 1024, 2 ** 31 - 1
    cfg = qs.KvConfig(page=1, n_pages=n_pages, max_pages=width)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(width, dtype=torch.int32, device="cuda").view(1, width)
    free_list = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free_list[:1023] = torch.arange(width, n_pages, dtype=torch.int32, device="cuda")
    others = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    pages, lens_out, free_out, left = qs.KvPages(table, i32(width), free_list, i32(1023)), i32(-1), i32(-1), i32(-1)
    work, moves, ok = qs.new_kv_pages_work(cfg, 1), qs.new_kv_moves(4), torch.zeros(1, dtype=torch.uint8, device="cuda")
    # every column's page is held: those that are not are the free ones, the lowest on top
    qs.qstate_kv_compact(cfg, pages, others, n_pages, moves, left, work, free_out=free_out)
    qs.qstate_check()
    assert free_out.item() == 1023 and left.item() == 0 and moves.src.tolist() == [-1] * 4
    assert same_as_range(free_list[:1023].flip(0), width)
    # one page behind the limit, in the last column, goes to the one place in front of it
    table[0, width - 1], table[0, 7] = n_pages - 1, width - 1
    qs.qstate_kv_compact(cfg, pages, others, width, moves, left, work, free_out=free_out)
    qs.qstate_check()
    assert moves.src.tolist() == [n_pages - 1, -1, -1, -1] and moves.dst.tolist() == [7, -1, -1, -1]
    assert (free_out.item(), left.item(), table[0, width - 1].item()) == (0, 0, 7)
    table[0, 7], table[0, width - 1] = 7, width - 1
    free_list[:1023] = torch.arange(width, n_pages, dtype=torch.int32, device="cuda")
    # half of it goes on, and what is behind comes back
    keep = 2 ** 30 + 5
    qs.qstate_kv_fork(cfg, pages, others, i32(0), i32(keep), moves, ok, work, lens_out=lens_out, free_out=free_out)
    qs.qstate_check()
    assert (lens_out.item(), free_out.item(), ok.item()) == (keep, 1023 + width - keep, 1)
    assert same_as_range(free_list[1023:1023 + width - keep], keep)
    # and all of it ends
    qs.qstate_kv_fork(cfg, pages, others, i32(-1), None, moves, ok, work, lens_out=lens_out, free_out=free_out)
    qs.qstate_check()
    assert (lens_out.item(), free_out.item()) == (0, 1023 + width)
    assert same_as_range(free_list[1023:1023 + width], 0)
    assert not bool(others.any())


def test_the_longest_list_of_moves(qs):
    """2^31 - 1 entries, of which none is needed: all are -1, and nothing in front of the list is touched."""
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 20 GB")
    n = 2 ** 31 - 1
    cfg = qs.KvConfig(page=4, n_pages=6, max_pages=2)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    front = 1 << 20   # words in front of each list, which a step above 2^31 would reach
    room = [torch.full((front + n,), 5, dtype=torch.int32, device="cuda") for _ in range(2)]
    moves = qs.KvMoves(*(x[front:] for x in room))
    pages = qs.KvPages(i32(), i32(), i32(3, 1, 2, 0, 4, 5), i32(4))
    others, work = torch.zeros(6, dtype=torch.int32, device="cuda"), qs.new_kv_pages_work(cfg, 0)
    for call in (lambda: qs.qstate_kv_compact(cfg, pages, None, 5, moves, None, work),
                 lambda: qs.qstate_kv_fork(cfg, pages, others, i32(), None, moves, torch.zeros(0, dtype=torch.uint8, device="cuda"), work)):
        for x in room:
            x.fill_(5)
        call()
        qs.qstate_check()
        for x in room:
            step = 1 << 28
            assert bool((x[:front] == 5).all())
            assert all(bool((x[i:i + step] == -1).all()) for i in range(front, front + n, step))
