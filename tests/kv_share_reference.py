"""Requests that hold pages together, in plain loops, and batches that share their first tokens."""
import random

import torch

import kv_reference as ref

pages_of = ref.pages_of


def fork(lens, table, free_list, free, others, parent, keep, page):
    """Lists in (changed in place: table, free_list, others); a dict of the rest out."""
    R, n_pages = len(lens), len(others)
    old = [table[r][: pages_of(lens[r], page)] for r in range(R)]
    rows = [list(t) for t in table]
    m = []
    for r, p in enumerate(parent):
        n = lens[p] if p >= 0 else 0
        m.append(min(n, keep[r]) if keep is not None and keep[r] >= 0 else n)
    # who goes on with the page of parent p that it is cut in
    goes_on = {}
    for p in range(R):
        heirs = [r for r in range(R) if parent[r] == p]
        deepest = max([m[r] // page for r in heirs], default=0)
        able = [r for r in heirs if m[r] % page and m[r] // page == deepest and others[rows[p][deepest]] == 0]
        if able:
            goes_on[p] = p if p in able else able[0]
    src, dst, ok, new, fresh, top, asked = [-1] * R, [-1] * R, [1] * R, [], set(), free, 0
    for r, p in enumerate(parent):
        w = m[r] // page
        mine = rows[p][:w] if p >= 0 else []
        if m[r] % page:
            if goes_on.get(p) == r:
                mine = mine + [rows[p][w]]
            else:
                asked += 1
                if asked <= free:
                    top -= 1
                    src[r], dst[r] = rows[p][w], free_list[top]
                    fresh.add(dst[r])
                    mine = mine + [dst[r]]
                else:
                    ok[r], m[r], mine = 0, 0, []
        new.append(mine)
    change = [0] * n_pages
    last = {x: r for r in range(R) for x in old[r]}   # who held it last
    for r in range(R):
        for x in old[r]:
            change[x] -= 1
        for x in new[r]:
            change[x] += x not in fresh or x in last
    count = top
    for r in range(R):
        for x in old[r]:
            if others[x] + change[x] == -1 and last[x] == r:
                free_list[count] = x
                count += 1
    for x in range(n_pages):
        others[x] = max(others[x] + change[x], 0) if x in last else 0
    for r in range(R):
        table[r][: len(new[r])] = new[r]
    return dict(lens=m, free=count, src=src, dst=dst, ok=ok)


def compact(lens, table, table_out, free_list, others, limit, many, page):
    n_pages = len(others)
    held = set(x for r, n in enumerate(lens) for x in table[r][: pages_of(n, page)])
    source = [x for x in range(limit, n_pages) if x in held]
    place = [x for x in range(limit) if x not in held]
    k = min(len(source), len(place), many)
    to = {x: y for x, y in zip(source[:k], place[:k])}
    for r, n in enumerate(lens):
        for c in range(pages_of(n, page)):
            table_out[r][c] = to.get(table[r][c], table[r][c])
    for x, y in to.items():
        others[y], others[x] = others[x], 0
    rest = place[k:]
    for i, x in enumerate(reversed(rest)):
        free_list[i] = x
    return dict(free=len(rest), left=len(source) - k, src=source[:k] + [-1] * (many - k), dst=place[:k] + [-1] * (many - k))


class Pool:
    """Tables of requests that hold pages together, on the host and on the device, changed by both alike."""

    def __init__(self, qs, R, page, n_pages, max_pages, seed, device="cuda"):
        self.qs, self.R, self.page, self.device = qs, R, page, device
        self.rng = random.Random(seed)
        self.cfg = qs.KvConfig(page=page, n_pages=n_pages, max_pages=max_pages)
        ids = list(range(n_pages))
        self.rng.shuffle(ids)
        self.lens, self.table, self.others = [0] * R, [[-5] * max_pages for _ in range(R)], [0] * n_pages
        self.free_list, self.free = ids, n_pages
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
        self.pages = qs.KvPages(i32(self.table).reshape(R, max_pages), i32(self.lens), i32(ids), i32([n_pages]))
        self.d_others = i32(self.others)
        self.work = qs.new_kv_pages_work(self.cfg, R, device=device)
        self.plan_work = qs.new_kv_work(self.cfg, device=device)
        self.ok = torch.zeros(R, dtype=torch.uint8, device=device)
        self.i32 = i32

    def grow(self, new, T=None):
        """qstate_kv_plan; nobody ends by it here."""
        T = sum(new) if T is None else T
        slots = self.qs.new_kv_slots(self.R, T, device=self.device)
        self.qs.qstate_kv_plan(self.cfg, self.pages, self.i32(new), slots, self.plan_work)
        stack = self.free_list[: self.free]
        got = ref.plan(self.lens, new, self.table, stack, self.page, T, self.cfg.max_pages)
        self.lens, self.free = got["lens"], len(stack)
        self.same()
        return slots, got

    def fork(self, parent, keep=None, spare_moves=0):
        moves = self.qs.new_kv_moves(self.R + spare_moves, device=self.device)
        moves.src.fill_(99), moves.dst.fill_(99)
        self.qs.qstate_kv_fork(self.cfg, self.pages, self.d_others, self.i32(parent), None if keep is None else self.i32(keep), moves,
                               self.ok, self.work)
        got = fork(self.lens, self.table, self.free_list, self.free, self.others, parent, keep, self.page)
        self.lens, self.free = got["lens"], got["free"]
        tail = [-1] * spare_moves
        assert moves.src.tolist() == got["src"] + tail and moves.dst.tolist() == got["dst"] + tail
        assert self.ok.tolist() == got["ok"]
        self.same()
        return moves, got

    def compact(self, limit, many, apart=False):
        moves, left = self.qs.new_kv_moves(many, device=self.device), self.i32([-3])
        out = torch.full_like(self.pages.table, -9) if apart else None
        self.qs.qstate_kv_compact(self.cfg, self.pages, self.d_others, limit, moves, left, self.work, table_out=out)
        to = [[-9] * self.cfg.max_pages for _ in self.table] if apart else self.table
        got = compact(self.lens, self.table, to, self.free_list, self.others, limit, many, self.page)
        assert left.tolist() == [got["left"]] and moves.src.tolist() == got["src"] and moves.dst.tolist() == got["dst"]
        if apart:
            assert out.tolist() == to
            self.pages.table.copy_(out)
            self.table = to
        self.free = got["free"]
        self.same()
        return moves, got

    def same(self):
        assert self.pages.lens.tolist() == self.lens
        assert self.pages.free_count.tolist() == [self.free]
        assert self.pages.free_list.tolist() == self.free_list
        assert self.d_others.tolist() == self.others
        assert self.pages.table.tolist() == self.table

    def sound(self):
        """Every page is held as often as `others` says, or once on the list."""
        held = [0] * len(self.others)
        for r, n in enumerate(self.lens):
            for x in self.table[r][: pages_of(n, self.page)]:
                held[x] += 1
        for x, h in enumerate(held):
            assert self.others[x] == max(h - 1, 0)
        stack = self.free_list[: self.free]
        assert sorted(stack) == [x for x, h in enumerate(held) if h == 0]


class Batch(ref.Batch):
    """A batch whose groups (first request, one behind the last, tokens in common) have those tokens alike: whole pages held
    together, the page that they end in a copy each."""

    def __init__(self, qs, lens, groups, *args, **kw):
        super().__init__(qs, lens, *args, **kw)
        page, c = self.cfg.page, self.cfg
        self.groups = groups
        exps = [self.cache.k_exp, self.cache.v_exp]
        for a, b, common in groups:
            having = [r for r in range(a, b) if lens[r] >= common]
            if not having or common == 0:
                continue
            first = having[0]
            whole, rest = common // page, common % page
            for r in range(a, b):
                n = min(lens[r], common)
                for col in range(pages_of(n, page)):
                    x, y = self.table[r][col], self.table[first][col]
                    if x == y:
                        continue
                    many = min(page, n - col * page)
                    if many == page and col < whole:
                        self.table[r][col] = y
                        continue
                    for t in (self.k, self.v, *exps):
                        if t is not None:
                            z = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
                            z[x, :, :many] = z[y, :, :many]
                    self.kval[x, :, :many] = self.kval[y, :, :many]
                    self.vval[x, :, :many] = self.vval[y, :, :many]
        dev = self.q.device
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        self.d_table = i32(self.table).reshape(len(lens), c.max_pages)
        starts, commons, at = [0], [], 0
        for a, b, common in groups:   # what lies between groups is a group with nothing in common
            if a > at:
                starts.append(a)
                commons.append(0)
            starts.append(b)
            commons.append(common)
            at = b
        self.start, self.common = i32(starts), i32(commons)
        self.d_groups = qs.new_kv_groups(self.cfg, len(lens), device=dev)
        self.work = qs.new_kv_shared_work(self.cfg, len(lens), device=dev)

    def group(self, qs, stream=None):
        qs.qstate_kv_group(self.cfg, self.d_lens, self.start, self.common, self.d_groups, stream=stream)

    def attend(self, qs, stream=None):
        qs.qstate_kv_attend_shared(self.cfg, self.cache, self.q, self.d_table, self.d_lens, self.d_groups, self.o, self.lse, self.work,
                                   stream=stream)

    def run(self, qs, stream=None):
        self.group(qs, stream)
        self.attend(qs, stream)

    def expect(self):
        """On the device: the batches of several tiles a worker are large."""
        if self.kval.device != self.q.device:
            self.kval, self.vval, self.qval = (x.to(self.q.device) for x in (self.kval, self.vval, self.qval))
        with torch.device(self.q.device):
            return tuple(x.cpu() for x in super().expect())
