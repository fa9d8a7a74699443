"""The calls on shared pages as a program uses them: samples of prompts that grow, split, end and move, over two kinds of layers, against
plain attention in 64 bits over the keys and values that each request was given."""
import random

import pytest
import torch

import kv_reference as ref
import kv_share_reference as share
from test_gpu_hybrid_example import attention

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def share_everything(qs):
    """Groups share whatever it costs: the cases here are small."""
    qs.qstate_set_shared_gain(0)
    yield
    qs.qstate_set_shared_gain(-1)


class Layer:
    def __init__(self, qs, pool, e4m3, d, seed):
        self.qs, self.e4m3 = qs, e4m3
        c = pool.cfg
        self.cfg = qs.KvConfig(Hq=8, Hkv=2, dk=d, dv=d, page=c.page, n_pages=c.n_pages, max_pages=c.max_pages, scale=d ** -0.5,
                               store=qs.KV_E4M3 if e4m3 else qs.KV_16)
        self.cache, self.groups = qs.new_kv_cache(self.cfg), qs.new_kv_groups(self.cfg, pool.R)
        for t in (self.cache.k, self.cache.v):   # what nobody wrote must not count
            t.view(torch.uint8).fill_(0x7F)
        self.work = qs.new_kv_shared_work(self.cfg, pool.R)
        self.g = torch.Generator().manual_seed(seed)
        self.held = [[] for _ in range(pool.R)]   # each request's keys and values, as the cache holds them

    def append(self, slots, rows):
        """rows: of each slot, its request (those that are granted)."""
        d, T = self.cfg.dk, slots.slot.numel()
        k, v = (torch.randn(T, 2, d, generator=self.g).to(torch.bfloat16) for _ in range(2))
        self.qs.qstate_kv_append(self.cfg, self.cache, k.cuda(), v.cuda(), slots.slot)
        for t, r in enumerate(rows):
            if r >= 0:
                pair = [x[t] for x in (k, v)]
                if self.e4m3:
                    pair = [x * torch.exp2(e.double() - 127)[..., None] for x, e in map(ref.quantise, pair)]
                self.held[r].append([x.double() for x in pair])

    def take_over(self, parent, lens):
        old = self.held
        self.held = [list(old[p][:n]) if p >= 0 else [] for p, n in zip(parent, lens)]

    def attend(self, pool, start, common):
        R, d = pool.R, self.cfg.dk
        q = torch.randn(R, 8, d, generator=self.g).to(torch.bfloat16)
        o = torch.full((R, 8, d), 9.0, dtype=torch.bfloat16, device="cuda")
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.qs.qstate_kv_group(self.cfg, pool.pages.lens, i32(start), i32(common), self.groups)
        self.qs.qstate_kv_attend_shared(self.cfg, self.cache, q.cuda(), pool.pages.table, pool.pages.lens, self.groups, o, None, self.work)
        o = o.double().cpu()
        for r in range(R):
            if not self.held[r]:
                assert not bool(o[r].any())
                continue
            K, V = (torch.stack([x[i] for x in self.held[r]]) for i in range(2))
            want, bound = attention(q[r], K, V, self.cfg.scale)
            assert bool(((o[r] - want).abs() <= bound).all()), r


@pytest.mark.parametrize("page,seed", [(4, 1), (16, 2), (64, 3)])
def test_samples_that_grow_split_end_and_move(qs, page, seed):
    R = 12   # two families of six; the first of each holds the prompt
    pool = share.Pool(qs, R, page, 9000 // page, 1000 // page, seed)
    layers = [Layer(qs, pool, False, 64, seed), Layer(qs, pool, True, 128, seed + 10)]
    rng = random.Random(seed)

    def grow(new):
        slots, got = pool.grow(new)
        rows = [r if s >= 0 else -1 for r, s in zip(got["req"], got["slot"])]
        for x in layers:
            x.append(slots, rows)

    def move(moves):
        for x in layers:
            qs.qstate_kv_copy(x.cfg, x.cache, moves)

    prompts = [301, 170]
    grow([prompts[0]] + [0] * 5 + [prompts[1]] + [0] * 5)
    for step in range(9):
        # samples begin, go on, end, go back to the prompt, or take another's place
        parent, keep = [], []
        for r in range(R):
            first = r // 6 * 6
            kind = 0.9 if r == first else rng.random()
            if not pool.lens[r] or kind < 0.15:
                parent.append(first)
                keep.append(prompts[r // 6])
            else:
                parent.append(-1 if kind < 0.25 else first + rng.randrange(1, 6) if kind < 0.4 else r)
                keep.append(-1)
                if parent[-1] >= 0 and not pool.lens[parent[-1]]:
                    parent[-1], keep[-1] = first, prompts[r // 6]
        moves, got = pool.fork(parent, keep)
        for x in layers:
            x.take_over(parent, pool.lens)
        move(moves)
        grow([rng.randrange(1, 5) if n and r % 6 else 0 for r, n in enumerate(pool.lens)])
        if step % 4 == 3:
            used = len(set(x for r, n in enumerate(pool.lens) for x in pool.table[r][: ref.pages_of(n, page)]))
            moves, _ = pool.compact(used + 3, 2 * used, apart=step == 3)
            move(moves)
            pool.compact(pool.cfg.n_pages, 0)
        pool.sound()
        for x in layers:
            x.attend(pool, [0, 6, 12], prompts)
    assert max(pool.others) > 0
    qs.qstate_check()
