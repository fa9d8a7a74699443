"""Requests that share what they begin with, as cases that can be timed and compared.

The pages of the attention layers' cache may be held by several requests: samples of one prompt, beams, users
behind one system prompt.  A case names one of the operators that this takes (``do``):

* ``fork``     requests take over the first tokens of others (or of themselves, or nothing): whole pages are held
               together, the page that is cut gets a copy, pages that nobody holds any more go on the free list;
* ``copy``     the pages that fork or compact moved, in one layer's cache;
* ``compact``  requests' pages move to the pool's low end, so that the pool can be cut to fewer pages;
* ``shared``   one new token of each request against its pages, where groups of requests have their first tokens in
               common: those are read once for the whole group.

``run`` makes the calls of the library where ``own`` is true, and else computes the same in elementary
torch operations.
"""
import math
import types

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # a step of a beam search: 16 requests of four beams that change places; launches and latency
        dict(name="fork_beams", do="fork", families=16, fan=4, page=16, prefix=1000, own=300, mix="beams", spare=1.0),
        # a large batch of samples: some end, some go back to an earlier token, some start from another's prompt
        dict(name="fork_samples", do="fork", families=75, fan=13, page=32, prefix=16000, own=5000, mix="samples", spare=0.4),
        # the pages that a fork of 48 requests cut, in a layer of four heads of 64
        dict(name="copy_fork", do="copy", moves=48, padding=0.25, Hkv=4, d=64, page=16, type="f16", store="16"),
        # a third of a large pool moves, keys and values in eight bits
        dict(name="copy_e4m3", do="copy", moves=2501, padding=0.0, Hkv=8, d=128, page=32, type="bf16", store="e4m3"),
        # a small pool
        dict(name="compact_small", do="compact", families=9, fan=3, page=16, prefix=500, own=300, full=0.6),
        # a pool of some hundred thousand pages, half of them held
        dict(name="compact_large", do="compact", families=60, fan=12, page=16, prefix=9000, own=2000, full=0.5),
        # four samples of one prompt: few rows, so that the cache's length has to be split
        dict(name="shared_few", do="shared", groups=1, members=4, alone=0, Hq=32, Hkv=8, d=128, page=16, prefix=3001, own=60,
             window=0, type="bf16", store="16"),
        # the full decode batch behind one system prompt, 32 heads
        dict(name="shared_batch", do="shared", groups=1, members=256, alone=0, Hq=32, Hkv=8, d=128, page=64, prefix=8192, own=250,
             window=0, type="bf16", store="16"),
        # several prompts, eight samples of each, heads of 64, and requests by themselves between them
        dict(name="shared_groups", do="shared", groups=12, members=8, alone=5, Hq=40, Hkv=8, d=64, page=32, prefix=15000, own=900,
             window=0, type="f16", store="16"),
        # one very long document, sixteen query heads to a key head
        dict(name="shared_long", do="shared", groups=1, members=19, alone=1, Hq=64, Hkv=4, d=128, page=128, prefix=100000, own=700,
             window=0, type="bf16", store="16"),
        # a cache in eight bits
        dict(name="shared_e4m3", do="shared", groups=2, members=37, alone=2, Hq=48, Hkv=8, d=128, page=32, prefix=12001, own=400,
             window=0, type="bf16", store="e4m3"),
        # heads of 256
        dict(name="shared_wide", do="shared", groups=3, members=21, alone=0, Hq=16, Hkv=2, d=256, page=64, prefix=20000, own=333,
             window=0, type="bf16", store="16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))

    do = rng.choice(["fork", "fork", "copy", "compact", "shared", "shared", "shared", "shared"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if do in ("fork", "compact"):
        families, fan = log_int(1, 100), log_int(1, 16)
        prefix, own_tokens = log_int(1, 16000), log_int(1, 5000)
        case = dict(do=do, families=families, fan=fan, page=page, prefix=prefix, own=own_tokens)
        if do == "fork":
            return dict(case, mix=rng.choice(["beams", "samples"]), spare=rng.choice([1.0, 0.4, 0.1]))
        return dict(case, full=rng.choice([0.3, 0.5, 0.9]))
    if do == "copy":
        Hkv, d, store = log_int(1, 16), rng.choice([64, 128, 128, 256]), rng.choice(["16", "16", "e4m3"])
        return dict(do=do, moves=log_int(1, max(1, 80_000_000 // (Hkv * d * page))), padding=rng.choice([0.0, 0.3]), Hkv=Hkv, d=d,
                    page=page, type="bf16" if store == "e4m3" else rng.choice(["bf16", "f16"]), store=store)
    Hkv, d, store = log_int(1, 16), rng.choice([64, 128, 128, 128, 256]), rng.choice(["16", "16", "e4m3"])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 6, 8, 16])
    groups, members = log_int(1, 12), log_int(2, 128)
    rows = groups * members
    own_tokens = log_int(1, max(1, min(3000, 100_000_000 // (rows * Hkv * d))))
    most = min(100000, 80_000_000 // (groups * Hkv * d), 6_000_000_000 // (rows * Hq * d))
    return dict(do=do, groups=groups, members=members, alone=rng.choice([0, 0, 1, 5]), Hq=Hq, Hkv=Hkv, d=d, page=page,
                prefix=log_int(1, max(1, most)), own=own_tokens, window=rng.choice([0, 0, 0, log_int(1, 30000)]),
                type="bf16" if store == "e4m3" else rng.choice(["bf16", "f16"]), store=store)


# ---- inputs --------------------------------------------------------------------------------------------


def family_sizes(case):
    """(whole pages that a family has in common, tokens of each of its requests behind them), family after family"""
    page, fan = case["page"], case["fan"]
    common = [case["prefix"] * (f + 1) // case["families"] // page for f in range(case["families"])]
    behind = [-(-case["own"] * (i + 1) // fan) for i in range(fan)]
    return common, behind


def pages_of(n, page):
    return -(-n // page)


def pool_pages(case):
    """(pages that are held, pages of the pool)"""
    common, behind = family_sizes(case)
    used = sum(common) + case["families"] * sum(pages_of(n, case["page"]) for n in behind)
    if case["do"] == "fork":
        return used, used + max(1, int(math.ceil(case["spare"] * case["families"] * case["fan"])))
    return used, max(used + 1, int(used / case["full"]))


def shared_lengths(case):
    """(first request, one behind the last, tokens in common) of each group, and all requests' lengths: the first of a
    group has just been forked, where a group has eight and more one request of it is empty; then those by themselves"""
    spans, lens, M = [], [], case["members"]
    for g in range(case["groups"]):
        common = max(1, case["prefix"] * (g + 1) // case["groups"])
        spans.append((len(lens), len(lens) + M, common))
        n = [common + case["own"] * i // max(1, M - 1) for i in range(M)]
        if M >= 8:
            n[1] = 0
        lens += n
    for i in range(case["alone"]):
        lens.append(case["own"] * i)
    return spans, lens


def split_e4m3(x):
    """Codes of x's last axis and the exponent byte k + 127 of each vector: the smallest power of two 2^k
    with |x| <= 448 * 2^k."""
    x = x.float()
    top = x.abs().amax(-1)
    mant, ex = torch.frexp(top)
    k = torch.where(top > 0, ex - 9 + (mant > 0.875).int(), 0).clamp(-126, 120).int()
    return (x * ((127 - k) << 23).view(torch.float32)[..., None]).to(E4M3), (k + 127).to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    perm = lambda n: torch.randperm(n, device="cuda", generator=gen)  # noqa: E731
    upto = lambda hi, *s: torch.randint(0, hi, s, device="cuda", generator=gen)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = types.SimpleNamespace(case=case, do=case["do"], page=case["page"])
    if s.do in ("fork", "compact"):
        families(s, case, perm, ints)
        if s.do == "fork":
            R, fan = s.R, case["fan"]
            row = torch.arange(R, device="cuda")
            parent, keep = row // fan * fan + upto(fan, R), torch.full((R,), -1, device="cuda")
            if case["mix"] == "samples":
                kind = upto(16, R)   # most go on as they are
                parent = torch.where(kind < 3, parent, row)
                parent = torch.where(kind == 3, -1, parent)
                keep = torch.where((kind < 2) | (kind == 4), upto(case["prefix"] + case["own"], R), keep)
            s.parent, s.keep = parent.int(), keep.int()
        else:
            s.limit = min(s.n_pages, s.used + 1 + s.used // 50)
            s.table_out, s.left = torch.full_like(s.table, -1), ints([0])
        n = s.R if s.do == "fork" else s.used
        s.src, s.dst = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
        s.lens_out, s.free_out = torch.empty_like(s.lens), torch.empty_like(s.free)
        s.ok = torch.empty(s.R, dtype=torch.uint8, device="cuda")
        return s
    s.type, s.e4m3, s.Hkv, s.d = TYPES[case["type"]], case["store"] == "e4m3", case["Hkv"], case["d"]
    loud = torch.exp(0.5 * rnd(s.Hkv, s.d))   # keys have a few channels much larger than the rest
    if s.do == "copy":
        n = case["moves"]
        s.n_pages = 3 * n + 1
        ids = perm(s.n_pages)
        s.src, s.dst = ids[:n].int(), ids[n:2 * n].int()
        idle = perm(n)[: int(n * case["padding"])]   # requests that needed no copy
        s.src[idle] = s.dst[idle] = -1
    else:
        s.Hq, s.window, s.scale = case["Hq"], case["window"], s.d ** -0.5
        s.spans, lens = shared_lengths(case)
        s.B, s.longest = len(lens), max(1, max(lens))
        s.lens = ints(lens)
        s.start, s.common = ints([a for a, _, _ in s.spans] + [s.spans[-1][1]]), ints([c for _, _, c in s.spans])
        shared_table(s, lens, perm)
    shape = (s.n_pages, s.Hkv, s.page, s.d)

    def pool(many):
        x = torch.empty(shape, dtype=E4M3 if s.e4m3 else s.type, device="cuda")
        e = torch.empty(shape[:3], dtype=torch.uint8, device="cuda") if s.e4m3 else None
        step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
        for at in range(0, s.n_pages, step):
            y = rnd(min(step, s.n_pages - at), *shape[1:]) * many
            if s.e4m3:
                x[at:at + step], e[at:at + step] = split_e4m3(y)
            else:
                x[at:at + step] = y
        return x, e

    (s.kc, s.ke), (s.vc, s.ve) = pool(loud[:, None]), pool(1.0)
    if s.do == "copy":
        return s
    for x in (s.kc, s.vc, s.ke, s.ve):   # each has a copy of the page that the common tokens end in
        if x is not None:
            y = x.view(torch.uint8) if s.e4m3 else x
            for mine, first in s.cut:
                y[mine] = y[first]
    s.q = (2.0 * rnd(s.B, s.Hq, s.d)).to(s.type)
    s.o = torch.empty((s.B, s.Hq, s.d), dtype=s.type, device="cuda")
    s.lse = torch.empty((s.B, s.Hq), dtype=torch.float32, device="cuda")
    return s


def families(s, case, perm, ints):
    """Requests in families that hold their first pages together; the pool's other pages on the free list."""
    page, fan, F = case["page"], case["fan"], case["families"]
    common, behind = family_sizes(case)
    s.R = F * fan
    s.used, s.n_pages = pool_pages(case)
    n = ints([c * page + b for c in common for b in behind])
    c = ints([c for c in common for _ in behind]).long()
    s.lens = n
    many = (n.long() + page - 1) // page
    s.width = max(common) + pages_of(max(behind), page) + 1
    family = torch.arange(s.R, device="cuda") // fan
    c_family = ints(common).long()
    first = c_family.cumsum(0) - c_family
    mine = many - c
    own_first = int(sum(common)) + mine.cumsum(0) - mine
    col = torch.arange(s.width, device="cuda")[None]
    at = torch.where(col < c[:, None], first[family][:, None] + col, own_first[:, None] + col - c[:, None])
    p = perm(s.n_pages)
    s.table = torch.where(col < many[:, None], p[at.clamp(max=s.n_pages - 1)], -1).int()
    s.others = torch.zeros(s.n_pages, dtype=torch.int32, device="cuda")
    s.others[p[: sum(common)]] = fan - 1
    s.free_list = torch.full((s.n_pages,), -1, dtype=torch.int32, device="cuda")
    s.free_list[: s.n_pages - s.used] = p[s.used:].int()
    s.free = ints([s.n_pages - s.used])


def shared_table(s, lens, perm):
    """Each group's whole common pages are held together; the page that they end in and what follows is each one's."""
    page = s.page
    s.width = pages_of(s.longest, page)
    used = sum(c // page for _, _, c in s.spans)
    rows = [0] * s.B   # whole pages in common
    for a, b, c in s.spans:
        rows[a:b] = [c // page] * (b - a)
    used += sum(max(0, pages_of(n, page) - k) for n, k in zip(lens, rows))
    s.n_pages = used + used // 10 + 1
    ids = perm(s.n_pages).tolist()
    table = [[-1] * s.width for _ in lens]
    s.cut = []
    for a, b, c in s.spans:
        whole = [ids.pop() for _ in range(c // page)]
        for r in range(a, b):
            if lens[r]:
                table[r][: len(whole)] = whole
    for r, n in enumerate(lens):
        for k in range(rows[r], pages_of(n, page)):
            table[r][k] = ids.pop()
    for a, b, c in s.spans:
        if c % page:
            s.cut += [(table[r][c // page], table[a][c // page]) for r in range(a + 1, b) if lens[r]]
    s.table = torch.tensor(table, dtype=torch.int32, device="cuda")


# ---- one pass ------------------------------------------------------------------------------------------


def handles(s):
    """What a program makes once and keeps: descriptions, the cache's and the tables' tensors, work spaces."""
    import paper_2609_30950_gb300 as qs

    s.qs = qs
    if s.do != "shared":
        s.moves = qs.KvMoves(s.src, s.dst)
    if s.do in ("fork", "compact"):
        s.cfg = qs.KvConfig(page=s.page, n_pages=s.n_pages, max_pages=s.width)
        s.pages = qs.KvPages(s.table, s.lens, s.free_list, s.free)
        s.work = qs.new_kv_pages_work(s.cfg, s.R)
        return
    s.cfg = qs.KvConfig(Hq=getattr(s, "Hq", s.Hkv), Hkv=s.Hkv, dk=s.d, dv=s.d, page=s.page, n_pages=s.n_pages,
                        max_pages=getattr(s, "width", s.n_pages), dtype=qs.KV_F16 if s.type == torch.float16 else qs.KV_BF16,
                        store=qs.KV_E4M3 if s.e4m3 else qs.KV_16, window=getattr(s, "window", 0), scale=getattr(s, "scale", 1.0))
    s.cache = qs.KvCache(s.kc, s.vc, s.ke, s.ve)
    if s.do == "shared":
        s.groups, s.work = qs.new_kv_groups(s.cfg, s.B), qs.new_kv_shared_work(s.cfg, s.B)


def run(s):
    if not own:
        return {"fork": plain_fork, "copy": plain_copy, "compact": plain_compact, "shared": plain_shared}[s.do](s)
    if not hasattr(s, "qs"):
        handles(s)
    qs = s.qs
    if s.do == "fork":
        qs.qstate_kv_fork(s.cfg, s.pages, s.others, s.parent, s.keep, s.moves, s.ok, s.work, s.lens_out, s.free_out)
        return forked(s)
    if s.do == "compact":
        qs.qstate_kv_compact(s.cfg, s.pages, s.others, s.limit, s.moves, s.left, s.work, s.table_out, s.free_out)
        return compacted(s)
    if s.do == "copy":
        qs.qstate_kv_copy(s.cfg, s.cache, s.moves)
        return copied(s)
    qs.qstate_kv_group(s.cfg, s.lens, s.start, s.common, s.groups)
    qs.qstate_kv_attend_shared(s.cfg, s.cache, s.q, s.table, s.lens, s.groups, s.o, s.lse, s.work)
    return dict(o=s.o, lse=s.lse)


def forked(s):
    return dict(table=s.table, lens=s.lens_out, others=s.others, free_list=s.free_list, free=s.free_out, src=s.src, dst=s.dst,
                ok=s.ok)


def compacted(s):
    return dict(table=s.table_out, others=s.others, free_list=s.free_list, free=s.free_out, src=s.src, dst=s.dst, left=s.left)


def copied(s):
    return dict(k=s.kc, v=s.vc, k_exp=s.ke, v_exp=s.ve) if s.e4m3 else dict(k=s.kc, v=s.vc)


def plain_fork(s):
    """Request r takes over the first m tokens of request p, as both were before: pages that m fills are held
    together.  The page that m ends in is r's alone: one request that takes it over and has no one beside it at that
    page goes on with it (p itself if it can, else the first), the others get a page from the list's top and a copy."""
    page, R, W = s.page, s.R, s.width
    lens, parent, keep = s.lens.long(), s.parent.long(), s.keep.long()
    row, col = torch.arange(R, device="cuda"), torch.arange(W, device="cuda")[None]
    par = parent.clamp(min=0)
    m = torch.where(parent >= 0, lens[par], 0)
    m = torch.where(keep >= 0, torch.minimum(m, keep), m)
    whole, cut = m // page, m % page > 0
    longest = torch.zeros(R, dtype=torch.long, device="cuda").scatter_reduce(0, par, whole, "amax")
    x = s.table[par, whole.clamp(max=W - 1)].long()
    could = cut & (whole == longest[par]) & (s.others[x.clamp(min=0)] == 0)
    turn = torch.where(could, torch.where(row == par, 0, row + 1), R + 1)
    best = torch.full((R,), R + 1, device="cuda").scatter_reduce(0, par, turn, "amin")
    need = cut & ~(could & (turn == best[par]))
    end = need.cumsum(0)
    free = s.free.long()
    ok = ~need | (end <= free)
    taken = need & ok
    fresh = s.free_list[(free - end).clamp(min=0)].long()
    m, whole, cut = (torch.where(ok, y, 0) for y in (m, whole, cut.long()))

    new = torch.where(col < whole[:, None], s.table[par].long(), s.table.long())
    last = torch.where(taken, fresh, x)
    new = torch.where((col == whole[:, None]) & (cut[:, None] > 0), last[:, None], new)
    held_old, held_new = col < ((lens + page - 1) // page)[:, None], col < ((m + page - 1) // page)[:, None]

    def holders(ids, held):   # of each page; what is not held is counted behind the pool
        ids = torch.where(held, ids, s.n_pages).reshape(-1)
        return torch.zeros(s.n_pages + 1, dtype=torch.long, device="cuda").scatter_add(0, ids, torch.ones_like(ids))[: s.n_pages]

    old = s.table.long()
    before = holders(old, held_old)
    now = torch.where(before > 0, s.others + 1, 0) + holders(new, held_new) - before
    back = (before > 0) & (now == 0)
    # pages come back in the order of the last request that held them and of its pages
    at = torch.where(held_old, old, s.n_pages).reshape(-1)
    order = torch.full((s.n_pages + 1,), -1, device="cuda").scatter_reduce(0, at, torch.arange(R * W, device="cuda"), "amax")
    back_first = torch.argsort(torch.where(back, order[: s.n_pages], R * W))
    base = free - taken.sum()
    free_out = base + back.sum()
    j = torch.arange(s.n_pages, device="cuda")
    s.free_list.copy_(torch.where((j >= base) & (j < free_out), back_first[(j - base).clamp(min=0)], s.free_list))
    s.free_out.copy_(free_out)
    s.others.copy_((now - 1).clamp(min=0))
    s.table.copy_(new)
    s.lens_out.copy_(m)
    s.ok.copy_(ok)
    s.src.copy_(torch.where(taken, x, -1))
    s.dst.copy_(torch.where(taken, fresh, -1))
    return forked(s)


def plain_compact(s):
    """The i-th page held behind the limit moves to the i-th free page in front of it, as far as there are such; the
    list is made again of the free pages in front of the limit, the lowest on top."""
    col, j = torch.arange(s.width, device="cuda")[None], torch.arange(s.n_pages, device="cuda")
    held = col < ((s.lens.long() + s.page - 1) // s.page)[:, None]
    used = torch.zeros(s.n_pages + 1, dtype=torch.bool, device="cuda")
    used[torch.where(held, s.table.long(), s.n_pages)] = True
    used = used[: s.n_pages]
    source, place = used & (j >= s.limit), ~used & (j < s.limit)
    many = s.src.numel()
    nth = lambda mark: torch.argsort(torch.where(mark, j, j + s.n_pages))  # noqa: E731
    moved = torch.minimum(source.sum(), place.sum()).clamp(max=many)
    i = torch.arange(many, device="cuda")
    src, dst = nth(source)[:many], nth(place)
    s.src.copy_(torch.where(i < moved, src, -1))
    s.dst.copy_(torch.where(i < moved, dst[:many], -1))
    rank = source.long().cumsum(0) - 1
    to = torch.where(source & (rank < moved), dst[rank.clamp(min=0)], j)
    table = torch.where(held, to[s.table.long().clamp(min=0)], s.table_out.long())
    others = s.others.clone()
    gone = source & (rank < moved)
    others[gone] = 0
    s.others.copy_(torch.where(place & (place.long().cumsum(0) - 1 < moved),
                               s.others[src[(place.long().cumsum(0) - 1).clamp(0, many - 1)]], others))
    free_out = place.sum() - moved
    s.free_list.copy_(torch.where(j < free_out, dst[(moved + free_out - 1 - j).clamp(min=0)], s.free_list))
    s.free_out.copy_(free_out)
    s.left.copy_(source.sum() - moved)
    s.table_out.copy_(table)
    return compacted(s)


def plain_copy(s):
    live = s.src >= 0
    src, dst = s.src[live].long(), s.dst[live].long()
    for x in (s.kc, s.vc, s.ke, s.ve):
        if x is not None:
            y = x.view(torch.uint8) if s.e4m3 else x
            y[dst] = y[src]
    return copied(s)


def plain_shared(s):
    G = s.Hq // s.Hkv

    def rows(x, e, ids, at):   # (..., tokens, Hkv, d) in 32 bits
        x = x[ids, :, at].float()
        return x * torch.exp2(e[ids, :, at].float() - 127)[..., None] if e is not None else x

    alone = s.spans[-1][1]
    for a, b, common in s.spans + ([(alone, s.B, 0)] if alone < s.B else []):
        n = s.lens[a:b, None]
        q = s.q[a:b].float().view(b - a, s.Hkv, G, s.d)
        first = n - s.window if s.window else torch.zeros_like(n)
        # the common tokens, which the group's first request has too
        pos = torch.arange(common, device="cuda")
        block = s.table[a, pos // s.page].long()
        z = torch.einsum("bhgd,lhd->bhgl", q, rows(s.kc, s.ke, block, pos % s.page)) * s.scale
        V = rows(s.vc, s.ve, block, pos % s.page)
        z = torch.where(((pos < n) & (pos >= first))[:, None, None], z, -math.inf)
        # each one's own
        pos = torch.arange(common, s.longest, device="cuda")
        live = (pos < n) & (pos >= first)
        block = s.table[a:b, pos // s.page].clamp(min=0).long()
        K = torch.where(live[..., None, None], rows(s.kc, s.ke, block, pos % s.page), 0.0)
        own_V = torch.where(live[..., None, None], rows(s.vc, s.ve, block, pos % s.page), 0.0)
        y = torch.einsum("bhgd,blhd->bhgl", q, K) * s.scale
        y = torch.where(live[:, None, None], y, -math.inf)
        top = torch.maximum(z.amax(-1, keepdim=True) if common else z.new_full((1,), -math.inf),
                            y.amax(-1, keepdim=True) if pos.numel() else y.new_full((1,), -math.inf)).clamp(min=-1e30)
        z, y = torch.exp(z - top), torch.exp(y - top)
        total = z.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
        scale = 1.0 / total.clamp(min=1e-30)
        o = torch.einsum("bhgl,lhd->bhgd", z * scale, V) + torch.einsum("bhgl,blhd->bhgd", y * scale, own_V)
        s.o[a:b] = o.reshape(b - a, s.Hq, s.d)
        s.lse[a:b] = torch.where(total > 0, top + torch.log(total), -math.inf).reshape(b - a, s.Hq)
    return dict(o=s.o, lse=s.lse)


# ---- what a pass cannot do without -----------------------------------------------------------------------


def work(case):
    do = case["do"]
    if do in ("fork", "compact"):
        # lengths, requests and their answers; an entry of the table for each page held, and what lies on the list
        used, n_pages = pool_pages(case)
        common, behind = family_sizes(case)
        R = case["families"] * case["fan"]
        entries = case["fan"] * sum(common) + case["families"] * sum(pages_of(n, case["page"]) for n in behind)
        if do == "fork":
            moved = entries * (3 / 4 if case["mix"] == "beams" else 5 / 16)   # requests that change what they hold
            return {"bytes": int(4 * 8 * R + 16 * moved), "flops": int(moved + R)}
        away = int(used * (1 - used / n_pages))
        return {"bytes": 8 * entries + 4 * R + 4 * (min(n_pages, used + used // 50) - used) + 16 * away, "flops": entries}
    if do == "copy":
        n = case["moves"] - int(case["moves"] * case["padding"])
        vector = case["d"] + 1 if case["store"] == "e4m3" else 2 * case["d"]
        return {"bytes": 4 * n * case["Hkv"] * case["page"] * vector + 8 * case["moves"], "flops": 0}
    spans, lens = shared_lengths(case)
    page, B, Hq, d, w = case["page"], len(lens), case["Hq"], case["d"], case["window"]
    first = [max(0, n - w) if w else 0 for n in lens]
    tokens = read = pages = 0
    common_of = [0] * B
    for a, b, common in spans:
        common_of[a:b] = [common] * (b - a)
        live = [r for r in range(a, b) if lens[r] > 0]
        seen = common - min(min(first[r], common) for r in live)
        read += seen
        pages += pages_of(seen, page)
    for n, f, c in zip(lens, first, common_of):
        tokens += n - f
        mine = max(0, n - max(f, c))
        read += mine
        pages += pages_of(mine, page)
    vector = d + 1 if case["store"] == "e4m3" else 2 * d
    return {"bytes": 2 * read * case["Hkv"] * vector + B * Hq * (4 * d + 4) + 4 * (B + pages + 2 * len(spans)),
            "flops": 4 * tokens * Hq * d}


# ---- the definitions, in 64 bits -------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if s.do == "fork":
        return exact_fork(s)
    if s.do == "compact":
        return exact_compact(s)
    if s.do == "copy":
        for x in (s.kc, s.vc, s.ke, s.ve):
            if x is not None:
                y = (x.view(torch.uint8) if s.e4m3 else x).cpu()
                for a, b in zip(s.src.tolist(), s.dst.tolist()):
                    if a >= 0:
                        y[b] = y[a]
                (x.view(torch.uint8) if s.e4m3 else x).copy_(y)
        return {k: v.double() if v.dtype == E4M3 else v for k, v in copied(s).items()}
    o = torch.zeros((s.B, s.Hq, s.d), dtype=torch.float64, device="cuda")
    lse = torch.full((s.B, s.Hq), -math.inf, dtype=torch.float64, device="cuda")
    G = s.Hq // s.Hkv
    for b, n in enumerate(s.lens.tolist()):
        first = max(0, n - s.window) if s.window else 0
        if n == 0:
            continue
        blocks = s.table[b, first // s.page:-(-n // s.page)].long()
        a = first - first // s.page * s.page

        def seen(x, e):   # (Hkv, tokens, d)
            y = x[blocks].double()
            if e is not None:
                y = torch.ldexp(y, e[blocks].double()[..., None] - 127)
            return y.transpose(0, 1).reshape(s.Hkv, -1, x.shape[-1])[:, a:a + n - first]

        z = s.q[b].double().view(s.Hkv, G, s.d) @ seen(s.kc, s.ke).transpose(1, 2) * s.scale
        lse[b] = torch.logsumexp(z, -1).reshape(-1)
        o[b] = (torch.softmax(z, -1) @ seen(s.vc, s.ve)).reshape(s.Hq, s.d)
    return dict(o=o, lse=lse)


def exact_fork(s):
    page, R = s.page, s.R
    lens, parent, keep, others = s.lens.tolist(), s.parent.tolist(), s.keep.tolist(), s.others.tolist()
    table, free_list = s.table.tolist(), s.free_list.tolist()
    count = int(s.free)
    m, longest = [], [0] * R
    for r, p in enumerate(parent):
        n = lens[p] if p >= 0 else 0
        m.append(min(n, keep[r]) if keep[r] >= 0 else n)
        if p >= 0:
            longest[p] = max(longest[p], m[r] // page)
    goes_on = {}
    for r, p in enumerate(parent):
        k = m[r] // page
        if m[r] % page and k == longest[p] and others[table[p][k]] == 0 and (p not in goes_on or r == p):
            goes_on[p] = r
    held = [table[r][: pages_of(lens[r], page)] for r in range(R)]
    holders, new, ok, src, dst, asked = {}, [], [], [-1] * R, [-1] * R, 0
    for pages in held:
        for x in pages:
            holders[x] = others[x] + 1
    for r, p in enumerate(parent):
        k, good = m[r] // page, 1
        pages = list(table[p][:k]) if p >= 0 else []
        if m[r] % page:
            x = table[p][k]
            if goes_on.get(p) == r:
                pages.append(x)
            else:
                asked += 1
                good = int(asked <= count)
                if good:
                    src[r], dst[r] = x, free_list[count - asked]
                    holders[dst[r]] = 0
                    pages.append(dst[r])
        ok.append(good)
        new.append(pages if good else [])
        m[r] = m[r] if good else 0
    last = {}
    for pages in held:
        for x in pages:
            holders[x] -= 1
            last.pop(x, None)   # to the end
            last[x] = True
    for pages in new:
        for x in pages:
            holders[x] += 1
    back = [x for x in last if holders[x] == 0]
    base = count - min(asked, count)
    free_list[base:base + len(back)] = back
    for x, h in holders.items():
        others[x] = max(h - 1, 0)
    for r in range(R):
        table[r][: len(new[r])] = new[r]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return dict(table=i32(table), lens=i32(m), others=i32(others), free_list=i32(free_list), free=i32([base + len(back)]),
                src=i32(src), dst=i32(dst), ok=torch.tensor(ok, dtype=torch.uint8))


def exact_compact(s):
    lens, others, free_list = s.lens.tolist(), s.others.tolist(), s.free_list.tolist()
    table, out = s.table.tolist(), s.table_out.tolist()
    held = [table[r][: pages_of(n, s.page)] for r, n in enumerate(lens)]
    used = set(x for pages in held for x in pages)
    source = [x for x in range(s.limit, s.n_pages) if x in used]
    place = [x for x in range(s.limit) if x not in used]
    many = s.src.numel()
    moved = min(len(source), len(place), many)
    to = dict(zip(source[:moved], place))
    for x, y in to.items():
        others[y], others[x] = others[x], 0
    for r, pages in enumerate(held):
        out[r][: len(pages)] = [to.get(x, x) for x in pages]
    rest = place[moved:]
    free_list[: len(rest)] = rest[::-1]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    pad = [-1] * (many - moved)
    return dict(table=i32(out), others=i32(others), free_list=i32(free_list), free=i32([len(rest)]),
                src=i32(source[:moved] + pad), dst=i32(place[:moved] + pad), left=i32([len(source) - moved]))
