"""The paged cache of a hybrid model's attention layers, as cases that can be timed and compared.

A model whose recurrent layers run on this library's packed states keeps some attention layers beside
them.  Their keys and values live in pages that requests take from one pool.  A case names one of
the four operators of a serving step (``do``):

* ``plan``    the block table, the slots of the step's new tokens and the pool's free list, made on the
              GPU from the requests' lengths;
* ``append``  the new tokens' keys and values into their slots, in 16 bits or as e4m3 codes with a
              power of two for each token and head;
* ``attend``  one new token of each request against its pages;
* ``latent``  the same where a token's keys and values are one latent vector that all heads share:
              the scores take the whole vector, the values are its first ``rank`` entries.

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
        # a serving step of the full decode batch: a token each, a few requests end; launches and latency
        dict(name="plan_decode", do="plan", R=256, page=16, context=4096, ended=0.02, prompts=0.0, prompt=1, spare=0.1),
        # a step that also takes new prompts in: some 300,000 tokens get their slots
        dict(name="plan_prompts", do="plan", R=700, page=64, context=20000, ended=0.05, prompts=0.1, prompt=8500, spare=0.1),
        # one token each of an odd, small batch
        dict(name="append_step", do="append", T=37, Hkv=4, d=64, page=16, type="f16", store="16"),
        # the prompts of a batch, cut out of one fused projection's rows
        dict(name="append_prompts", do="append", T=16384, Hkv=8, d=128, page=32, type="bf16", store="16"),
        # an odd number of tokens into a cache held in eight bits
        dict(name="append_e4m3", do="append", T=20011, Hkv=8, d=128, page=64, type="bf16", store="e4m3"),
        # one sequence being generated: few rows, so the cache's length has to be split
        dict(name="attend_one", do="attend", B=1, Hq=32, Hkv=4, d=128, page=16, length=3001, window=0, type="bf16", store="16"),
        # the full decode batch of 32 heads, ragged lengths, among them nothing and one token
        dict(name="attend_batch", do="attend", B=256, Hq=32, Hkv=16, d=128, page=64, length=1024, window=0, type="f16", store="16"),
        # a layer that sees the last 1000 tokens only, heads of 64
        dict(name="attend_window", do="attend", B=48, Hq=40, Hkv=8, d=64, page=32, length=16000, window=1000, type="bf16", store="16"),
        # a few very long contexts, sixteen query heads to a key head
        dict(name="attend_long", do="attend", B=5, Hq=64, Hkv=4, d=128, page=128, length=100000, window=0, type="bf16", store="16"),
        # a cache in eight bits
        dict(name="attend_e4m3", do="attend", B=64, Hq=48, Hkv=8, d=128, page=32, length=12000, window=0, type="bf16", store="e4m3"),
        # a handful of requests on a layer with latents of 256 + 64
        dict(name="latent_few", do="latent", B=3, Hq=32, rank=256, rope=64, page=64, length=20000, type="bf16"),
        # a batch on wide latents and twice the heads
        dict(name="latent_batch", do="latent", B=64, Hq=64, rank=512, rope=64, page=32, length=8000, type="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))

    do = rng.choice(["plan", "append", "attend", "attend", "attend", "latent", "latent"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if do == "plan":
        R = log_int(1, 2000)
        prompts = rng.choice([0.0, 0.05, 0.2])
        return dict(do=do, R=R, page=page, context=log_int(16, 32768), ended=rng.choice([0.0, 0.02, 0.2]), prompts=prompts,
                    prompt=log_int(1, max(1, min(20000, int(300000 / (R * max(prompts, 0.01)))))),
                    spare=rng.choice([0.1, 0.1, 0.0, -0.5]))
    if do == "append":
        Hkv, d, store = log_int(1, 16), rng.choice([64, 128, 128, 256]), rng.choice(["16", "16", "e4m3"])
        return dict(do=do, T=log_int(1, min(30000, 20_000_000 // (Hkv * d))), Hkv=Hkv, d=d, page=page,
                    type="bf16" if store == "e4m3" else rng.choice(["bf16", "f16"]), store=store)
    B = log_int(1, 256)
    if do == "attend":
        Hkv, d, store = log_int(1, 16), rng.choice([64, 128, 128, 128, 256]), rng.choice(["16", "16", "e4m3"])
        most = 180_000_000 // (B * Hkv * d)
        return dict(do=do, B=B, Hq=Hkv * rng.choice([1, 2, 3, 4, 6, 8, 16]), Hkv=Hkv, d=d, page=page,
                    length=log_int(1, max(1, min(100000, most))), window=rng.choice([0, 0, 0, log_int(1, 4096)]),
                    type="bf16" if store == "e4m3" else rng.choice(["bf16", "f16"]), store=store)
    rank, rope, Hq = rng.choice([128, 256, 512]), rng.choice([0, 32, 64]), log_int(1, 128)
    most = 295_000_000 // (B * (rank + rope)) * 64 // max(64, Hq)
    return dict(do=do, B=B, Hq=Hq, rank=rank, rope=rope, page=page, length=log_int(1, max(1, min(100000, most))),
                type=rng.choice(["bf16", "f16"]))


# ---- inputs --------------------------------------------------------------------------------------------


def lengths(B, longest):
    """Evenly spread up to `longest`; a batch of eight and more also has an empty row and one of a token."""
    n = [-(-longest * (i + 1) // B) for i in range(B)]
    if B >= 8:
        n[:2] = [0, 1]
    return n


def taken_tokens(case):
    n = lengths(case["B"], case["length"])
    return [min(x, case["window"]) for x in n] if case.get("window") else n


def requests(case):
    """(tokens cached, tokens to come) of a plan's requests: -1 to come for one that has ended."""
    R = case["R"]
    ended, prompts = int(R * case["ended"]), int(math.ceil(R * case["prompts"]))
    rest = max(0, R - ended - prompts)
    old, new = [], []
    for i in range(R):
        if i < rest:
            old.append(-(-case["context"] * (i + 1) // rest))
            new.append(0 if i % 29 == 28 else 1)
        elif i < rest + ended:
            old.append(-(-case["context"] * (i - rest + 1) // ended))
            new.append(-1)
        else:
            old.append(0)
            new.append(-(-case["prompt"] * (i - rest - ended + 1) // prompts))
    return old, new


def plan_sizes(case):
    """(pages in use, pages that the step asks for, its tokens)"""
    old, new = requests(case)
    pages = lambda n: -(-n // case["page"])  # noqa: E731
    return (sum(pages(a) for a in old), sum(pages(a + n) - pages(a) for a, n in zip(old, new) if n > 0),
            sum(n for n in new if n > 0))


def block_table(lens, page, width, perm):
    """(B, width): the pages of each request, in the order of `perm`; -1 behind them."""
    many = (lens + page - 1) // page
    table = torch.full((lens.numel(), width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None] < many[:, None]] = perm[: int(many.sum())].int()
    return table


def split_e4m3(x):
    """Codes of x's last axis and the exponent byte k + 127 of each vector: the smallest power of two 2^k
    with |x| <= 448 * 2^k; a vector that is not finite has the byte 255 and codes of zero."""
    x = x.float()
    top = x.abs().amax(-1)
    mant, ex = torch.frexp(top)
    k = torch.where(top > 0, ex - 9 + (mant > 0.875).int(), 0).clamp(-126, 120)
    fine = torch.isfinite(x).all(-1)
    k = torch.where(fine, k, 0).int()
    codes = (torch.where(fine[..., None], x, 0.0) * ((127 - k) << 23).view(torch.float32)[..., None]).to(E4M3)
    return codes, torch.where(fine, k + 127, 255).to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    perm = lambda n: torch.randperm(n, device="cuda", generator=gen)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = types.SimpleNamespace(case=case, do=case["do"], page=case["page"])
    if s.do == "plan":
        old, new = requests(case)
        order = perm(case["R"])
        s.lens, s.n_new = ints(old)[order], ints(new)[order]
        used, wanted, tokens = plan_sizes(case)
        s.n_pages = used + max(1, int(math.ceil(wanted * (1 + case["spare"]))))
        s.width = -(-(max(old) + max(max(new), 1)) // s.page) + 1
        p = perm(s.n_pages)
        s.table = block_table(s.lens, s.page, s.width, p)
        s.free_list = torch.full((s.n_pages,), -1, dtype=torch.int32, device="cuda")
        s.free_list[: s.n_pages - used] = p[used:].int()
        s.free = ints([s.n_pages - used])
        s.T = max(1, -(-tokens // 64) * 64)   # a captured graph's fixed number of rows
        empty = lambda n, t=torch.int32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
        s.lens_out, s.free_out, s.cu, s.ok = empty(case["R"]), empty(1), empty(case["R"] + 1), empty(case["R"], torch.uint8)
        s.slot, s.pos, s.req = empty(s.T), empty(s.T), empty(s.T)
        return s
    latent = s.do == "latent"
    s.type = TYPES[case["type"]]
    s.e4m3 = case.get("store") == "e4m3"
    s.Hkv = 1 if latent else case["Hkv"]
    s.dk = case["rank"] + case["rope"] if latent else case["d"]
    s.dv = case["rank"] if latent else case["d"]
    # keys have a few channels much larger than the rest
    loud = torch.exp(0.5 * rnd(s.Hkv, s.dk))
    if s.do == "append":
        T = case["T"]
        s.n_pages = -(-(T + T // 8) // s.page) + 3
        wide = rnd(T, 3 * s.Hkv, s.dk)
        wide[:, s.Hkv:2 * s.Hkv] *= loud
        wide = wide.to(s.type)   # queries, keys and values of one projection: the cache's rows are views
        s.k, s.v = wide[:, s.Hkv:2 * s.Hkv], wide[:, 2 * s.Hkv:]
        s.slot = perm(s.n_pages * s.page)[:T].int()
        s.slot[perm(T)[: T // 50]] = -1   # rows that pad the step
        s.slots = None
        shape = (s.n_pages, s.Hkv, s.page, s.dk)
        s.kc, s.vc = (torch.zeros(shape, dtype=E4M3 if s.e4m3 else s.type, device="cuda") for _ in range(2))
        s.ke, s.ve = (torch.full(shape[:3], 127, dtype=torch.uint8, device="cuda") if s.e4m3 else None for _ in range(2))
        return s
    s.B, s.Hq, s.window = case["B"], case["Hq"], case.get("window", 0)
    s.lens = ints(lengths(s.B, case["length"]))[perm(s.B)]
    used = sum(-(-n // s.page) for n in lengths(s.B, case["length"]))
    s.n_pages = used + used // 10 + 1
    s.width = -(-case["length"] // s.page)
    s.table = block_table(s.lens, s.page, s.width, perm(s.n_pages))
    shape = (s.n_pages, s.Hkv, s.page, s.dk)

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

    s.kc, s.ke = pool(loud[:, None])
    s.vc, s.ve = (None, None) if latent else pool(1.0)
    s.q = (2.0 * rnd(s.B, s.Hq, s.dk)).to(s.type)
    s.scale = s.dk ** -0.5
    s.o = torch.empty((s.B, s.Hq, s.dv), dtype=s.type, device="cuda")
    s.lse = torch.empty((s.B, s.Hq), dtype=torch.float32, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------


def handles(s):
    """What a program makes once and keeps: the layer's description, its cache and the work space."""
    import paper_2609_30950_gb300 as qs

    s.qs = qs
    if s.do == "plan":
        s.cfg = qs.KvConfig(page=s.page, n_pages=s.n_pages, max_pages=s.width)
        s.pages = qs.KvPages(s.table, s.lens, s.free_list, s.free)
        s.slots = qs.KvSlots(s.cu, s.slot, s.pos, s.req, s.ok)
        s.work = qs.new_kv_work(s.cfg)
        return
    s.cfg = qs.KvConfig(kind=qs.KV_LATENT if s.do == "latent" else qs.KV_HEADS, Hq=getattr(s, "Hq", s.Hkv), Hkv=s.Hkv, dk=s.dk,
                        dv=s.dv, page=s.page, n_pages=s.n_pages, max_pages=getattr(s, "width", s.n_pages),
                        dtype=qs.KV_F16 if s.type == torch.float16 else qs.KV_BF16,
                        store=qs.KV_E4M3 if s.e4m3 else qs.KV_16, window=getattr(s, "window", 0),
                        scale=getattr(s, "scale", 1.0))
    s.cache = qs.KvCache(s.kc, s.vc, s.ke, s.ve)
    s.work = qs.new_kv_work(s.cfg) if s.do != "append" else None


def run(s):
    if not own:
        return {"plan": plain_plan, "append": plain_append, "attend": plain_attend, "latent": plain_attend}[s.do](s)
    if not hasattr(s, "qs"):
        handles(s)
    qs = s.qs
    if s.do == "plan":
        qs.qstate_kv_plan(s.cfg, s.pages, s.n_new, s.slots, s.work, s.lens_out, s.free_out)
        return planned(s)
    if s.do == "append":
        qs.qstate_kv_append(s.cfg, s.cache, s.k, s.v, s.slot)
        return appended(s)
    qs.qstate_kv_attend(s.cfg, s.cache, s.q, s.table, s.lens, s.o, s.lse, s.work)
    return dict(o=s.o, lse=s.lse)


def planned(s):
    return dict(table=s.table, lens=s.lens_out, free_list=s.free_list, free=s.free_out, cu=s.cu, ok=s.ok, slot=s.slot,
                pos=s.pos, req=s.req)


def appended(s):
    return dict(k=s.kc, v=s.vc, k_exp=s.ke, v_exp=s.ve) if s.e4m3 else dict(k=s.kc, v=s.vc)


def plain_plan(s):
    """Ended requests give their pages back, in order, on top of the free list; the others take theirs from
    its top, in order.  A request whose pages are no longer there, or whose tokens run past the rows or the
    table, gets none: its tokens have the slot -1."""
    page, R = s.page, s.lens.numel()
    lens, n = s.lens.long(), s.n_new.long()
    free = s.free.long()
    ended, add = n < 0, n.clamp(min=0)
    end = add.cumsum(0)
    have, total = (lens + page - 1) // page, (lens + add + page - 1) // page
    valid = ~ended & (end <= s.T) & (total <= s.width)
    need = torch.where(valid, total - have, 0)
    back = torch.where(ended, have, 0)
    need_end, back_end = need.cumsum(0), back.cumsum(0)
    avail = free + back_end[-1]
    ok = valid & ((need == 0) | (need_end <= avail))
    granted = (need * ok).sum()

    # the j-th page from the top of the stack: free list below, returned pages above
    j = torch.arange(s.n_pages, device="cuda")
    returned = torch.searchsorted(back_end, j, right=True).clamp(max=R - 1)
    page_back = s.table[returned, (j - back_end[returned] + back[returned]).clamp(0, s.width - 1)]
    stack = torch.where(j < free, s.free_list, page_back[(j - free).clamp(min=0)])
    who = torch.searchsorted(need_end, j, right=True).clamp(max=R - 1)
    column = have[who] + j - need_end[who] + need[who]
    taken = stack[(avail - 1 - j).clamp(min=0)]
    live = j < granted
    s.table[who[live], column[live]] = taken[live]
    free_out = avail - granted
    s.free_list.copy_(torch.where((j >= free) & (j < free_out), stack, s.free_list))
    s.free_out.copy_(free_out)
    s.lens_out.copy_(torch.where(ended, 0, torch.where(ok, lens + add, lens)))
    s.ok.copy_(ok | ended)
    s.cu[0] = 0
    s.cu[1:] = end

    t = torch.arange(s.T, device="cuda")
    r = torch.searchsorted(end, t, right=True)
    inside, r = r < R, r.clamp(max=R - 1)
    pos = lens[r] + t - end[r] + add[r]
    at = s.table[r, (pos // page).clamp(max=s.width - 1)].long() * page + pos % page
    s.slot.copy_(torch.where(inside & ok[r], at, -1))
    s.pos.copy_(torch.where(inside, pos, -1))
    s.req.copy_(torch.where(inside, r, -1))
    return planned(s)


def plain_append(s):
    live = s.slot >= 0
    at = s.slot[live].long()
    block, row = at // s.page, at % s.page
    k, v = s.k[live], s.v[live]
    if s.e4m3:
        (k, s.ke[block, :, row]), (v, s.ve[block, :, row]) = split_e4m3(k), split_e4m3(v)
        k, v = k.view(torch.uint8), v.view(torch.uint8)
        s.kc.view(torch.uint8)[block, :, row], s.vc.view(torch.uint8)[block, :, row] = k, v
    else:
        s.kc[block, :, row], s.vc[block, :, row] = k, v
    return appended(s)


def plain_attend(s):
    pos = torch.arange(s.case["length"], device="cuda")
    block, row = s.table[:, pos // s.page].clamp(min=0).long(), pos % s.page
    n = s.lens[:, None]
    live = (pos < n) & (pos >= n - s.window) if s.window else pos < n

    def rows(x, e):   # (B, length, Hkv, d) in 32 bits, zero where nothing is seen
        x = x[block, :, row].float()
        if e is not None:
            x = x * torch.exp2(e[block, :, row].float() - 127)[..., None]
        return torch.where(live[..., None, None], x, 0.0)

    K = rows(s.kc, s.ke)
    q = s.q.float().view(s.B, s.Hkv, s.Hq // s.Hkv, s.dk)
    logit = torch.einsum("bhgd,blhd->bhgl", q, K) * s.scale
    logit = torch.where(live[:, None, None], logit, -math.inf)
    top = logit.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logit - top)
    total = p.sum(-1, keepdim=True)
    V = K[..., : s.dv] if s.vc is None else rows(s.vc, s.ve)
    o = torch.einsum("bhgl,blhd->bhgd", p / total.clamp(min=1e-30), V)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    s.o.copy_(o.reshape(s.o.shape))
    s.lse.copy_(lse.reshape(s.lse.shape))
    return dict(o=s.o, lse=s.lse)


# ---- what a pass cannot do without -----------------------------------------------------------------------


def work(case):
    do = case["do"]
    if do == "plan":
        used, wanted, tokens = plan_sizes(case)
        # lengths, requests, their answers; each token's slot, position and request; pages moved
        return {"bytes": 4 * (4 * case["R"] + 1) + case["R"] + 12 * tokens + 8 * wanted, "flops": tokens + case["R"]}
    if do == "append":
        n = 2 * case["T"] * case["Hkv"]
        out = n * (case["d"] + 1) if case["store"] == "e4m3" else 2 * n * case["d"]
        return {"bytes": 2 * n * case["d"] + out + 4 * case["T"], "flops": n * case["d"]}
    tokens, B, Hq = sum(taken_tokens(case)), case["B"], case["Hq"]
    if do == "latent":
        dk, dv = case["rank"] + case["rope"], case["rank"]
        cache = tokens * dk * 2
    else:
        dk = dv = case["d"]
        cache = 2 * tokens * case["Hkv"] * (dk + 1 if case["store"] == "e4m3" else 2 * dk)
    pages = sum(-(-n // case["page"]) for n in taken_tokens(case))
    return {"bytes": cache + B * Hq * (2 * dk + 2 * dv + 4) + 4 * (B + pages), "flops": 2 * tokens * Hq * (dk + dv)}


# ---- the definitions, in 64 bits -------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if s.do == "plan":
        return exact_plan(s)
    if s.do == "append":
        return exact_append(s)
    o = torch.zeros((s.B, s.Hq, s.dv), dtype=torch.float64, device="cuda")
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

        K = seen(s.kc, s.ke)
        V = K[..., : s.dv] if s.vc is None else seen(s.vc, s.ve)
        z = s.q[b].double().view(s.Hkv, G, s.dk) @ K.transpose(1, 2) * s.scale
        lse[b] = torch.logsumexp(z, -1).reshape(-1)
        o[b] = (torch.softmax(z, -1) @ V).reshape(s.Hq, s.dv)
    return dict(o=o, lse=lse)


def exact_append(s):
    power = lambda k: ((k.long() + 1023) << 52).view(torch.float64)  # noqa: E731
    out = {}
    for name, x, cache, e in (("k", s.k, s.kc, s.ke), ("v", s.v, s.vc, s.ve)):
        y = cache.double()
        for t0 in range(0, x.shape[0], 4096):
            slot = s.slot[t0:t0 + 4096].long()
            z = x[t0:t0 + 4096].double()[slot >= 0]
            slot = slot[slot >= 0]
            if s.e4m3:
                # 448 = 1.75 * 2^8, so 2^k is the power of two in top / 1.75, rounded up, over 2^8
                top = z.abs().amax(-1, keepdim=True)
                half, up = torch.frexp(top / 1.75)
                k = torch.where(top > 0, (up - (half == 0.5).int() - 8).clamp(-126, 120), 0)
                z = z * power(-k)
                unit = power(torch.frexp(z.abs().clamp(min=2.0 ** -6))[1] - 4)
                z = torch.round(z / unit) * unit
                e[slot // s.page, :, slot % s.page] = (k[..., 0] + 127).to(torch.uint8)
            y[slot // s.page, :, slot % s.page] = z
        out[name] = y
        if s.e4m3:
            out[name + "_exp"] = e
    return out


def exact_plan(s):
    page, width, T = s.page, s.width, s.T
    lens, new, table = s.lens.tolist(), s.n_new.tolist(), s.table.tolist()
    stack = s.free_list[: int(s.free)].tolist()
    free_list = s.free_list.tolist()
    before = len(stack)
    pages = lambda n: -(-n // page)  # noqa: E731
    for r, n in enumerate(new):
        if n < 0:
            stack += table[r][: pages(lens[r])]
    whole, avail = list(stack), len(stack)
    cu, ok, slot, pos, req, lens_out, asked = [0], [], [-1] * T, [-1] * T, [-1] * T, [], 0
    for r, n in enumerate(new):
        at = cu[-1]
        cu.append(at + max(n, 0))
        if n < 0:
            ok.append(1)
            lens_out.append(0)
            continue
        have, total = pages(lens[r]), pages(lens[r] + n)
        good = cu[-1] <= T and total <= width
        if good:
            asked += total - have
            good = total == have or asked <= avail
        if good:
            for c in range(have, total):
                table[r][c] = stack.pop()
        ok.append(int(good))
        lens_out.append(lens[r] + n if good else lens[r])
        for i in range(n):
            if at + i < T:
                p = lens[r] + i
                pos[at + i], req[at + i] = p, r
                slot[at + i] = table[r][p // page] * page + p % page if good else -1
    if len(stack) > before:
        free_list[before:len(stack)] = whole[before:len(stack)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return dict(table=i32(table), lens=i32(lens_out), free_list=i32(free_list), free=i32([len(stack)]), cu=i32(cu),
                ok=torch.tensor(ok, dtype=torch.uint8), slot=i32(slot), pos=i32(pos), req=i32(req))
