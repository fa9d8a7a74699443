"""The paged cache's four operators in 64 bits and plain loops, and inputs to compare them on."""
import math

import torch


def pages_of(n, page):
    return -(-n // page)


def plan(lens, n_new, table, free, page, T, max_pages):
    """Lists in, dict of lists out; `table` and `free` (the stack) are changed in place."""
    for r, a in enumerate(n_new):
        if a < 0:
            free.extend(table[r][: pages_of(lens[r], page)])
    avail, asked = len(free), 0
    cu, ok, out, slot, pos, req = [0], [], [], [-1] * T, [-1] * T, [-1] * T
    whole = list(free)
    for r, a in enumerate(n_new):
        start = cu[-1]
        cu.append(min(start + max(a, 0), 2 ** 31 - 1))
        if a < 0:
            ok.append(1)
            out.append(0)
            continue
        have, want = pages_of(lens[r], page), pages_of(lens[r] + a, page)
        good = cu[-1] <= T and want <= max_pages
        if good:
            asked += want - have
            good = want == have or asked <= avail
        if good:
            for c in range(have, want):
                table[r][c] = free.pop()
        ok.append(int(good))
        out.append(lens[r] + a if good else lens[r])
        for i in range(min(a, T - start)):
            p = lens[r] + i
            pos[start + i], req[start + i] = p, r
            if good:
                slot[start + i] = table[r][p // page] * page + p % page
    return dict(cu=cu, ok=ok, lens=out, slot=slot, pos=pos, req=req, stack=free, whole=whole)


def quantise(x):
    """Codes (as values) and exponent bytes of vectors along x's last axis, from the definition."""
    x = x.double()
    fine = torch.isfinite(x).all(-1)
    x = torch.where(fine[..., None], x, 0.0)
    powers = torch.tensor([math.ldexp(1.0, k) for k in range(-126, 122)], dtype=torch.float64)
    top = x.abs().amax(-1)
    k = torch.searchsorted(448 * powers, top)   # the first power that is enough
    k = torch.where(top > 0, k, 126)
    y = x / powers[k][..., None]
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step, torch.where(fine, k + 1, 255).to(torch.uint8)


class Batch:
    """A cache of random contents with every unused place poisoned, and a batch of queries on it."""

    def __init__(self, qs, lens, Hq, Hkv, dk, dv=None, page=16, latent=False, dtype="bf16", e4m3=False, window=0,
                 scale=None, seed=0, spread=1.0, spare=3, device="cuda", poison=float("nan"), order="shuffled"):
        g = torch.Generator().manual_seed(seed)
        dv = dk if dv is None else dv
        R = len(lens)
        self.t = torch.float16 if dtype == "f16" else torch.bfloat16
        used = sum(pages_of(n, page) for n in lens)
        n_pages, max_pages = used + spare, max([pages_of(n, page) for n in lens] + [1]) + 1
        self.cfg = qs.KvConfig(kind=qs.KV_LATENT if latent else qs.KV_HEADS, Hq=Hq, Hkv=Hkv, dk=dk, dv=dv, page=page,
                               n_pages=n_pages, max_pages=max_pages, dtype=qs.KV_F16 if dtype == "f16" else qs.KV_BF16,
                               store=qs.KV_E4M3 if e4m3 else qs.KV_16, window=window,
                               scale=dk ** -0.5 if scale is None else scale)
        ids = torch.randperm(n_pages, generator=g).tolist() if order == "shuffled" else list(range(n_pages))
        table = [[-7] * max_pages for _ in lens]   # what lies behind a request's pages is never looked up
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for r, n in enumerate(lens):
            for c in range(pages_of(n, page)):
                table[r][c] = ids.pop()
                live[table[r][c], : min(page, n - c * page)] = True
        self.lens, self.table = lens, table
        shape = (n_pages, Hkv, page)

        def pool(d):
            x = torch.randn(shape + (d,), generator=g).to(self.t)
            e = None
            if e4m3:
                x, e = quantise(x)
                value = x * torch.exp2(e.double() - 127)[..., None]
                x = x.float().to(torch.float8_e4m3fn)
                e[~live[:, None].expand(shape)] = 255
                raw = x.view(torch.uint8)
                raw[~live[:, None].expand(shape)] = 0x7F   # the type's NaN
            else:
                x[~live[:, None].expand(shape)] = poison
                value = x.double()
            return x.to(device), None if e is None else e.to(device), value

        self.k, ke, self.kval = pool(dk)
        self.v, ve, self.vval = (None, None, self.kval[..., :dv]) if latent else pool(dv)
        self.cache = qs.KvCache(self.k, self.v, ke, ve)
        self.qval = (spread * torch.randn(R, Hq, dk, generator=g)).to(self.t)
        self.q = self.qval.to(device)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
        self.d_table, self.d_lens = i32(table).reshape(R, max_pages), i32(lens)
        self.o = torch.full((R, Hq, dv), 77.0, dtype=self.t, device=device)
        self.lse = torch.full((R, Hq), 77.0, dtype=torch.float32, device=device)
        self.work = qs.new_kv_work(self.cfg, device=device)

    def run(self, qs, stream=None):
        qs.qstate_kv_attend(self.cfg, self.cache, self.q, self.d_table, self.d_lens, self.o, self.lse, self.work,
                            stream=stream)

    def expect(self):
        """(o, lse, bound of o's error, bound of lse's error), in 64 bits.

        First-order bounds.  A score is a sum of dk exact products in 32 bits: its error is at most
        dk 2^-23 times the sum of their magnitudes (sums and the scale; twice the unit roundoff covers
        any order of summation), and a weight's relative error is the scores' twice (its own and the
        normalisation's) and a few 2^-23 of the exponential and the rescalings.  The weight may be rounded
        to the 16-bit type (unit roundoff u = 2^-9 for bf16, 2^-12 for f16; under 2^-14 f16 has steps of
        2^-24 of the largest weight), twice with the normalisation; sums of n terms in 32 bits add
        n 2^-24.  At the end o itself is rounded once."""
        c, u = self.cfg, 2.0 ** -12 if self.t == torch.float16 else 2.0 ** -9
        R, G = len(self.lens), c.Hq // c.Hkv
        o, lse = torch.zeros(R, c.Hq, c.dv, dtype=torch.float64), torch.full((R, c.Hq), -math.inf, dtype=torch.float64)
        do, dl = torch.zeros_like(o), torch.zeros(R, c.Hq, dtype=torch.float64)
        for r, n in enumerate(self.lens):
            first = max(0, n - c.window) if c.window else 0
            if n == 0:
                continue
            at = torch.arange(first, n)
            ids = torch.tensor([self.table[r][t // c.page] for t in range(first, n)], dtype=torch.long)
            K, V = self.kval[ids, :, at % c.page], self.vval[ids, :, at % c.page]   # (n, Hkv, d)
            q = self.qval[r].double().view(c.Hkv, G, c.dk)
            z = torch.einsum("hgd,nhd->hgn", q, K) * c.scale
            dz = torch.einsum("hgd,nhd->hgn", q.abs(), K.abs()).amax(-1) * abs(c.scale) * (c.dk * 2.0 ** -23)
            top = z.amax(-1, keepdim=True)
            w = torch.exp(z - top)
            total = w.sum(-1, keepdim=True)
            w = w / total
            out = torch.einsum("hgn,nhd->hgd", w, V)
            mag = torch.einsum("hgn,nhd->hgd", w, V.abs())
            rel = 2 * u + 2 * dz + 2.0 ** -18 + z.abs().amax(-1) * 2.0 ** -22 + (n - first) * 2.0 ** -24
            small = (n - first) * 2.0 ** -24 * V.abs().amax(0)[:, None] if self.t == torch.float16 else 0.0
            o[r], do[r] = out.reshape(c.Hq, c.dv), (u * out.abs() + rel[..., None] * mag + small + 2.0 ** -24).reshape(c.Hq, c.dv)
            lse[r] = (top + torch.log(total))[..., 0].reshape(-1)
            dl[r] = (dz + 2.0 ** -20 + (n - first) * 2.0 ** -24 + lse[r].view(c.Hkv, G).abs() * 2.0 ** -22).reshape(-1)
        return o, lse, do, dl

    def check(self, qs):
        qs.qstate_check()
        o, lse, do, dl = self.expect()
        got, gl = self.o.double().cpu(), self.lse.double().cpu()
        bad = ~((got - o).abs() <= do)
        assert not bool(bad.any()), f"o: {int(bad.sum())} of {bad.numel()} off, rows {sorted(set(bad.nonzero()[:, 0].tolist()))[:8]}, " \
                                    f"worst {float(((got - o).abs() / do.clamp(min=1e-30)).max()):.3g} bounds"
        empty = torch.isinf(lse)
        assert torch.equal(empty, gl == -math.inf)
        assert bool(((gl - lse)[~empty].abs() <= dl[~empty]).all()), f"lse off by {float((gl - lse)[~empty].abs().max()):.3g}"
        assert not bool(self.work.view(torch.int32)[:1024].any()), "the work space's counters are not zero"
