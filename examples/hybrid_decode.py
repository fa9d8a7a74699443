"""Decoding with a hybrid stack on one GPU: recurrent layers with states of few bits beside attention layers
over a paged cache.

Random weights; four layers, each added to the residual: gated delta-rule recurrence (4-bit state), attention
with keys and values in bf16, attention with keys and values in e4m3 seen through a window, and attention over
one latent vector a token.  More requests come than may run at once.  Each is fed its prompt a token at a
time, then its own most likely tokens; when it ends its pages go back to the pool and the next one takes them.
Who runs, who ends and who gets which page is decided on the GPU: no step waits for the host.

    python examples/hybrid_decode.py --requests 12 --running 5 --page 16
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_30950_gb300 as qs  # noqa: E402

WIDTH, VOCABULARY = 256, 512


def _weights(g, rows, cols):
    return (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(torch.bfloat16).cuda()


class Recurrence:
    """Gated delta rule, one write-back a token.  Requests that do not run get k = beta = 0 and next to no
    decay (rates are positive): nothing is erased, written or forgotten."""

    def __init__(self, g, R, steps, heads=2, d=64):
        self.cfg = qs.Config(B=R, H=heads, dk=d, dv=d, bbar_num=4, bmin=1, bmax=8)
        self.now, self.next, self.stats = qs.new_state(self.cfg), qs.new_state(self.cfg), qs.new_stats(self.cfg)
        qs.qstate_init(self.cfg, self.now, self.next)
        zeros = lambda *tail: torch.zeros(R, steps, heads, *tail, device="cuda")  # noqa: E731
        self.x = qs.Inputs(zeros(d), zeros(d), zeros(d), s=zeros(d), beta=zeros(), T=steps)
        self.o = zeros(d)
        self.heads, self.d = heads, d
        self.w_in, self.w_out = _weights(g, WIDTH, heads * (4 * d + 1)), _weights(g, heads * d, WIDTH)

    def __call__(self, x, step, serving):
        q, k, v, s, beta = (x @ self.w_in).float().view(-1, self.heads, 4 * self.d + 1).split([self.d] * 4 + [1], -1)
        runs = serving.runs[:, None, None]
        unit = lambda y: torch.nn.functional.normalize(y, dim=-1)  # noqa: E731
        self.x.q[:, step] = unit(q)
        self.x.k[:, step] = unit(k) * runs
        self.x.v[:, step] = v
        self.x.s[:, step] = torch.where(runs, torch.nn.functional.softplus(s - 2), 1e-20)
        self.x.beta[:, step] = torch.sigmoid(beta[..., 0]) * runs[..., 0]
        qs.qstate_step(self.cfg, self.now, self.next, self.x, step, step + 1, step, self.o, self.stats)
        self.now, self.next = self.next, self.now
        return self.o[:, step].reshape(len(x), -1).to(torch.bfloat16) @ self.w_out


class Attention:
    """Grouped heads, or (`latent`) one vector a token for all heads, over the paged cache."""

    def __init__(self, g, pool, heads=8, kv_heads=2, d=64, latent=False, e4m3=False, window=0):
        dk, dv = (d + 32, d) if latent else (d, d)
        kv_heads = 1 if latent else kv_heads
        self.cfg = qs.KvConfig(kind=qs.KV_LATENT if latent else qs.KV_HEADS, Hq=heads, Hkv=kv_heads, dk=dk, dv=dv,
                               store=qs.KV_E4M3 if e4m3 else qs.KV_16, window=window, scale=dk ** -0.5, **pool)
        self.cache, self.work = qs.new_kv_cache(self.cfg), qs.new_kv_work(self.cfg)
        self.sizes = [heads * dk, kv_heads * dk] + ([] if latent else [kv_heads * dv])
        self.w_in, self.w_out = _weights(g, WIDTH, sum(self.sizes)), _weights(g, heads * dv, WIDTH)

    def __call__(self, x, step, serving):
        c, R = self.cfg, len(x)
        q, k, *v = (x @ self.w_in).split(self.sizes, -1)
        q, k = q.view(R, c.Hq, c.dk), k.view(R, c.Hkv, c.dk)
        v = v[0].view(R, c.Hkv, c.dv) if v else None
        # the step's rows are those of the requests that run, in their order
        rows = serving.slots.req.clamp(min=0)
        qs.qstate_kv_append(c, self.cache, k[rows], None if v is None else v[rows], serving.slots.slot)
        o = torch.empty(R, c.Hq, c.dv, dtype=x.dtype, device="cuda")
        qs.qstate_kv_attend(c, self.cache, q, serving.pages.table, serving.pages.lens, o, None, self.work)
        if serving.record is not None:
            serving.record.append((self, serving.runs.clone(), q, k, v, o))
        return o.reshape(R, -1) @ self.w_out


class Serving:
    """Requests, the pages that they hold, and this step's rows."""

    def __init__(self, prompts, generate, running, page, record):
        R = len(prompts)
        longest = max(len(p) for p in prompts)
        i64 = lambda rows: torch.tensor(rows, device="cuda")  # noqa: E731
        self.prompt = i64([p + [0] * (longest - len(p)) for p in prompts])
        self.prompt_len = i64([len(p) for p in prompts])
        self.total = self.prompt_len + generate - 1     # the last token that is generated is not fed
        self.fed, self.sampled = torch.zeros_like(self.total), torch.zeros_like(self.total)
        self.out = torch.full((R, generate), -1, dtype=torch.long, device="cuda")
        self.running, self.record = running, record
        columns = -(-(longest + generate) // page)
        self.pool = dict(page=page, n_pages=running * columns, max_pages=columns)
        self.cfg = qs.KvConfig(**self.pool)
        self.pages, self.slots, self.work = qs.new_kv_pages(self.cfg, R), qs.new_kv_slots(R, R), qs.new_kv_work(self.cfg)

    def begin(self):
        """Pages and rows of a step; the tokens to feed."""
        done = self.fed >= self.total
        first = torch.cumsum(~done, 0) <= self.running   # the oldest that have not ended
        n_new = torch.where(done, -(self.pages.lens > 0).int(), first.int()).int()
        qs.qstate_kv_plan(self.cfg, self.pages, n_new, self.slots, self.work)
        self.runs = (n_new > 0) & self.slots.ok.bool()
        asked = self.prompt.gather(1, self.fed.clamp(max=self.prompt.shape[1] - 1)[:, None])[:, 0]
        return torch.where(self.fed < self.prompt_len, asked, self.sampled)

    def end(self, logits):
        self.sampled = logits.argmax(-1)
        self.fed += self.runs
        at = self.fed - self.prompt_len
        speaks = (self.runs & (at >= 0))[:, None] & (torch.arange(self.out.shape[1], device="cuda") == at[:, None])
        self.out = torch.where(speaks, self.sampled[:, None], self.out)


def decode(prompts, generate=24, running=4, page=16, window=20, seed=0, record=None):
    """Tokens generated for each prompt (lists of ids under 512), R x generate."""
    g = torch.Generator().manual_seed(seed)
    s = Serving(prompts, generate, running, page, record)
    # each request takes one step a token, and one more passes before its place is taken
    steps = sum(len(p) + generate for p in prompts)
    table, w_out = _weights(g, VOCABULARY, WIDTH) * VOCABULARY ** 0.5, _weights(g, WIDTH, VOCABULARY)
    layers = [Recurrence(g, len(prompts), steps), Attention(g, s.pool),
              Attention(g, s.pool, e4m3=True, window=window), Attention(g, s.pool, d=128, latent=True)]
    norm = lambda x: torch.nn.functional.rms_norm(x, (WIDTH,))  # noqa: E731
    taken = 0
    for step in range(steps):
        if step % 16 == 0 and bool((s.fed >= s.total).all()):
            break   # looked at now and then only: it waits for the GPU
        x = table[s.begin()]
        for layer in layers:
            x = x + layer(norm(x), step, s)
        s.end(norm(x) @ w_out)
        taken += 1
    s.begin()   # the last pages go back
    qs.qstate_check()
    return s, taken


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--running", type=int, default=5)
    ap.add_argument("--generate", type=int, default=24)
    ap.add_argument("--page", type=int, default=16)
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCABULARY, (5 + 7 * (r % 5),), generator=g).tolist() for r in range(a.requests)]
    qs.load()
    s, steps = decode(prompts, a.generate, a.running, a.page)
    print(f"{a.requests} requests, {a.running} at once, {s.pool['n_pages']} pages of {a.page}: {steps} steps, "
          f"{int(s.fed.sum())} tokens; {int(s.pages.free_count)} pages free at the end")
    for r in range(min(4, a.requests)):
        print(f"request {r}: {len(prompts[r])} tokens ->", *s.out[r].tolist())


if __name__ == "__main__":
    main()
