"""The example of a hybrid stack: every attention layer's answers against plain attention in 64 bits over the keys
and values that the layer was given, and the pages all back at the end."""
import importlib.util
import os

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_decode.py")
    spec = importlib.util.spec_from_file_location("hybrid_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def attention(q, K, V, scale):
    """One token in 64 bits: q (Hq, dk) against K (n, Hkv, dk), V (n, Hkv, dv); (o, bound of o's error).  The bound is
    first order, for bf16 (unit roundoff u = 2^-9): scores are sums of dk products in 32 bits, so a weight is off
    by twice their error; it may be rounded to bf16, twice with the normalisation; sums of n terms and a few
    2^-23 of the exponential; o is rounded once."""
    n, Hkv, dk = K.shape
    q = q.double().view(Hkv, -1, dk)
    u = 2.0 ** -9
    z = torch.einsum("hgd,nhd->hgn", q, K) * scale
    dz = torch.einsum("hgd,nhd->hgn", q.abs(), K.abs()).amax(-1) * scale * (dk * 2.0 ** -23)
    w = torch.softmax(z, -1)
    o, mag = torch.einsum("hgn,nhd->hgd", w, V), torch.einsum("hgn,nhd->hgd", w, V.abs())
    rel = 2 * u + 2 * dz + 2.0 ** -18 + z.abs().amax(-1) * 2.0 ** -22 + n * 2.0 ** -24
    return o.flatten(0, 1), (u * o.abs() + rel[..., None] * mag + 2.0 ** -24).flatten(0, 1)


@pytest.mark.parametrize("page,running", [(1, 2), (16, 3), (64, 7)])
def test_a_hybrid_stack(qs, example, page, running):
    g = torch.Generator().manual_seed(page)
    prompts = [torch.randint(0, 512, (n,), generator=g).tolist() for n in (1, 9, 30, 17, 3, 40, 16)]
    record = []
    s, _ = example.decode(prompts, generate=10, running=running, page=page, window=20, seed=3, record=record)
    assert int(s.pages.free_count) == s.cfg.n_pages and not bool(s.pages.lens.any())
    assert sorted(s.pages.free_list.tolist()) == list(range(s.cfg.n_pages))
    assert bool((s.out >= 0).all()) and s.fed.tolist() == [len(p) + 9 for p in prompts]
    history = {}   # what each layer was given, request by request
    for layer, runs, q, k, v, o in record:
        c = layer.cfg
        rows = history.setdefault(id(layer), [[] for _ in prompts])
        for r in runs.nonzero()[:, 0].tolist():
            kv = [k[r].cpu()] + ([] if v is None else [v[r].cpu()])
            if c.store == qs.KV_E4M3:
                kv = [ref.quantise(x) for x in kv]
                kv = [x * torch.exp2(e.double() - 127)[..., None] for x, e in kv]
            rows[r].append([x.double() for x in kv])
            seen = rows[r][-c.window:] if c.window else rows[r]
            K = torch.stack([x[0] for x in seen])
            V = torch.stack([x[-1] for x in seen])[..., : c.dv]
            want, bound = attention(q[r].cpu(), K, V, c.scale)
            assert bool(((o[r].double().cpu() - want).abs() <= bound).all()), (page, r, len(seen))
