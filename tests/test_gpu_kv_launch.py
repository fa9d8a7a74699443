"""Launches of the paged cache's kernels: request counts whose shared memory lies about 48 KB, and calls of several host
threads whose kernels are the same with different amounts of shared memory."""
import os
import subprocess
import sys
import threading

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))

# ascending, in a process that has launched no larger one: a limit that was raised for more requests would hide a refusal
COUNTS = """
import sys
sys.path[:0] = [{here!r}, {root!r}]
import paper_2609_30950_gb300 as qs
import test_gpu_kv as t
qs.load()
for R in (2047, 2048, 2049, 2431, 2432, 2445, 2457, 2458, 2500):
    lens = [(7 * r) % 50 for r in range(R)]
    t.run_plan(qs, lens, [-1 if r % 9 == 0 else {new} for r in range(R)], 16, R, T={T}, max_pages=9)
"""


@pytest.mark.parametrize("new,T", [(1, 2600), (20, 50000)])
def test_plan_of_any_number_of_requests(qs, new, T):
    code = COUNTS.format(here=HERE, root=os.path.dirname(HERE), new=new, T=T)
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def at_once(calls, seconds=4.0):
    """Repeats each call in a thread of its own, on a stream of its own; what any of them raised."""
    errors, stop = [], threading.Event()

    def work(call):
        stream = torch.cuda.Stream()
        try:
            for i in range(100000):
                if stop.is_set():
                    return
                call(stream)
                if i % 64 == 63:
                    stream.synchronize()
        except Exception as e:   # any refusal ends the test
            errors.append(e)
            stop.set()

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    stop.wait(seconds)
    stop.set()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return errors


def test_layers_of_different_widths_from_several_threads(qs):
    batches = [ref.Batch(qs, [40, 3], 64, 1, dk, 128, page=64, latent=True, seed=dk) for dk in (128, 160, 192)]
    torch.cuda.synchronize()
    errors = at_once([lambda s, b=b: b.run(qs, stream=s) for b in batches])
    assert not errors, errors[0]
    for b in batches:
        b.check(qs)


def test_plans_of_different_sizes_from_several_threads(qs):
    def plan(R):
        cfg = qs.KvConfig(page=16, n_pages=R, max_pages=2)
        pages, slots, work = qs.new_kv_pages(cfg, R), qs.new_kv_slots(R, R), qs.new_kv_work(cfg)
        n_new = torch.zeros(R, dtype=torch.int32, device="cuda")
        return lambda s: qs.qstate_kv_plan(cfg, pages, n_new, slots, work, stream=s)
    calls = [plan(R) for R in (2600, 5000, 8192)]
    torch.cuda.synchronize()
    errors = at_once(calls)
    assert not errors, errors[0]
    qs.qstate_check()
