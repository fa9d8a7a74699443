"""An order within the attention over latents that no run can show to be missing, read from the source."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_30950_gb300", "csrc")


def test_tensor_memory_of_latents_is_taken_between_wait_and_release():
    """A kernel that is let in before this one holds its tensor memory could take it first and then wait for this one."""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "qs_kv_latent.cuh")).read())
    body = src[src.index("kv_latent_kernel(const KvAttendParams p"):src.index("pool_map(CUtensorMap")]
    at = [body.index(s) for s in ("chain_enter();", "tmem_alloc(", "tmem_relinquish();", "chain_release();", "__syncthreads();")]
    assert at == sorted(at)
    assert body.count("chain_") == 2 and "chain_wait" not in src
