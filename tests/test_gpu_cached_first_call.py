"""The first call of attn_fwd_cached in a process, which prepares its kernels."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import torch
import paper_2603_24517_b200 as lib
g = torch.Generator(device="cuda").manual_seed(0)
new = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
q, k, v = new(1, {rows}, 8, 128), new(1, 300, 2, 128), new(1, 300, 2, 128)
lib.attention_forward(q, k, v, causal=True)  # the device's own set-up
cache = lib.new_kv_cache(5, 64, 2)
table, lens = torch.arange(5, device="cuda", dtype=torch.int32)[None], torch.tensor([300], device="cuda", dtype=torch.int32)
lib.kv_cache_append(cache, k, v, table, lens)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    o, lse = lib.attention_cached(q, cache, table, lens)
graph.replay()
torch.cuda.synchronize()
o2, lse2 = lib.attention_cached(q, cache, table, lens)
assert torch.equal(o, o2) and torch.equal(lse, lse2) and bool(o.isfinite().all()) and bool((o != 0).any())
"""


@pytest.mark.parametrize("rows", [1, 200])
def test_the_first_call_may_be_a_captured_one(rows):
    """After another entry point has set the device up, as the header says of captured calls."""
    r = subprocess.run([sys.executable, "-c", CHILD.format(rows=rows)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
