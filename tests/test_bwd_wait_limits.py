"""The store warp of the backward kernel waits as long as a work item lasts, twice: for an item's results, and, where the item
leaves partial sums and this warp has nothing to store, for the next item.  Both limits have to grow with the item."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNEL = os.path.join(ROOT, "paper_2603_24517_b200", "csrc", "attn_bwd_kernel.cuh")


def test_waits_of_the_store_warp_grow_with_the_item():
    with open(KERNEL) as f:
        source = f.read()
    body = source[source.index("void role_store("):]
    body = body[:body.index("\n}\n")]
    waits = re.findall(r"(next_item|mbar_wait)\(((?:[^()]|\([^()]*\))*)\)", body)
    assert sorted(name for name, _ in waits) == ["mbar_wait", "next_item"]
    for name, args in waits:
        assert "whole_item(ctx, " in args, (name, args)


CHILD = """
import hashlib, sys, torch
import paper_2603_24517_b200 as lib
rows, scale = int(sys.argv[1]), 128 ** -0.5
g = torch.Generator(device="cuda").manual_seed(3)
q, dout = (torch.randn(1, rows, 1, 128, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
k, v = (torch.randn(1, 128, 1, 128, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
o, lse = torch.zeros_like(q), torch.full((1, 1, rows), 5.4, device="cuda")   # near the log-sum-exp of 128 such scores
dq, dk, dv = lib.attention_backward(dout, q, k, v, o, lse)
torch.cuda.synchronize()
print(lib.attn_last_device_status()[0], *(hashlib.sha256(t.contiguous().view(torch.int16).cpu().numpy()).hexdigest() for t in (dq[:, ::97], dk, dv)))
"""


@pytest.mark.gpu
def test_items_longer_than_the_limit(tmp_path):
    """A build whose waits give up after 1 ms, on 32 key items of 1500 tile pairs each (2 ms or more): the same results."""
    import paper_2603_24517_b200 as lib
    from paper_2603_24517_b200 import build as lib_build
    lib_build.build()
    short = str(tmp_path / "libattn_b200_1ms.so")
    lib_build.build_variant(short, ["-DATTN_WAIT_LIMIT_NS=1000000ull"])
    rows = 32 * 1500 * 128
    stats = 2 * 4 * rows
    assert lib.attn_bwd_workspace_bytes(1, 1, 1, rows, 128, 128, False) == stats + 2 * 32 * 128 * 128 * 4   # 32 parts of one tile
    out = []
    for path in (lib_build.LIB_PATH, short):
        res = subprocess.run([sys.executable, "-c", CHILD, str(rows)], capture_output=True, text=True, cwd=ROOT, timeout=300,
                             env=dict(os.environ, ATTN_B200_LIB=path))
        assert res.returncode == 0, res.stderr
        out.append(res.stdout.split())
    assert out[0][0] == "0" and out[1] == out[0]
