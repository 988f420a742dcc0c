"""GPU tests of backward launches in several runs of units, equal and unequal ones, and of longer sequences, against the 64-bit
definition with the bounds of ``test_gpu_backward``."""
import pytest
import torch

import paper_2603_24517_b200 as lib
from paper_2603_24517_b200 import build as lib_build
from test_gpu_backward import SCALE, check, grads, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,causal,extra", [
    (13, 10, 10, 512, 512, True, 1), (13, 10, 10, 512, 512, False, 1), (16, 8, 8, 512, 512, True, 2),
    (10, 38, 19, 300, 400, True, 1), (13, 72, 24, 260, 129, True, None),
])
def test_several_runs(B, Hq, Hkv, Sq, Sk, causal, extra):
    plan = lib.attn_bwd_plan(B, Hq, Hkv, Sq, Sk, 128, causal)
    assert plan["run"] < B * Hkv and (extra is None or plan["run_extra"] == extra)
    dout, q, k, v = make(B, Hq, Hkv, Sq, Sk)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE)
    if causal and Sq > Sk:
        assert bool((got[0][:, :Sq - Sk] == 0).all())


@pytest.mark.parametrize("Hq,Hkv,S,causal", [(1, 1, 8192, True), (2, 1, 7001, True), (1, 1, 8192, False)])
def test_longer_sequences(Hq, Hkv, S, causal):
    dout, q, k, v = make(1, Hq, Hkv, S, S)
    o, lse, got = grads(dout, q, k, v, causal)
    check(got, dout, q, k, v, o, lse, causal, SCALE)
    torch.cuda.empty_cache()
