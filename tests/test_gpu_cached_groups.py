"""Packed batches of prompts and single tokens where the heads a key head are not a power of two, or more than 16."""
import pytest
import torch

import paper_2603_24517_b200 as lib
from test_gpu_cached_attention import E4M3, INT8, Batch, _library, check  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,page,kind", [(3, 16, INT8), (9, 64, E4M3), (12, 32, INT8), (15, 128, INT8), (17, 16, E4M3), (32, 64, INT8)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_and_short_sequences_of_odd_groups(group, page, kind, causal):
    """Each row is written once, whichever kernel has it; rows of tokens that straddle two tiles too."""
    seqs = [(1, 900), (150, 700), (0, 40), (1, 1), (2, 333), (65, 65), (5, 500), (1, 0), (9, 129), (1, 2500), (3, 17)]
    b = Batch(seqs, 2, page, kind, seed=group, scale_spread=1.0)
    q = b.queries(2 * group)
    for hint in (150, 1, None):
        o = torch.full_like(q, 7.0)
        lse = torch.full((2 * group, q.shape[0]), 7.0, device="cuda")
        lib.attn_fwd_cached(q, b.cache, o, lse, b.table, b.lens, b.starts, max_new=hint, causal=causal)
        check(b, q, o, lse, causal)
