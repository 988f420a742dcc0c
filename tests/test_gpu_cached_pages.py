"""Pages that do not exist, rows in front of the first sequence, sequences shorter than their rows, captured calls at once."""
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import cache_oracle as orc
from test_gpu_cached_attention import E4M3, INT8, U, Batch, _library, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("rows", [1, 3, 140])
@pytest.mark.parametrize("causal", [True, False])
def test_missing_pages_of_every_size(page, kind, rows, causal):
    """NaN for the rows that see a key of a missing page, the definition's values (within the bounds of test_gpu_cached_attention)
    for the others."""
    t = 3 * 128 + 41
    b = Batch([(rows, t)] * 4, 1, page, kind, seed=page + rows)
    q = b.queries(2)
    table, lens = b.table.clone(), b.lens.clone()
    late = (t - 20) // page
    table[0, late] = b.n_pages      # the rows in front of it see none of it
    table[1, 128 // page] = -1      # the first of a step of 128 keys
    table[2, 256 // page - 1] = -5  # the last of one
    lens[3] = page * table.shape[1] + 5  # beyond the table, whose last block does not exist either
    o, lse = lib.attention_cached(q, b.cache, table, lens, b.starts, max_new=rows, causal=causal)
    for seq, first in enumerate((late * page, 128, (256 // page - 1) * page)):
        at = slice(seq * rows, (seq + 1) * rows)
        k, v = b.values(0, seq), b.values(1, seq)
        sees = torch.arange(t - rows, t, device="cuda") >= first if causal else torch.ones(rows, dtype=torch.bool, device="cuda")
        assert bool(o[at][sees].isnan().all()) and bool(lse[:, at][:, sees].isnan().all())
        want, z, spread, size = orc.attend(q[at], k, v, t - rows, causal, 1 / math.sqrt(128))
        rel = 600 * U * size + 2.0 ** -20 + t * U / 8
        bound = (rel.T[:, :, None] + 2.0 ** -11) * spread + t * 2.0 ** -30 * float(v.abs().max()) + 2.0 ** -8 * want.abs()
        good = (o[at].double() - want).abs() <= bound * (1 + 2.0 ** -7)
        assert bool(good[~sees].all())
        assert bool(((lse[:, at].double() - z).abs() <= rel + 8 * U * (z.abs() + size))[:, ~sees].all())
    assert bool(o[4 * rows - 1].isnan().all()) and bool(lse[:, 4 * rows - 1].isnan().all())


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("front", [1, 37, 500])
def test_rows_in_front_of_the_first_sequence_are_left(page, kind, front):
    b = Batch([(1, 100), (150, 400), (0, 3), (7, 7)], 2, page, kind, seed=front)
    n = b.rows[-1]
    starts = b.starts + front
    k, v, q = (rand(b.g, front + n, h, 128).bfloat16() for h in (2, 2, 4))
    for x in (k, v, q):
        x[:front] = float("nan")
    other = lib.KVCache(*(x.clone() for x in b.cache))
    lib.kv_cache_append(b.cache, k, v, b.table, b.lens, starts)
    lib.kv_cache_append(other, k[front:].contiguous(), v[front:].contiguous(), b.table, b.lens, b.starts)
    for x, y in zip(b.cache, other):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    out = [torch.full_like(k, 5.0) for _ in "kv"]
    lib.attn_kv_read(b.cache, *out, b.table, b.lens, starts)
    for x, y in zip(out, lib.kv_cache_read(b.cache, b.table, b.lens, b.starts, n=n)):
        assert bool((x[:front] == 5).all()) and torch.equal(x[front:], y)
    for hint in (1, 150):
        o, lse = torch.full_like(q, 5.0), torch.full((4, front + n), 5.0, device="cuda")
        lib.attn_fwd_cached(q, b.cache, o, lse, b.table, b.lens, starts, max_new=hint)
        want, want_lse = lib.attention_cached(q[front:].contiguous(), b.cache, b.table, b.lens, b.starts, max_new=hint)
        assert bool((o[:front] == 5).all()) and bool((lse[:, :front] == 5).all())
        assert torch.equal(o[front:], want) and torch.equal(lse[:, front:], want_lse)


@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("S", [2, 70])
def test_uniform_batch_of_sequences_shorter_than_their_rows(kind, S):
    """S rows a sequence of which only the last seq_lens are tokens: the others are dropped, read back as zeros, and see no key."""
    g = torch.Generator(device="cuda").manual_seed(S)
    lens = torch.tensor([0, 1, S - 1, S], dtype=torch.int32, device="cuda")
    table = torch.arange(4 * 3, dtype=torch.int32, device="cuda").view(4, 3)
    cache = lib.new_kv_cache(12, 32, 2, kind)
    k, v = (rand(g, 4, S, 2, 128).bfloat16() for _ in "kv")
    q = rand(g, 4, S, 8, 128).bfloat16()
    lib.kv_cache_append(cache, k, v, table, lens)
    back = lib.kv_cache_read(cache, table, lens, n=S)
    o, lse = lib.attention_cached(q, cache, table, lens)
    for b, n in enumerate(lens.tolist()):
        assert not bool(back[0][b, :S - n].any()) and not bool(o[b, :S - n].any()) and bool((lse[b, :, :S - n] == -math.inf).all())
        if n == 0:
            assert not bool(cache.k[3 * b:3 * b + 3].float().any())
            continue
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        alone = lib.new_kv_cache(12, 32, 2, kind)
        lib.kv_cache_append(alone, k[b, S - n:].contiguous(), v[b, S - n:].contiguous(), table[b:b + 1], lens[b:b + 1], starts)
        for x, y in zip(cache, alone):
            assert torch.equal(x[3 * b:3 * b + 3].contiguous().view(torch.uint8), y[3 * b:3 * b + 3].contiguous().view(torch.uint8))
        want, z, spread, size = orc.attend(q[b, S - n:], back[0][b, S - n:].double(), back[1][b, S - n:].double(), 0, True, 1 / math.sqrt(128))
        # what is read back is rounded once more than what the cache holds, 2^-8 of each key and value: scores are off by 2^-8 A, and
        # weights by twice that
        again = 2.0 ** -7 * size.T[:, :, None] + 2.0 ** -8
        assert bool(((o[b, S - n:].double() - want).abs() <= (again + 2.0 ** -11) * spread + 2.0 ** -8 * want.abs() + 1e-6).all())


def test_captured_calls_at_once():
    """Two captured steps on one cache, replayed on two streams: each has the workspace that its capture made."""
    b = Batch([(1, 5000), (90, 3000)], 4, 64, E4M3, seed=13)
    qs = [b.queries(16), b.queries(16)]
    want = [lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=90) for q in qs]
    graphs, got = [], []
    for q in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=90))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
