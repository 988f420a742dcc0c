"""Attention over the cache where the scales of the values differ widely, or are near the ends of their range.

A row's result may depend on the tokens that it sees, and only on those.  Bounds, with U = 2^-24, vs the V scale of a token's page and
head, and for each row P = the largest exp(s_j - lse) vs_j among the keys it sees (vs_j at least 2^-64 of the sequence's largest, and 2^-84):
* a weight enters the product with the values as an f16 number of 64 times exp(s_j) vs_j / 2^M, where 2^M is at most twice the
  largest exp(s_i) vs_i so far: rounded to 11 bits (2^-12 of itself), or to a multiple of 2^-24 (off by at most 2^-25) where f16 runs
  out of exponent, which is 2^-31 2^M <= 2^-30 P and counts for each key that is seen, times its code (448 or 127 at most);
* its exponent has the logarithm of the scale in it: numbers of at most 2^8 in size, rounded three times, 2^-17 each, and a logarithm
  of at most 2^7 in size that is off by 2^-22 of itself (2^-14 in all);
* scores, sums and the rounding of the result as for ordinary scales: 600 U A + 2^-20 + n U / 8 relative, half a BF16 step (2^-8).
"""
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import cache_oracle as orc
from test_gpu_cached_attention import E4M3, INT8, U, Batch, _library, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def check(batch, q, o, lse, causal=True):
    """o [rows, Hq, 128], lse [Hq, rows] of a packed batch against the definition."""
    scale = 1 / math.sqrt(128)
    hq = q.shape[1]
    group = hq // batch.heads
    largest_code = 448 if batch.kind == E4M3 else 127
    for b, (n, t) in enumerate(batch.seqs):
        if n == 0:
            continue
        at = slice(batch.rows[b], batch.rows[b] + n)
        k, v = batch.values(0, b), batch.values(1, b)
        want, z, spread, size = orc.attend(q[at], k, v, t - n, causal, scale)
        token = torch.arange(t, device="cuda")
        vs = batch.cache.v_scale[batch.ids[b][token // batch.page]].double()  # [t, heads]
        seen = token[None] <= (t - n + torch.arange(n, device="cuda"))[:, None] if causal else torch.ones(n, t, dtype=torch.bool, device="cuda")
        rel = 600 * U * size + 2.0 ** -20 + t * U / 8 + 2.0 ** -14
        for h in range(hq):
            p = torch.exp(q[at, h].double() @ k[:, h // group].T * scale - z[h][:, None]).masked_fill(~seen, 0)
            counts = vs[:, h // group].clamp(min=2.0 ** -84)
            top = (p * counts.clamp(min=float(counts.max()) * 2.0 ** -64)).max(1).values
            floor = seen.sum(1) * 2.0 ** -30 * top * largest_code
            bound = (rel[h][:, None] + 2.0 ** -12) * spread[:, h] + floor[:, None] + 2.0 ** -8 * want[:, h].abs()
            off = (o[at, h].double() - want[:, h]).abs()
            # what is rounded is not the definition's value but one within the bound of it
            assert bool((off <= bound * (1 + 2.0 ** -7)).all()), (b, h, float((off / bound).max()))
        off = (lse[:, at].double() - z).abs()
        assert bool((off <= rel + 8 * U * (z.abs() + size)).all()), (b, float(off.max()))


FORMS = [  # rows a sequence, heads, group, page, kind
    (2, 2, 1, 16, E4M3),
    (3, 1, 4, 32, INT8),
    (2, 2, 8, 64, INT8),
    (40, 1, 4, 16, INT8),
    (90, 2, 4, 32, E4M3),
    (300, 1, 2, 64, E4M3),
    (300, 2, 1, 128, INT8),
]


@pytest.mark.parametrize("rows,heads,group,page,kind", FORMS)
@pytest.mark.parametrize("factor", [2.0 ** 24, 2.0 ** 40, 2.0 ** 70])
def test_rows_do_not_depend_on_the_scales_of_tokens_they_do_not_see(rows, heads, group, page, kind, factor):
    """The page of a sequence's last token has a V scale far larger than all before it: rows in front of that page see none of it."""
    t = (rows // page + 4 | 1) * page + 1  # the last token has a page of its own, in the middle of 128 keys where pages are shorter
    b = Batch([(rows, t), (rows, t + 1)], heads, page, kind, seed=rows + page)
    for ids in b.ids:
        b.cache.v_scale[ids[-1]] *= factor
    q = b.queries(heads * group)
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
    check(b, q, o, lse)


@pytest.mark.parametrize("rows,heads,group,page,kind", FORMS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("spread,low,high", [(15, -40, 40), (60, -80, 110)])
def test_weights_and_scales_that_differ_widely(rows, heads, group, page, kind, causal, spread, low, high):
    """Keys that hardly count on pages of large values, keys that count on pages of small ones."""
    b = Batch([(rows, 1500), (rows, 401)], heads, page, kind, seed=rows + 2 * page)
    b.cache.v_scale.mul_(torch.exp2((spread * rand(b.g, *b.cache.v_scale.shape)).clamp(low, high)))
    q = b.queries(heads * group, gain=12.0)
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows, causal=causal)
    check(b, q, o, lse, causal)


@pytest.mark.parametrize("rows,heads,group,page,kind", FORMS)
@pytest.mark.parametrize("size", [2.0 ** 126, 2.0 ** 100, 2.0 ** -60, 2.0 ** -90])
def test_values_near_the_ends_of_the_range(rows, heads, group, page, kind, size):
    """Whatever the values' size, the result is a mean of them: nothing on the way may overflow or vanish."""
    b = Batch([(rows, 900), (rows, rows)], heads, page, kind, seed=rows + 3 * page)
    # codes are at most 448 or 127; the mean of values of both signs is well below their largest
    b.cache.v_scale.copy_((size / (256 if kind == E4M3 else 64)) * torch.exp2(-rand(b.g, *b.cache.v_scale.shape).abs().clamp(max=4)))
    q = b.queries(heads * group)
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
    assert bool(o.isfinite().all()) and bool(lse.isfinite().all())
    check(b, q, o, lse)


@pytest.mark.parametrize("rows,heads,group,page,kind", FORMS)
def test_pages_of_zero_values_that_take_the_weight(rows, heads, group, page, kind):
    """The first page has V scale 0 and most of each row's weight, the others values of ordinary and of great size."""
    for size in (1.0, 2.0 ** 50):
        b = Batch([(rows, 700), (rows, max(rows, page))], heads, page, kind, seed=rows + 4 * page)
        for ids in b.ids:
            b.cache.v_scale[ids[0]] = 0
        b.cache.v_scale.mul_(size)
        b.cache.k_scale[b.ids[0][0]] *= 4
        q = b.queries(heads * group)
        o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
        check(b, q, o, lse)
        # rows that see nothing but that page: codes that stand for 0
        first = (b.rows[1], min(page, rows))
        if max(rows, page) == rows or rows <= page:
            assert not bool(o[first[0]:first[0] + first[1]].any())


def test_all_values_zero():
    for rows in (1, 200):
        b = Batch([(rows, 500)], 2, 32, E4M3, seed=rows)
        b.cache.v_scale.zero_()
        q = b.queries(4)
        o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
        assert not bool(o.any())
        check(b, q, o, lse)


def test_extreme_values_through_append():
    """Values of 2.9e38 and of 1e-30 through the whole path, prompt and single token."""
    for kind in (E4M3, INT8):
        for size in (2.9e38, 1e-30):
            cache = lib.new_kv_cache(8, 64, 1, kind)
            g = torch.Generator(device="cuda").manual_seed(5)
            k = rand(g, 1, 200, 1, 128).bfloat16()
            v = (torch.where(rand(g, 1, 200, 1, 128) > 0, 1.0, -1.0) * size).bfloat16()
            table, lens = torch.arange(8, dtype=torch.int32, device="cuda")[None], torch.tensor([200], dtype=torch.int32, device="cuda")
            lib.kv_cache_append(cache, k, v, table, lens)
            b = Batch.__new__(Batch)
            b.page, b.heads, b.kind, b.cache, b.ids = 64, 1, kind, cache, [torch.arange(4, device="cuda")]
            for rows in (1, 200):
                q = rand(g, 1, rows, 4, 128).bfloat16()
                o, lse = lib.attention_cached(q, cache, table, lens)
                b.seqs, b.rows = [(rows, 200)], [0, rows]
                assert bool(o.isfinite().all())
                check(b, q[0], o[0], lse[0])
