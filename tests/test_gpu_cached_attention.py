"""GPU tests of the paged 8-bit cache (append, read back) and of attention over it against 64-bit definitions.

Codes and scales are exact: every step of the definition is one correctly rounded FP32 operation.

Attention.  With U = 2^-24, A = the largest scale * sum_d |q_d k_jd| a row sees, n = its keys:
* a score is a sum of 128 exact products, in a tree of tensor-core additions that may cut instead of round, times three factors:
  off by at most 300 U A (in nats; 128 additions, 2 U each, and the factors);
* a weight exp(s - m) is off by twice that, relative, plus 2^-21 (exp2 and its argument), and rounded to 11 bits: 2^-12, and as
  a number held as 2^6 .. 2^14 times itself, 2^-30 of the largest where f16 runs out of exponent;
* the sums over n keys add at most n / 8 U;
* so |o - o*| <= (600 U A + 2^-11 + 2^-20 + n U / 8) sum_j p_j |v_j| + n 2^-30 max |v| + half a BF16 step, and
  |lse - lse*| <= 600 U A + 2^-20 + n U / 8 + 8 U (|lse| + A).
"""
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import cache_oracle as orc
from paper_2603_24517_b200 import build as lib_build

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3, INT8 = torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


class Batch:
    """Sequences of (rows of this call, tokens in all) in a cache of their own, filled with random codes everywhere."""

    def __init__(self, seqs, heads, page, kind, seed=0, token_major=False, spare=2, scale_spread=0.0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.seqs, self.page, self.kind, self.heads = seqs, page, kind, heads
        blocks = [-(-max(t, 0) // page) for _, t in seqs]
        self.n_pages = sum(blocks) + spare
        order = torch.randperm(self.n_pages, generator=self.g, device="cuda").to(torch.int32)
        width = max(max(blocks), 1) + 1
        self.table = torch.full((len(seqs), width), -7, dtype=torch.int32, device="cuda")
        at = 0
        self.ids = []
        for b, n in enumerate(blocks):
            self.table[b, :n] = order[at:at + n]
            self.ids.append(order[at:at + n].long())
            at += n
        self.lens = torch.tensor([t for _, t in seqs], dtype=torch.int32, device="cuda")
        rows = [0]
        for n, _ in seqs:
            rows.append(rows[-1] + n)
        self.rows = rows
        self.starts = torch.tensor(rows, dtype=torch.int32, device="cuda")
        if token_major:
            z = [torch.zeros(self.n_pages, page, heads, 128, dtype=kind, device="cuda") for _ in "kv"]
            self.cache = lib.KVCache(*z, *(torch.zeros(self.n_pages, heads, device="cuda") for _ in "kv"))
        else:
            self.cache = lib.new_kv_cache(self.n_pages, page, heads, kind)
        for x in self.cache[:2]:  # any code, the NaN of E4M3 too, where no token of these sequences lives
            x.view(torch.uint8).copy_(torch.randint(0, 256, x.shape, generator=self.g, device="cuda", dtype=torch.uint8))
        for x in self.cache[2:]:
            x.copy_(torch.exp2(scale_spread * rand(self.g, *x.shape)) * (1 / 64 if kind == E4M3 else 1 / 40))
        for ids, (_, t) in zip(self.ids, seqs):
            for x in self.cache[:2]:
                for j in range(-(-max(t, 0) // page)):
                    m = min(page, t - j * page)
                    if kind == E4M3:
                        x[ids[j], :m] = (rand(self.g, m, heads, 128) * 64).to(kind)
                    else:
                        x[ids[j], :m] = (rand(self.g, m, heads, 128) * 40).round().clamp(-127, 127).to(kind)

    def values(self, which, b):
        """float64 [tokens, heads, 128]"""
        t = max(self.seqs[b][1], 0)
        if t == 0:
            return torch.zeros(0, self.heads, 128, dtype=torch.float64, device="cuda")
        return orc.gather(self.cache[which].float(), self.cache[2 + which], self.ids[b], t, self.page)

    def queries(self, hq, gain=1.0):
        return (rand(self.g, self.rows[-1], hq, 128) * gain).bfloat16()


def check(batch, q, o, lse, causal=True, scale=None, rows=None):
    """o [rows, Hq, 128], lse [Hq, rows] of a packed batch against the definition."""
    scale = 1 / math.sqrt(128) if scale is None else scale
    for b, (n, t) in enumerate(batch.seqs):
        if n == 0:
            continue
        at = slice(batch.rows[b], batch.rows[b] + n)
        k, v = batch.values(0, b), batch.values(1, b)
        want, z, spread, size = orc.attend(q[at], k, v, max(t, 0) - n, causal, scale)
        keys = max(t, 0)
        rel = 600 * U * size + 2.0 ** -20 + keys * U / 8
        floor = keys * 2.0 ** -30 * (float(v.abs().max()) if keys else 0.0)
        bound = (rel.T[:, :, None] + 2.0 ** -11) * spread + floor + 2.0 ** -8 * want.abs()
        got = o[at].double()
        assert bool(((got - want).abs() <= bound * (1 + 2.0 ** -7)).all()), (b, float(((got - want).abs() - bound).max()))
        if lse is not None:
            none = z == -math.inf
            got = lse[:, at].double()
            assert bool((got[none] == -math.inf).all())
            off = torch.where(none, torch.zeros_like(z), (got - z).abs())
            assert bool((off <= rel + 8 * U * (torch.where(none, torch.zeros_like(z), z).abs() + size)).all()), (b, float(off.max()))


ATTEND = [  # sequences (rows, tokens), heads, group, page, kind, token-major
    ([(1, 1)], 1, 1, 16, E4M3, False),
    ([(1, 1), (1, 2), (1, 16), (1, 17), (1, 127), (1, 128), (1, 129)], 2, 4, 16, INT8, False),
    ([(1, 513)] * 3, 8, 1, 64, E4M3, True),
    ([(1, 4097), (1, 30)], 3, 7, 128, INT8, True),
    ([(1, 0), (1, 77), (0, 50), (2, 1), (1, 300)], 1, 16, 32, E4M3, False),
    ([(5, 3), (3, 700), (0, 0), (4, 4)], 2, 8, 32, INT8, False),
    ([(17, 900), (1, 5), (16, 16)], 2, 3, 64, E4M3, False),
    ([(130, 131), (1, 1000), (257, 1500)], 1, 1, 16, INT8, False),
    ([(200, 2000)], 2, 5, 128, E4M3, True),
    ([(33, 40), (64, 64), (1, 4000), (31, 999)], 4, 4, 64, INT8, True),
    ([(128, 128), (129, 385)], 2, 2, 32, E4M3, False),
    ([(1, 60000)], 1, 8, 64, E4M3, False),
    ([(1, 20 + 7 * b) for b in range(300)], 2, 2, 16, INT8, False),
    ([(300, 300), (45, 2900)], 1, 6, 16, E4M3, False),
    ([(70, 3000)], 1, 128, 64, INT8, False),
]


@pytest.mark.parametrize("seqs,heads,group,page,kind,token_major", ATTEND)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_matches_definition(seqs, heads, group, page, kind, token_major, causal):
    b = Batch(seqs, heads, page, kind, seed=len(seqs) + page, token_major=token_major, scale_spread=1.0)
    q = b.queries(heads * group)
    o = torch.full_like(q, 7.0)
    lse = torch.full((heads * group, q.shape[0]), 7.0, device="cuda")
    lib.attn_fwd_cached(q, b.cache, o, lse, b.table, b.lens, b.starts, causal=causal)
    check(b, q, o, lse, causal)
    # one row each and many rows may take different kernels: the answer is the same attention
    hint = torch.empty_like(o)
    lib.attn_fwd_cached(q, b.cache, hint, None, b.table, b.lens, b.starts, max_new=1, causal=causal)
    check(b, q, hint, None, causal)
    again, _ = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, causal=causal)
    assert torch.equal(again, o)


@pytest.mark.parametrize("S,t,hq,hkv,kind", [(1, 333, 8, 2, E4M3), (3, 500, 12, 4, INT8), (150, 1000, 4, 4, E4M3), (1, 129, 3, 1, INT8)])
def test_uniform_batch_is_the_packed_one(S, t, hq, hkv, kind):
    b = Batch([(S, t), (S, t + 65), (S, S)], hkv, 32, kind, seed=S)
    q = b.queries(hq)
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=S)
    u, ulse = lib.attention_cached(q.view(3, S, hq, 128), b.cache, b.table, b.lens)
    assert torch.equal(u.flatten(0, 1), o)
    assert torch.equal(ulse.permute(1, 0, 2).flatten(1), lse)


def test_sharp_scores_and_other_scales():
    b = Batch([(1, 3000), (1, 257), (40, 2000)], 2, 64, E4M3, seed=3, scale_spread=3.0)
    for gain, scale in ((30.0, None), (1e-3, None), (1.0, 1.7), (1e5, 1e-6)):
        q = b.queries(8, gain)
        o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, scale=scale)
        check(b, q, o, lse, scale=scale)


def test_rows_of_zeros_and_pages_of_zeros():
    b = Batch([(1, 700), (20, 700)], 2, 32, INT8, seed=4)
    b.cache.k_scale[b.ids[0][3]] = 0
    b.cache.v_scale[b.ids[0][5]] = 0
    b.cache.v_scale[b.ids[1][:2]] = 0
    q = b.queries(4)
    q[0] = 0
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts)
    check(b, q, o, lse)


@pytest.mark.parametrize("rows", [1, 150])
def test_strided_queries_outputs_and_cache(rows):
    b = Batch([(rows, 400), (rows, 300)], 2, 16, E4M3, seed=5)
    q = b.queries(4)
    packed = torch.zeros(q.shape[0], 3, 4, 128, dtype=torch.bfloat16, device="cuda")
    packed[:, 1] = q
    out = torch.full((q.shape[0], 2, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    layers = [torch.stack((torch.zeros_like(x), x), 1) for x in b.cache[:2]]  # [page, layer, slot, head, D]
    layer = lib.KVCache(layers[0][:, 1], layers[1][:, 1], *b.cache[2:])
    lib.attn_fwd_cached(packed[:, 1], layer, out[:, 0], None, b.table, b.lens, b.starts, max_new=rows)
    o, _ = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
    assert torch.equal(out[:, 0], o) and bool((out[:, 1] == 3.0).all())
    # head-first queries [B, H, S, D] of a uniform batch, a wider table
    u = q.view(2, rows, 4, 128).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    wide = torch.full((2, 2 * b.table.shape[1]), -1, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = b.table
    uo, _ = lib.attention_cached(u, b.cache, wide[:, :b.table.shape[1]], b.lens)
    assert torch.equal(uo.flatten(0, 1), o)


@pytest.mark.parametrize("rows", [1, 3, 140])
def test_missing_pages_make_nan_of_the_rows_that_see_them(rows):
    b = Batch([(rows, 300), (rows, 300), (rows, 300), (rows, 300)], 1, 16, E4M3, seed=6)
    q = b.queries(2)
    good, good_lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=rows)
    table, lens = b.table.clone(), b.lens.clone()
    table[0, 12] = b.n_pages          # positions 192 .. 207
    table[1, 18] = -1                 # 288 .. 299
    lens[2] = 16 * table.shape[1] + 5  # beyond the table: the last block is -7, too
    o, lse = lib.attention_cached(q, b.cache, table, lens, b.starts, max_new=rows)
    for i, (seq, first) in enumerate(((0, 192), (1, 288), (3, 300))):
        at = slice(seq * rows, (seq + 1) * rows)
        sees = torch.arange(300 - rows, 300, device="cuda") >= first
        assert bool(o[at][sees].isnan().all()) and bool(lse[:, at][:, sees].isnan().all())
        # the others: both are within (2^-11 + little) sum p |v| + 2^-8 |o| of one number
        off = (o[at][~sees].float() - good[at][~sees].float()).abs()
        largest = max(float(b.values(1, x).abs().max()) for x in range(4))
        assert bool((off <= 2.0 ** -9 * largest + 2.0 ** -6 * good[at][~sees].float().abs()).all())
        assert bool(((lse[:, at][:, ~sees] - good_lse[:, at][:, ~sees]).abs() <= 1e-3).all())
    last = o[3 * rows - 1]
    assert bool(last.isnan().all())


def test_rows_behind_the_last_sequence_are_left():
    b = Batch([(1, 100), (150, 200)], 2, 16, INT8, seed=7)
    q = torch.cat((b.queries(4), torch.full((9, 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")))
    for hint in (1, 151):
        o = torch.full_like(q, 5.0)
        lse = torch.full((4, q.shape[0]), 5.0, device="cuda")
        lib.attn_fwd_cached(q, b.cache, o, lse, b.table, b.lens, b.starts, max_new=hint)
        assert bool((o[151:] == 5).all()) and bool((lse[:, 151:] == 5).all())
        check(b, q[:151], o[:151], lse[:, :151])


def test_pages_beyond_32_bits():
    """A cache of 5 GB whose last pages are read and written, and a page number times its stride far beyond 2^32."""
    page, heads = 128, 8
    n_pages = 5 * 2 ** 30 // (page * heads * 128)
    k = torch.empty(n_pages, heads, page, 128, dtype=INT8, device="cuda").transpose(1, 2)
    v = torch.empty(n_pages, heads, page, 128, dtype=INT8, device="cuda").transpose(1, 2)
    cache = lib.KVCache(k, v, *(torch.zeros(n_pages, heads, device="cuda") for _ in "kv"))
    small = lib.new_kv_cache(4, page, heads, INT8)
    g = torch.Generator(device="cuda").manual_seed(8)
    new_k, new_v = (rand(g, 1, 400, heads, 128).bfloat16() for _ in "kv")
    lens = torch.tensor([400], dtype=torch.int32, device="cuda")
    far = torch.tensor([[n_pages - 1, n_pages - 3, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[3, 1, 0, 2]], dtype=torch.int32, device="cuda")
    q = rand(g, 1, 200, 16, 128).bfloat16()
    out = []
    for c, t in ((cache, far), (small, near)):
        lib.kv_cache_append(c, new_k, new_v, t, lens)
        out.append((*lib.kv_cache_read(c, t, lens, n=400), *lib.attention_cached(q, c, t, lens),
                    *lib.attention_cached(q[:, -1:], c, t, lens)))
    assert all(torch.equal(a, b) for a, b in zip(*out))


# ---- append and read ----------------------------------------------------------------------------------------------

APPEND = [  # page, kind, heads, rounds of (rows, ...) a sequence
    (16, E4M3, 1, [(1, 5, 0), (1, 1, 3), (40, 0, 1)]),
    (32, INT8, 3, [(31, 33, 64), (1, 1, 1), (100, 7, 32)]),
    (64, E4M3, 2, [(64, 1, 200), (1, 63, 1), (65, 500, 0)]),
    (128, INT8, 5, [(1, 127, 300), (128, 1, 1), (1, 257, 90)]),
    (64, INT8, 2, [(0, 0, 1), (0, 70, 0)]),
    (128, E4M3, 4, [(700, 3, 1)]),
]


@pytest.mark.parametrize("page,kind,heads,rounds", APPEND)
@pytest.mark.parametrize("token_major", [False, True])
def test_append_and_read_match_definition(page, kind, heads, rounds, token_major):
    g = torch.Generator(device="cuda").manual_seed(page + heads)
    B = len(rounds[0])
    total = [sum(r[b] for r in rounds) for b in range(B)]
    blocks = [-(-t // page) for t in total]
    n_pages = sum(blocks) + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, max(blocks), dtype=torch.int32, device="cuda")
    ids, at = [], 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        ids.append(order[at:at + n].tolist())
        at += n
    if token_major:
        cache = lib.KVCache(*(torch.zeros(n_pages, page, heads, 128, dtype=kind, device="cuda") for _ in "kv"),
                            *(torch.full((n_pages, heads), 3.0, device="cuda") for _ in "kv"))
    else:
        cache = lib.new_kv_cache(n_pages, page, heads, kind)
        cache.k_scale.fill_(3.0)
        cache.v_scale.fill_(3.0)
    codes = [x.float().double().cpu() for x in cache[:2]]
    scales = [x.double().cpu() for x in cache[2:]]
    have = [0] * B
    for step, r in enumerate(rounds):
        starts = torch.tensor([0] + [sum(r[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
        rows = [(rand(g, sum(r), heads, 128) * torch.exp(rand(g, sum(r), heads, 1) * (1 + step))).bfloat16() for _ in "kv"]
        if step == 1 and rows[0].numel():
            rows[0][0] = 0
        lens = torch.tensor([h + n for h, n in zip(have, r)], dtype=torch.int32, device="cuda")
        lib.kv_cache_append(cache, *rows, table, lens, starts)
        for b, n in enumerate(r):
            for t in range(2):
                if n:
                    orc.append(codes[t], scales[t], rows[t][starts[b]:starts[b] + n].cpu(), ids[b], have[b], page, kind == INT8)
            have[b] += n
    for t in range(2):
        assert torch.equal(cache[2 + t].double().cpu(), scales[t])
        assert torch.equal(cache[t].float().double().cpu(), codes[t])
    # everything back, and the tails
    for n in (total, [min(t, 3) for t in total], [t // 2 for t in total]):
        starts = torch.tensor([0] + [sum(n[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
        back = lib.kv_cache_read(cache, table, torch.tensor(total, dtype=torch.int32, device="cuda"), starts, n=sum(n))
        for t in range(2):
            for b in range(B):
                full = orc.gather(cache[t].float(), cache[2 + t], ids[b], total[b], page)[total[b] - n[b]:] if n[b] else None
                got = back[t][starts[b]:starts[b + 1]]
                assert full is None or torch.equal(got, full.float().bfloat16())


@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("page", [16, 128])
def test_uniform_rows_strided(kind, page):
    g = torch.Generator(device="cuda").manual_seed(9)
    B, S, H = 3, 150, 2
    qkv = rand(g, B, S, 4 + 2 * H, 128).bfloat16()
    table = torch.arange(B * 20, dtype=torch.int32, device="cuda").view(B, 20)
    lens = torch.full((B,), S, dtype=torch.int32, device="cuda")
    a, b = lib.new_kv_cache(B * 20, page, H, kind), lib.new_kv_cache(B * 20, page, H, kind)
    lib.kv_cache_append(a, qkv[:, :, 4:4 + H], qkv[:, :, 4 + H:], table, lens)
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda") * S
    lib.kv_cache_append(b, qkv[:, :, 4:4 + H].flatten(0, 1), qkv[:, :, 4 + H:].contiguous().flatten(0, 1), table, lens, starts)
    for x, y in zip(a, b):
        assert torch.equal(x.float(), y.float())
    before = [x.clone() for x in a]
    lib.kv_cache_append(a, qkv[:, :, 4:4 + H], qkv[:, :, 4 + H:], table, lens)  # the same again
    for x, y in zip(a, before):
        assert torch.equal(x.float(), y.float())
    out = torch.zeros(B, S, 3, H, 128, dtype=torch.bfloat16, device="cuda")
    lib.attn_kv_read(a, out[:, :, 0], out[:, :, 2], table, lens)
    k, v = lib.kv_cache_read(b, table, lens, n=S)
    assert torch.equal(out[:, :, 0], k) and torch.equal(out[:, :, 2], v) and not bool(out[:, :, 1].any())


@pytest.mark.parametrize("kind", [E4M3, INT8])
def test_values_that_are_not_finite_or_extreme(kind):
    cache = lib.new_kv_cache(2, 16, 1, kind)
    k = torch.ones(1, 4, 1, 128, dtype=torch.bfloat16, device="cuda")
    k[0, 0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1.75])
    v = torch.zeros_like(k)
    v[0, 0, 0, 0] = 3.38e38
    v[0, 1, 0, 0] = 1e-39
    table = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([4], dtype=torch.int32, device="cuda")
    lib.kv_cache_append(cache, k, v, table, lens)
    codes = cache.k[1, 0, 0, :4].float().tolist()
    if kind == E4M3:
        assert float(cache.k_scale[1, 0]) == 2.0 ** -8 and codes[:2] == [448, -448] and math.isnan(codes[2]) and codes[3] == 448
    else:
        assert codes[:3] == [127, -127, 0] and codes[3] == 127
    x = float(v[0, 0, 0, 0])
    kept, _ = lib.kv_cache_read(lib.KVCache(cache.v, cache.v, cache.v_scale, cache.v_scale), table, lens, n=4)
    if kind == E4M3:  # x is 254 * 2^120 (rounded to BF16), the nearest codes are 240 and 256, and 256 * 2^120 = 2^128 is no BF16 number
        assert x / 2.0 ** 120 == 254 and float(kept[0, 0, 0, 0]) == math.inf and float(cache.v[1, 0, 0, 0].float()) == 256
    else:
        assert abs(float(kept[0, 0, 0, 0]) - x) <= x * (2.0 ** -8 + 2.0 ** -8)
    # nothing but tiny values, then nothing but zeros
    tiny = torch.full((1, 16, 1, 128), 1e-39, dtype=torch.bfloat16, device="cuda")
    lens[0] = 16
    lib.kv_cache_append(cache, tiny, torch.zeros_like(tiny), table, lens)
    assert float(cache.k_scale[1, 0]) == 2.0 ** -100 and float(cache.v_scale[1, 0]) == 0.0
    assert not bool(cache.v[1].float().any())


@pytest.mark.parametrize("kind", [E4M3, INT8])
def test_missing_pages_and_short_sequences_in_append_and_read(kind):
    cache = lib.new_kv_cache(4, 16, 2, kind)
    g = torch.Generator(device="cuda").manual_seed(10)
    rows = [rand(g, 60, 2, 128).bfloat16() for _ in "kv"]
    table = torch.tensor([[0, 9, 1], [-1, 2, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 10], dtype=torch.int32, device="cuda")  # 20 rows each and 20 that belong to nobody
    starts = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    lib.kv_cache_append(cache, *rows, table, lens, starts)  # positions 20 .. 39: page 9 does not exist; -10 .. 9: block 0 does not
    assert not bool(cache.k[0].float().any()) and not bool(cache.k[2:].float().any())
    assert bool(cache.k[1, :8].float().any()) and not bool(cache.k[1, 8:].float().any())
    out = [torch.full_like(rows[0], 4.0) for _ in "kv"]
    lib.attn_kv_read(cache, *out, table, lens, starts)
    for x, r in zip(out, rows):
        assert bool(x[:12].isnan().all()) and not bool(x[12:20].isnan().any())
        assert bool((x[20:30] == 0).all()) and bool(x[30:40].isnan().all()) and bool((x[40:] == 4).all())
    lens = torch.tensor([60, 60], dtype=torch.int32, device="cuda")  # beyond the table
    lib.kv_cache_append(cache, *rows, table, lens, starts)
    lib.attn_kv_read(cache, *out, table, lens, starts)
    assert bool(out[0][8:20].isnan().all()) and bool(out[1][28:40].isnan().all())


# ---- together, on streams, captured -----------------------------------------------------------------------------------

def test_a_conversation():
    """Prompt, chunk and decoding steps through norm and rotation, cache and attention, against BF16 attention over what the
    cache gives back."""
    g = torch.Generator(device="cuda").manual_seed(11)
    B, hq, hkv, page = 2, 8, 2, 16
    cache = lib.new_kv_cache(B * 20, page, hkv)
    table = torch.randperm(B * 20, generator=g, device="cuda").to(torch.int32).view(B, 20)
    angle = torch.arange(400, device="cuda")[:, None] * 1e4 ** (-torch.arange(0, 128, 2, device="cuda") / 128)
    done = 0
    for n in (100, 37, 1, 1, 1):
        q, k, v = (rand(g, B, n, h, 128).bfloat16() for h in (hq, hkv, hkv))
        positions = (done + torch.arange(n, device="cuda")).expand(B, n)
        q, k = lib.qk_norm_rope(q, k, None, None, angle.cos(), angle.sin(), positions=positions)
        done += n
        lens = torch.full((B,), done, dtype=torch.int32, device="cuda")
        lib.kv_cache_append(cache, k, v, table, lens)
        o, lse = lib.attention_cached(q, cache, table, lens)
        all_k, all_v = lib.kv_cache_read(cache, table, lens, n=done)  # powers of two: E4M3 values are exact in BF16
        want, want_lse = lib.attention_forward(q, all_k, all_v, causal=True)
        # the BF16 path rounds its weights to 8 bits
        assert bool(((o.float() - want.float()).abs() <= 2e-2).all()) and bool(((lse - want_lse).abs() <= 1e-3).all())
        b = Batch.__new__(Batch)
        b.seqs, b.rows, b.page, b.heads, b.cache = [(n, done)] * B, [0, n, 2 * n], page, hkv, cache
        b.ids = [table[i].long() for i in range(B)]
        check(b, q.flatten(0, 1), o.flatten(0, 1), lse.permute(1, 0, 2).flatten(1))


@pytest.mark.parametrize("rows", [1, 140])
def test_other_stream_and_captured(rows):
    b = Batch([(rows, 900), (rows, 1400)], 2, 32, E4M3, seed=12)
    q = b.queries(8)
    k, v = (rand(b.g, q.shape[0], 2, 128).bfloat16() for _ in "kv")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lib.kv_cache_append(b.cache, k, v, b.table, b.lens, b.starts)
        o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts)
    torch.cuda.current_stream().wait_stream(side)
    check(b, q, o, lse)
    out = torch.empty_like(o)
    lib.attn_fwd_cached(q, b.cache, out, None, b.table, b.lens, b.starts, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(out, o)
    # a captured step follows its inputs: new queries, keys and lengths in the same buffers
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.kv_cache_append(b.cache, k, v, b.table, b.lens, b.starts)
        o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts)
    q.copy_(b.queries(8))
    k.copy_(rand(b.g, *k.shape))
    b.lens -= 13
    b.seqs = [(rows, 887), (rows, 1387)]
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        check(b, q, o, lse)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, on one cache."""
    b = Batch([(1, 5000), (1, 3000)], 4, 64, E4M3, seed=13)
    c = Batch([(100, 1500)], 4, 64, INT8, seed=14)
    qs = [b.queries(16), c.queries(16)]
    want = [lib.attention_cached(q, x.cache, x.table, x.lens, x.starts) for q, x in zip(qs, (b, c))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = []
        for s, q, x in zip(streams, qs, (b, c)):
            with torch.cuda.stream(s):
                got.append(lib.attention_cached(q, x.cache, x.table, x.lens, x.starts))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


@pytest.mark.parametrize("group,page,kind", [(4, 32, E4M3), (16, 16, INT8), (1, 128, E4M3)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_and_short_sequences_in_one_batch(group, page, kind, causal):
    """Prompts next to single tokens, sequences without rows and without tokens: each row is written once, whichever kernel has it."""
    seqs = [(1, 900), (300, 700), (0, 40), (1, 1), (2, 333), (65, 65), (8, 500), (1, 0), (9, 129), (1, 2500), (17, 17)]
    b = Batch(seqs, 2, page, kind, seed=group, scale_spread=1.0)
    q = b.queries(2 * group)
    o = torch.full_like(q, 7.0)
    lse = torch.full((2 * group, q.shape[0]), 7.0, device="cuda")
    lib.attn_fwd_cached(q, b.cache, o, lse, b.table, b.lens, b.starts, max_new=300, causal=causal)
    check(b, q, o, lse, causal)


def test_many_sequences_on_shared_pages():
    """4096 sequences of 32768 tokens, all on the same 512 pages (a table whose rows are one): a million steps of work, where the cut
    needs 64 bits, and more sequences than a warp counts."""
    b = Batch([(1, 32768)], 1, 64, E4M3, seed=20, spare=0)
    B = 4096
    q = (rand(b.g, 4, 8, 128)).bfloat16().repeat(B // 4, 1, 1)[:, None].contiguous()
    o, lse = lib.attention_cached(q, b.cache, b.table.expand(B, -1), b.lens.expand(B).contiguous())
    one = Batch.__new__(Batch)
    one.seqs, one.rows, one.page, one.heads, one.cache, one.ids = [(1, 32768)] * 4, [0, 1, 2, 3, 4], 64, 1, b.cache, b.ids * 4
    for first in (0, 4, 2048, B - 4):
        check(one, q[first:first + 4, 0], o[first:first + 4, 0], lse[first:first + 4, :, 0].T.contiguous())
    # every sequence's result is within the bounds of the same numbers: of those that share a query, none differs by more than both
    spread = (o.view(B // 4, 4, 8, 128).float().amax(0) - o.view(B // 4, 4, 8, 128).float().amin(0)).max()
    assert float(spread) <= 2.0 ** -9 * float(b.values(1, 0).abs().max()) + 2.0 ** -6 * float(o.float().abs().max())


@pytest.mark.parametrize("kind", [E4M3, INT8])
def test_forty_long_sequences(kind):
    """More sequences than a warp counts, in the kernel for many rows, keys and values in different orders in memory."""
    seqs = [(30 + 7 * i, 200 + 31 * i) for i in range(40)]
    b = Batch(seqs, 2, 32, kind, seed=21)
    v = torch.zeros(b.n_pages, 32, 2, 128, dtype=kind, device="cuda")  # slot by slot, the keys head by head
    v.view(torch.uint8).copy_(b.cache.v.view(torch.uint8))
    b.cache = lib.KVCache(b.cache.k, v, *b.cache[2:])
    q = b.queries(6)
    o, lse = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=max(n for n, _ in seqs))
    check(b, q, o, lse)
    small, _ = lib.attention_cached(q, b.cache, b.table, b.lens, b.starts, max_new=3)
    check(b, q, small, None)


def test_outputs_that_start_at_16_bytes():
    """Rows of o at odd multiples of 16 bytes, in the kernel that writes 32 at a time."""
    b = Batch([(200, 500)], 2, 64, E4M3, seed=22)
    q = b.queries(4)
    wide = torch.full((200, 4, 136 * 2), 9.0, dtype=torch.bfloat16, device="cuda")
    for at in (8, 16):
        o = wide[:, :, at:at + 128]
        lib.attn_fwd_cached(q, b.cache, o, None, b.table, b.lens, b.starts)
        check(b, q, o, None)
    assert bool((wide[:, :, :8] == 9).all()) and bool((wide[:, :, 144:] == 9).all())
