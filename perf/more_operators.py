"""The paged 8-bit key/value cache of serving, as cases that can be timed and compared with their plain forms.

Three calls a user makes around ``attention_forward`` once keys and values outlive the call:

* ``kv_cache_append``   quantises the keys and values of new tokens into the pages of their sequences, a scale for each page and head;
* ``kv_cache_read``     gives the last tokens of each sequence back in BF16;
* ``attention_cached``  attention of new tokens (one, a few, a long chunk) over the pages of their sequences.

Sequence b owns the rows ``starts[b] .. starts[b + 1]`` of a packed batch (or S rows each of a [B, S, H, D] batch); they stand at its
positions ``seq_lens[b] - n .. seq_lens[b] - 1``, and position p is slot ``p % page`` of page ``block_table[b, p // page]``.

A page and head has one scale.  E4M3: the smallest power of two that brings the largest magnitude to 448 or less; INT8: the largest
magnitude / 127.  A page that already holds tokens keeps the larger of its scale and the new tokens' one; where that is larger than
it was, the codes it holds are rounded to the new scale.

``own = False`` computes them by elementary torch operations in 32 bits, ``own = True`` by the library.
"""
import math
import random

import torch

own = False

D = 128            # head dimension of every path of the library
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
PAIRS = 1 << 27    # scores that the plain form holds at a time


def listed():
    return [
        # one decoding step of 8 conversations: the new token's keys and values into the middle of a page
        case("append_decode_b8", "append", 8, 8, 8, 64, "e4m3", 1, 4096, "ragged"),
        # a prefill of 32768 tokens, as 4 sequences
        case("append_prefill_32k", "append", 4, 8, 8, 64, "e4m3", 8192, 0, "same"),
        # ragged chunks behind earlier ones, small pages, few heads
        case("append_ragged_int8", "append", 7, 4, 4, 16, "int8", 1500, 777, "ragged"),
        # 4 cached prompts of 8192 tokens back in BF16 (to hand on, or to run the BF16 path over them)
        case("read_32k", "read", 4, 8, 8, 64, "e4m3", 8192, 0, "same"),
        # the tails of 9 sequences
        case("read_tails_int8", "read", 9, 5, 5, 32, "int8", 700, 3000, "ragged"),
        # one short conversation, one token: a call's latency
        case("decode_b1_s512", "attend", 1, 16, 16, 64, "e4m3", 1, 511, "same"),
        # a decoding step of 64 conversations, grouped queries
        case("decode_b64_s8192", "attend", 64, 32, 8, 64, "e4m3", 1, 8191, "ragged"),
        # one token behind a very long document, eight query heads a key head
        case("decode_b1_s131072_int8", "attend", 1, 32, 4, 128, "int8", 1, 131071, "same"),
        # 4 proposed tokens verified for each of 16 sequences, small pages
        case("verify_b16_int8", "attend", 16, 32, 4, 16, "int8", 4, 12000, "ragged"),
        # 512 new rows behind a 65536-key context (the library's own chunk workload, over the cache)
        case("chunk_512_of_65536", "attend", 1, 16, 16, 64, "e4m3", 512, 65024, "same"),
        # a server's step: prompts of different lengths next to conversations that decode
        case("mixed_step_b24", "attend", 24, 32, 8, 32, "e4m3", 1001, 6000, "mixed"),
        # the last 8192 tokens of a 32768-token prompt
        case("prefill_8192_of_32768", "attend", 1, 32, 8, 64, "e4m3", 8192, 24576, "same"),
    ]


def case(name, op, batch, hq, hkv, page, kind, new, context, lengths):
    return {"name": name, "op": op, "batch": batch, "hq": hq, "hkv": hkv, "page": page, "kind": kind, "new": new,
            "context": context, "lengths": lengths}


def _lengths(c):
    """New tokens and tokens in all of each sequence."""
    if c["lengths"] == "same":
        return [c["new"]] * c["batch"], [c["context"] + c["new"]] * c["batch"]
    rng = random.Random(c["batch"] * 1000003 + c["new"] * 1009 + c["context"])
    new, total = [], []
    for b in range(c["batch"]):
        n = c["new"] if b == 0 else rng.randint((c["new"] + 1) // 2, c["new"]) if c["new"] <= 8 else rng.randint(1, c["new"])
        if c["lengths"] == "mixed" and b % 8:  # seven of eight sequences decode
            n = 1
        new.append(n)
        total.append(n + (c["context"] if b == 0 else rng.randint(c["context"] // 3, c["context"])))
    return new, total


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend", "attend"])
    hkv = rng.choice([1, 2, 4, 5, 8, 16])
    hq = hkv * (rng.choice([1, 2, 3, 4, 6, 7, 8]) if op == "attend" else 1)
    batch = _log_uniform(rng, 1, 64)
    context = _log_uniform(rng, 1, 131072)
    kind = rng.random()
    new = 1 if kind < 0.4 else rng.randint(2, 8) if kind < 0.55 else _log_uniform(rng, 9, 8192)
    if op == "read":
        new = _log_uniform(rng, 1, 8192)
    while batch * (context + new) * hkv > 64 * 8192 * 8 or batch * new * (context + new) * hq > 8192 * 32768 * 32:
        batch, context, new = (batch + 1) // 2, (context + 1) // 2, (new + 1) // 2
    c = case("", op, batch, hq, hkv, rng.choice([16, 32, 64, 128]), rng.choice(["e4m3", "int8"]), new, context,
             rng.choice(["same", "ragged", "ragged", "mixed"]))
    del c["name"]
    return c


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, n, heads):
    """Keys of n tokens, some channels stronger than others as a learned norm leaves them."""
    return (_normal(gen, n, heads, D) * (1.0 + 0.3 * _normal(gen, heads, D))).to(torch.bfloat16)


def _values(gen, n, heads):
    """Values of n tokens, some tokens stronger than others."""
    return (_normal(gen, n, heads, D) * torch.exp(0.4 * _normal(gen, n, heads, 1))).to(torch.bfloat16)


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new, total = _lengths(c)
    B, Hkv, page, kind = c["batch"], c["hkv"], c["page"], TYPES[c["kind"]]
    blocks = [-(-t // page) for t in total]
    n_pages = sum(blocks) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(B, max(blocks) + 1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    # pages lie head by head, [page, head, slot, D] in memory
    codes = [torch.zeros(n_pages, Hkv, page, D, dtype=kind, device="cuda").transpose(1, 2) for _ in "kv"]
    scales = [torch.zeros(n_pages, Hkv, dtype=torch.float32, device="cuda") for _ in "kv"]
    st = {"op": c["op"], "page": page, "table": table, "new": new, "total": total,
          "lens": torch.tensor(total, dtype=torch.int32, device="cuda"),
          "k_codes": codes[0], "v_codes": codes[1], "k_scale": scales[0], "v_scale": scales[1],
          "starts": None if c["lengths"] == "same" else torch.tensor(starts, dtype=torch.int32, device="cuda")}
    if c["op"] == "append":
        for b in range(B):  # what earlier steps have left
            if total[b] > new[b]:
                n = total[b] - new[b]
                _append_one(st, b, _keys(gen, n, Hkv), _values(gen, n, Hkv), 0)
        k, v = _keys(gen, starts[-1], Hkv), _values(gen, starts[-1], Hkv)
        st["k"], st["v"] = (x if st["starts"] is not None else x.view(B, c["new"], Hkv, D) for x in (k, v))
        return st
    # slots that no token has been written to hold what an earlier owner left
    for x in codes:
        raw = x.transpose(1, 2).view(torch.uint8)
        raw.copy_(torch.randint(0, 256, raw.shape, generator=gen, device="cuda", dtype=torch.uint8))
    for b in range(B):
        _append_one(st, b, _keys(gen, total[b], Hkv), _values(gen, total[b], Hkv), 0)
    if c["op"] == "attend":
        q = _normal(gen, starts[-1], c["hq"], D).to(torch.bfloat16)
        st["q"] = q if st["starts"] is not None else q.view(B, c["new"], c["hq"], D)
    return st


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "append":
        k, v = (x.flatten(0, 1) if st["starts"] is None else x for x in (st["k"], st["v"]))
        row = 0
        for b, n in enumerate(st["new"]):
            _append_one(st, b, k[row:row + n], v[row:row + n], st["total"][b] - n)
            row += n
        return st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"]
    if st["op"] == "read":
        out = [torch.cat([_values_of(st, x, b)[st["total"][b] - n:].to(torch.bfloat16) for b, n in enumerate(st["new"])]) for x in "kv"]
        return [x if st["starts"] is not None else x.view(len(st["new"]), -1, *x.shape[1:]) for x in out]
    q = st["q"].flatten(0, 1) if st["starts"] is None else st["q"]
    row, o, lse = 0, [], []
    for b, n in enumerate(st["new"]):
        o_b, lse_b = _attend_one(q[row:row + n], _values_of(st, "k", b), _values_of(st, "v", b))
        o.append(o_b)
        lse.append(lse_b)
        row += n
    if st["starts"] is None:
        return torch.stack(o), torch.stack(lse)
    return torch.cat(o), torch.cat(lse, 1)


def _run_own(st):
    import paper_2603_24517_b200 as lib

    cache = lib.KVCache(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"])
    where = (st["table"], st["lens"], st["starts"])
    if st["op"] == "append":
        lib.kv_cache_append(cache, st["k"], st["v"], *where)
        return tuple(cache)
    if st["op"] == "read":
        return lib.kv_cache_read(cache, *where, n=st["new"][0] if st["starts"] is None else sum(st["new"]))
    return lib.attention_cached(st["q"], cache, *where, max_new=max(st["new"]))


# ---- plain forms ---------------------------------------------------------------------------------------

def _scale_for(largest, kind):
    """The scale of a page and head whose largest magnitude is `largest`."""
    if kind == torch.int8:
        s = largest / 127.0
    else:
        m, e = torch.frexp(largest)  # largest = m 2^e, m in [1/2, 1); 448 = (7 / 8) 2^9
        s = torch.ldexp(torch.ones_like(largest), torch.where(m <= 0.875, e - 9, e - 8))
    return torch.where(largest > 0, s.clamp(min=2.0 ** -100), torch.zeros_like(largest))


def _encode(x, scale, kind):
    """Codes of the values x at a scale of their shape."""
    y = x / torch.where(scale > 0, scale, torch.ones_like(scale))
    if kind == torch.int8:
        return y.round().clamp(-127, 127).to(kind)
    return y.clamp(-448, 448).to(kind)


def _append_one(st, b, k, v, begin):
    """Rows k, v of one sequence at the positions from `begin` on."""
    page, n = st["page"], k.shape[0]
    first, last = begin // page, (begin + n - 1) // page
    pages = st["table"][b, first:last + 1].long()
    lead = begin - first * page  # slots of the first page that hold earlier tokens
    for name, x in (("k", k), ("v", v)):
        codes, scales = st[name + "_codes"], st[name + "_scale"]
        kind = codes.dtype
        room = torch.zeros((len(pages) * page,) + x.shape[1:], device=x.device)
        room[lead:lead + n] = x.float()
        room = room.view(len(pages), page, *x.shape[1:])
        scale = _scale_for(room.abs().amax((1, 3)), kind)
        if lead:
            before = scales[pages[0]]
            scale[0] = torch.maximum(scale[0], before)
            old = codes[pages[0], :lead].float() * before[None, :, None]
            codes[pages[0], :lead] = _encode(old, scale[0][None, :, None].expand_as(old), kind)
        enc = _encode(room, scale[:, None, :, None].expand_as(room), kind).flatten(0, 1)[lead:lead + n]
        slot = torch.arange(begin, begin + n, device=x.device)
        codes[st["table"][b, slot // page].long(), slot % page] = enc
        scales[pages] = scale


def _values_of(st, name, b):
    """fp32 [length, heads, D]: what the cache holds for sequence b."""
    n = st["total"][b]
    pages = st["table"][b, :-(-n // st["page"])].long()
    x = st[name + "_codes"][pages].float() * st[name + "_scale"][pages][:, None, :, None]
    return x.flatten(0, 1)[:n]


def _attend_one(q, k, v):
    """q BF16 [n, Hq, D] at the last n of the positions of k, v fp32 [L, Hkv, D] -> o BF16 like q, lse [Hq, n]."""
    n, hq, _ = q.shape
    L, hkv, _ = k.shape
    kt, vt = k.permute(1, 2, 0), v.permute(1, 0, 2)
    step = max(1, PAIRS // (hq * L))
    o, lse = [], []
    for i in range(0, n, step):
        rows = q[i:i + step].float()
        m = rows.shape[0]
        g = rows.view(m, hkv, hq // hkv, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)
        s = (g @ kt).mul_(1.0 / math.sqrt(D)).view(hkv, hq // hkv, m, L)
        if m > 1 or i + m < n:
            hidden = torch.arange(L, device=q.device) > torch.arange(L - n + i, L - n + i + m, device=q.device)[:, None]
            s.masked_fill_(hidden, -math.inf)
        z = torch.logsumexp(s, -1)
        p = s.sub_(z[..., None]).exp_().view(hkv, -1, L)
        o.append((p @ vt).view(hkv, hq // hkv, m, D).permute(2, 0, 1, 3).reshape(m, hq, D).to(torch.bfloat16))
        lse.append(z.reshape(hq, m))
    return torch.cat(o), torch.cat(lse, 1)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(c):
    new, total = _lengths(c)
    B, Hq, Hkv, page = c["batch"], c["hq"], c["hkv"], c["page"]
    T = sum(new)
    if c["op"] in ("append", "read"):  # 2 bytes on one side, 1 on the other, keys and values; scales; page numbers
        pages = sum((t - 1) // page - (t - n) // page + 1 for n, t in zip(new, total))
        extra = (4 if c["op"] == "append" else 2) * Hkv * pages * 4 // 2 + pages * 4 + B * 8
        return {"bytes": T * Hkv * D * 3 * 2 + extra, "flops": T * Hkv * D * 2 * 2}
    pages = sum(-(-t // page) for t in total)
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(new, total))
    return {"bytes": sum(total) * Hkv * D * 2 + pages * (Hkv * 8 + 4) + T * Hq * (D * 4 + 4) + B * 8, "flops": 4 * Hq * pairs * D}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def exact(c, seed):
    st = prepare(c, seed)
    new, total = st["new"], st["total"]
    page = st["page"]
    if c["op"] == "append":
        return _exact_append(c, st)
    # every slot's value, then the sequence's own ones in their order
    table = {}
    for name in "kv":
        table[name] = st[name + "_codes"].to(torch.float32).double() * st[name + "_scale"].double()[:, None, :, None]
    out = [[], []]
    for b, (n, t) in enumerate(zip(new, total)):
        at = torch.arange(t, device="cuda")
        page_of, slot = st["table"][b, torch.div(at, page, rounding_mode="floor")].long(), at % page
        K, V = table["k"][page_of, slot], table["v"][page_of, slot]
        if c["op"] == "read":
            out[0].append(K[t - n:])
            out[1].append(V[t - n:])
            continue
        Q = (st["q"][b] if st["starts"] is None else st["q"][int(sum(new[:b])):int(sum(new[:b])) + n]).double()
        G = c["hq"] // c["hkv"]
        o, z = torch.empty(n, c["hq"], D, dtype=torch.float64, device="cuda"), torch.empty(c["hq"], n, dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // t)
        for h in range(c["hq"]):
            for i in range(0, n, step):
                j = min(n, i + step)
                s = torch.einsum("id,jd->ij", Q[i:j, h], K[:, h // G]) * D ** -0.5
                seen = at[None] < torch.arange(t - n + i + 1, t - n + j + 1, device="cuda")[:, None]
                top = torch.where(seen, s, s.new_full((), -math.inf)).max(1).values
                w = torch.where(seen, torch.exp(s - top[:, None]), s.new_zeros(()))
                z[h, i:j] = top + torch.log(w.sum(1))
                o[i:j, h] = torch.einsum("ij,jd->id", w, V[:, h // G]) / w.sum(1)[:, None]
        out[0].append(o)
        out[1].append(z)
    if st["starts"] is None:
        return torch.stack(out[0]), torch.stack(out[1])
    return torch.cat(out[0]), torch.cat(out[1], 0 if c["op"] == "read" else 1)


def _exact_append(c, st):
    """The codes as numbers and the scales.  INT8 codes have no 64-bit value: the definition divides by a scale of 32 bits."""
    new, total, page, e4m3 = st["new"], st["total"], st["page"], c["kind"] == "e4m3"
    answer = []
    for name in "kv":
        codes, scales = st[name + "_codes"].to(torch.float32).double(), st[name + "_scale"].double()
        rows = (st[name].flatten(0, 1) if st["starts"] is None else st[name]).double()
        owner = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        place = torch.cat([torch.arange(t - n, t) for n, t in zip(new, total)]).cuda()
        where = st["table"][owner, place // page].long()
        begin = torch.tensor(total).cuda()[owner] - torch.tensor(new).cuda()[owner]
        top = torch.zeros_like(scales).index_reduce_(0, where, rows.abs().amax(2), "amax")
        if e4m3:
            part, power = torch.frexp(top / 448)  # in [1/2, 1); 1/2 is a power of two itself
            need = torch.where(top > 0, torch.ldexp(torch.ones_like(top), power - (part == 0.5).int()), top)
        else:
            need = top / 127
        touched = torch.zeros(len(scales), dtype=torch.bool, device="cuda")
        touched[where] = True
        kept = torch.zeros_like(touched)  # pages that hold earlier tokens too
        kept[where[(place // page) == (begin // page)]] = True
        first = place == begin
        kept[where[first & (begin % page == 0)]] = False
        after = torch.where(touched[:, None], torch.where(kept[:, None], torch.maximum(need, scales), need), scales)
        safe = torch.where(after > 0, after, torch.ones_like(after))

        def rounded(x):  # to the nearest E4M3 number, ties to even: 3 bits behind the first, steps of 2^-9 at the least
            power = torch.frexp(x.abs().clamp(min=2.0 ** -6))[1]
            unit = torch.ldexp(torch.ones_like(x), power - 4)
            return torch.round(x / unit) * unit

        if e4m3:
            old = codes * scales[:, None, :, None] / safe[:, None, :, None]
            full = torch.where(kept[:, None, None, None], rounded(old), codes)
            full[where, place % page] = rounded(rows / safe[where][:, :, None])
            answer.append(full)
        else:
            answer.append(None)
        answer.append(after)
    return answer[0], answer[2], answer[1], answer[3]
