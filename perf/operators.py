"""The training-side attention operators, as cases that can be timed and compared with their plain forms.

Three calls a user makes around ``attention_forward``:

* ``qk_norm_rope``            queries and keys are normalised per head (root mean square, learned weight) and rotated by position;
* ``attention_backward``      dq, dk, dv of the attention forward pass, from its inputs, its result and its log-sum-exp;
* ``qk_norm_rope_backward``   the gradient of the first with respect to queries, keys and both weights.

``own = False`` computes them by elementary torch operations in 32 bits, ``own = True`` by the library.
"""
import math

import torch

own = False

D = 128          # head dimension of every path of the library
LOG2_MAX = 31    # a case's score matrix has at most 2^31 elements
EPS = 1e-6


def listed():
    return [
        # one short sequence, two heads (the library's smallest benchmark workload): latency of a backward call
        bwd("bwd_mha_tiny_s512", 1, 2, 2, 512, 512, False),
        # pre-training batch, the benchmark's 32768 tokens as 8 sequences
        bwd("bwd_mha_causal_s4096", 8, 16, 16, 4096, 4096, True),
        # long bidirectional sequence (encoder, document model), heads of one device
        bwd("bwd_mha_noncausal_s16384", 1, 8, 8, 16384, 16384, False),
        # grouped-query training: four query heads share a key head, gradients of shared heads add up
        bwd("bwd_gqa4_causal_s8192", 1, 32, 8, 8192, 8192, True),
        # cross attention of ragged lengths, eight query heads a key head, neither length a multiple of a tile
        bwd("bwd_gqa8_cross_ragged", 3, 32, 4, 1001, 1537, False),
        # 512 new rows behind a 65536-key context (fine-tuning on the tail of a long document), sharper scores
        bwd("bwd_mha_chunk_512_of_65536", 1, 16, 16, 512, 65536, True, 4.0),
        # one decoding step of 4 sequences, far and different positions, a step's latency
        rope("rope_decode_b4", False, 4, 1, 32, 8, 128, False, "bf16", True, False, 131072),
        # the queries and keys of a training step, 32768 tokens
        rope("rope_gqa4_32k", False, 4, 8192, 32, 8, 128, False, "bf16", False, False, 8192),
        # ragged batch on slices of a packed QKV projection, adjacent pairs, half of the head rotated
        rope("rope_packed_ragged", False, 3, 1237, 16, 16, 64, True, "f32", True, True, 40960),
        # gradients of the training step's norm and rotation
        rope("rope_bwd_gqa4_32k", True, 4, 8192, 32, 8, 128, False, "bf16", False, False, 8192),
        # gradients for one ragged micro-batch, packed projection
        rope("rope_bwd_packed_ragged", True, 2, 777, 16, 16, 64, True, "f32", True, True, 40960),
    ]


def bwd(name, batch, hq, hkv, sq, sk, causal, q_gain=1.0):
    return {"name": name, "op": "bwd", "batch": batch, "hq": hq, "hkv": hkv, "sq": sq, "sk": sk, "causal": causal,
            "q_gain": q_gain}


def rope(name, backward, batch, seq, hq, hkv, rot, interleaved, weights, positions, packed, table):
    return {"name": name, "op": "rope_bwd" if backward else "rope", "batch": batch, "seq": seq, "hq": hq, "hkv": hkv,
            "rot": rot, "interleaved": interleaved, "weights": weights, "positions": positions, "packed": packed,
            "table": table}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        hkv = rng.choice([1, 2, 3, 4, 8, 16])
        hq = hkv * rng.choice([1, 1, 2, 3, 4, 8])
        batch = rng.choice([1, 1, 2, 3, 4, 8])
        sk = _log_uniform(rng, 2, 65536)  # one key alone has the weight 1, and no gradient but rounding
        sq = sk if rng.random() < 0.5 else _log_uniform(rng, 1, 16384)
        while batch * hq * sq * sk > 1 << LOG2_MAX or batch * (hq * sq + hkv * sk) > 1 << 20:
            sq, sk = (sq + 1) // 2, (sk + 2) // 2
        case = bwd("", batch, hq, hkv, sq, sk, rng.random() < 0.6, rng.choice([1.0, 1.0, 2.0, 4.0]))
    else:
        hkv = rng.choice([1, 2, 4, 5, 8, 16])
        hq = hkv * rng.choice([1, 2, 4, 7, 8])
        seq = _log_uniform(rng, 1, 8192)
        batch = _log_uniform(rng, 1, 64)
        while batch * seq * (hq + hkv) > 32768 * 36:
            batch, seq = (batch + 1) // 2, (seq + 1) // 2
        positions = rng.random() < 0.6
        table = rng.choice([40960, 131072]) if positions else max(seq, rng.choice([2048, 8192]))
        case = rope("", rng.random() < 0.5, batch, seq, hq, hkv, rng.choice([128, 128, 64, 32, 96]),
                    rng.random() < 0.4, rng.choice(["bf16", "f32"]), positions, rng.random() < 0.4, table)
    del case["name"]
    return case


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "bwd":
        B, Hq, Hkv, Sq, Sk = (case[n] for n in ("batch", "hq", "hkv", "sq", "sk"))
        q = (_normal(gen, B, Sq, Hq, D) * case["q_gain"]).to(torch.bfloat16)
        k = _normal(gen, B, Sk, Hkv, D).to(torch.bfloat16)
        v = _normal(gen, B, Sk, Hkv, D).to(torch.bfloat16)
        do = _normal(gen, B, Sq, Hq, D).to(torch.bfloat16)
        scale = 1.0 / math.sqrt(D)
        o, lse = _attention(q, k, v, case["causal"], scale)  # what the forward pass has left
        return {"op": "bwd", "q": q, "k": k, "v": v, "do": do, "o": o, "lse": lse, "causal": case["causal"],
                "scale": scale}
    B, S, Hq, Hkv, R = (case[n] for n in ("batch", "seq", "hq", "hkv", "rot"))
    if case["packed"]:  # slices of a fused projection's output
        qkv = _normal(gen, B, S, Hq + 2 * Hkv, D).to(torch.bfloat16)
        q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    else:
        q, k = _normal(gen, B, S, Hq, D).to(torch.bfloat16), _normal(gen, B, S, Hkv, D).to(torch.bfloat16)
    wt = torch.bfloat16 if case["weights"] == "bf16" else torch.float32
    wq, wk = ((1.0 + 0.2 * _normal(gen, D)).to(wt) for _ in range(2))
    # the tables a model keeps: angles in 64 bits, rounded once
    freq = 500000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    angle = torch.arange(case["table"], device="cuda", dtype=torch.float64)[:, None] * freq
    state = {"op": case["op"], "q": q, "k": k, "wq": wq, "wk": wk, "cos": angle.cos().float(), "sin": angle.sin().float(),
             "positions": None, "interleaved": case["interleaved"]}
    if case["positions"]:  # every sequence continues at a place of its own
        start = torch.randint(0, max(1, case["table"] - S), (B, 1), generator=gen, device="cuda")
        state["positions"] = (start + torch.arange(S, device="cuda")) % case["table"]
    if case["op"] == "rope_bwd":
        state["dq"], state["dk"] = _normal(gen, B, S, Hq, D).to(torch.bfloat16), _normal(gen, B, S, Hkv, D).to(torch.bfloat16)
    return state


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "bwd":
        return _attention_backward(state["do"], state["q"], state["k"], state["v"], state["o"], state["lse"],
                                   state["causal"], state["scale"])
    rot = (state["cos"], state["sin"], state["positions"], state["interleaved"])
    if state["op"] == "rope":
        return (_norm_rope(state["q"], state["wq"], *rot), _norm_rope(state["k"], state["wk"], *rot))
    dq, dwq = _norm_rope_backward(state["dq"], state["q"], state["wq"], *rot)
    dk, dwk = _norm_rope_backward(state["dk"], state["k"], state["wk"], *rot)
    return dq, dk, dwq, dwk


def _run_own(state):
    import paper_2603_24517_b200 as lib

    if state["op"] == "bwd":
        return lib.attention_backward(state["do"], state["q"], state["k"], state["v"], state["o"], state["lse"],
                                      causal=state["causal"], scale=state["scale"])
    named = dict(positions=state["positions"], eps=EPS, interleaved=state["interleaved"])
    args = (state["q"], state["k"], state["wq"], state["wk"], state["cos"], state["sin"])
    if state["op"] == "rope":
        return lib.qk_norm_rope(*args, **named)
    return lib.qk_norm_rope_backward(state["dq"], state["dk"], *args, **named)


# ---- plain forms ---------------------------------------------------------------------------------------

def _grouped(x, hkv):
    """[B, S, Hq, D] -> fp32 [B, Hkv, Hq / Hkv, S, D]"""
    B, S, H, d = x.shape
    return x.float().view(B, S, hkv, H // hkv, d).permute(0, 2, 3, 1, 4)


def _ungrouped(x):
    """[B, Hkv, G, S, D] -> BF16 [B, S, Hkv * G, D]"""
    B, hkv, g, S, d = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(B, S, hkv * g, d).to(torch.bfloat16)


def _hidden(sq, sk, device):
    """True where a key is not visible under the causal mask (aligned to the last row and key)."""
    rows = torch.arange(sq, device=device)[:, None]
    return torch.arange(sk, device=device) > rows + (sk - sq)


def _attention(q, k, v, causal, scale):
    hkv = k.shape[2]
    s = _grouped(q, hkv) @ _grouped(k, hkv).transpose(-1, -2)
    s *= scale
    if causal:
        s.masked_fill_(_hidden(q.shape[1], k.shape[1], q.device), -math.inf)
    lse = torch.logsumexp(s, dim=-1)                       # -inf where a row sees no key
    s -= torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None]
    o = s.exp_() @ _grouped(v, hkv)
    return _ungrouped(o), lse.reshape(q.shape[0], q.shape[2], q.shape[1]).contiguous()


def _attention_backward(do, q, k, v, o, lse, causal, scale):
    B, Sq, Hq, _ = q.shape
    hkv, G = k.shape[2], Hq // k.shape[2]
    qf, kf, vf, dof = _grouped(q, hkv), _grouped(k, hkv), _grouped(v, hkv), _grouped(do, hkv)
    p = qf @ kf.transpose(-1, -2)
    p *= scale
    row_lse = lse.view(B, hkv, G, Sq)
    p -= torch.where(row_lse == -math.inf, torch.zeros_like(row_lse), row_lse)[..., None]
    if causal:
        p.masked_fill_(_hidden(Sq, k.shape[1], q.device), -math.inf)
    p.exp_()
    dv = (p.transpose(-1, -2) @ dof).sum(2, keepdim=True)  # heads that share a key head add up
    ds = dof @ vf.transpose(-1, -2)
    ds -= (dof * _grouped(o, hkv)).sum(-1, keepdim=True)
    ds *= p
    del p
    dq = (ds @ kf) * scale
    dk = (ds.transpose(-1, -2) @ qf).sum(2, keepdim=True) * scale
    return _ungrouped(dq), _ungrouped(dk), _ungrouped(dv)


def _angles(cos, sin, positions, seq):
    """Rows of the tables for each token, [B or 1, S, 1, R / 2]"""
    if positions is None:
        return cos[None, :seq, None], sin[None, :seq, None]
    return cos[positions][:, :, None], sin[positions][:, :, None]


def _rotate(x, cos, sin, interleaved):
    """Rotates the first R elements of each row: pairs (2i, 2i + 1), or (i, i + R / 2)."""
    half = cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _norm_rope(x, w, cos, sin, positions, interleaved):
    xf = x.float()
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    c, s = _angles(cos, sin, positions, x.shape[1])
    return _rotate(xf * r * w.float(), c, s, interleaved).to(torch.bfloat16)


def _norm_rope_backward(dy, x, w, cos, sin, positions, interleaved):
    xf = x.float()
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    c, s = _angles(cos, sin, positions, x.shape[1])
    dn = _rotate(dy.float(), c, -s, interleaved)           # the rotation's transpose turns back
    normed = xf * r
    dw = (dn * normed).sum((0, 1, 2))
    a = dn * w.float()
    dx = r * (a - normed * (a * normed).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), dw


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    if case["op"] == "bwd":
        B, Hq, Hkv, Sq, Sk = (case[n] for n in ("batch", "hq", "hkv", "sq", "sk"))
        pairs = Sq * Sk
        if case["causal"]:  # row i sees min(Sk, max(0, i + 1 + Sk - Sq)) keys
            n = min(Sq, Sk)
            pairs = n * (n + 1) // 2 + n * (Sk - n)
        rows = B * Sq * Hq
        # q, o, do read and dq written; k, v read and dk, dv written; lse read.  Five products of 2 D a pair.
        return {"bytes": rows * D * 2 * 4 + B * Sk * Hkv * D * 2 * 4 + rows * 4, "flops": 10 * B * Hq * pairs * D}
    B, S, Hq, Hkv, R = (case[n] for n in ("batch", "seq", "hq", "hkv", "rot"))
    values = B * S * (Hq + Hkv) * D
    angles = (min(B * S, case["table"]) if case["positions"] else S) * R * 4  # a row of both tables
    extra = B * S * 8 if case["positions"] else 0
    weights = 2 * D * (2 if case["weights"] == "bf16" else 4)
    if case["op"] == "rope":
        return {"bytes": values * 4 + angles + extra + weights, "flops": 7 * values}
    return {"bytes": values * 6 + angles + extra + weights + 2 * D * 4, "flops": 16 * values}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "bwd":
        if case["batch"] * case["hq"] * case["sq"] * case["sk"] > 1 << LOG2_MAX:
            return None
        B, Hq, Hkv, Sq, Sk = (case[n] for n in ("batch", "hq", "hkv", "sq", "sk"))
        out = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (st["q"], st["k"], st["v"])]
        step = max(1, (1 << 26) // Sk)  # rows of scores held at a time
        keys = torch.arange(Sk, device="cuda")
        for b in range(B):
            for h in range(Hq):
                g = h // (Hq // Hkv)
                K, V = st["k"][b, :, g].double(), st["v"][b, :, g].double()
                for i in range(0, Sq, step):
                    rows = slice(i, min(Sq, i + step))
                    Q, G, O = (st[n][b, rows, h].double() for n in ("q", "do", "o"))
                    prob = torch.exp(torch.einsum("id,jd->ij", Q, K) * st["scale"] - st["lse"][b, h, rows].double()[:, None])
                    if case["causal"]:
                        seen = keys[None] <= torch.arange(rows.start, rows.stop, device="cuda")[:, None] + (Sk - Sq)
                        prob = torch.where(seen, prob, torch.zeros((), dtype=torch.float64, device="cuda"))
                    out[2][b, :, g] += torch.einsum("ij,id->jd", prob, G)
                    inner = torch.einsum("id,jd->ij", G, V) - torch.einsum("id,id->i", G, O)[:, None]
                    grad = inner * prob * st["scale"]
                    out[0][b, rows, h] = torch.einsum("ij,jd->id", grad, K)
                    out[1][b, :, g] += torch.einsum("ij,id->jd", grad, Q)
        return tuple(out)
    where = st["positions"] if st["positions"] is not None else torch.arange(case["seq"], device="cuda")[None].expand(case["batch"], -1)
    cos, sin = st["cos"].double()[where], st["sin"].double()[where]  # [B, S, R / 2]
    turn = torch.complex(cos, sin)[:, :, None]
    R = case["rot"]

    def spin(t, by):  # each pair as one complex number
        head, tail = t[..., :R], t[..., R:]
        z = torch.complex(head[..., 0::2], head[..., 1::2]) if st["interleaved"] else torch.complex(head[..., :R // 2], head[..., R // 2:])
        z = z * by
        head = torch.stack((z.real, z.imag), -1 if st["interleaved"] else -2).flatten(-2)
        return torch.cat((head, tail), -1)

    results, weights = [], []
    for name in ("q", "k"):
        x, w = st[name].double(), st["w" + name].double()
        scale = ((x ** 2).sum(-1, keepdim=True) / D + EPS) ** -0.5
        if case["op"] == "rope":
            results.append(spin(x * scale * w, turn))
            continue
        g = spin(st["d" + name].double(), turn.conj())
        weights.append(torch.einsum("bshd,bshd->d", g, x * scale))
        gw = g * w
        results.append(scale * gw - scale ** 3 * x * ((gw * x).sum(-1, keepdim=True) / D))
    return tuple(results + weights)
