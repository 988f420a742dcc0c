"""64-bit definitions of the paged 8-bit cache and of attention over it, one sequence and head at a time; test infrastructure only."""
import torch


def e4m3_round(x):
    """float64 -> the nearest E4M3 number, ties to even, saturating (NaN stays)."""
    mag = x.abs().clamp(max=448.0)
    unit = torch.exp2(torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(mag / unit) * unit, x)


def scale_for(largest: float, int8: bool) -> float:
    """The scale of a page and head with this largest magnitude, as the FP32 number the cache holds."""
    if largest == 0.0:
        return 0.0
    if int8:
        s = float(torch.tensor(largest, dtype=torch.float32) * (torch.tensor(1.0, dtype=torch.float32) / torch.tensor(127.0, dtype=torch.float32)))
        return max(s, 2.0 ** -100)
    s = 2.0 ** -100
    while largest > 448.0 * s:
        s *= 2.0
    return s


def encode(x, scale: float, int8: bool):
    """Codes (as float64 numbers) of float64 values x."""
    s = scale if scale > 0 else 1.0
    if int8:  # the quotient of two FP32 numbers, rounded to FP32 and then to the nearest integer
        y = (x.to(torch.float32) / torch.tensor(s, dtype=torch.float32)).double()
        return torch.where(y.isnan(), torch.zeros_like(y), torch.round(y).clamp(-127, 127))
    return e4m3_round(x / s)


def append(codes, scales, k_rows, page_ids, begin, page, int8):
    """codes float64 [pages, page, H, D] and scales float64 [pages, H] are updated with k_rows [n, H, D] at positions begin..."""
    n, H = k_rows.shape[:2]
    x = k_rows.double()
    for first in range(begin - begin % page, begin + n, page):
        pid = page_ids[first // page]
        lo, hi = max(first, begin), min(first + page, begin + n)
        rows = x[lo - begin:hi - begin]
        for h in range(H):
            mags = rows[:, h].abs()
            mags = mags[mags.isfinite()]
            s = scale_for(float(mags.max()) if mags.numel() else 0.0, int8)
            held = lo - first
            if held:
                before = float(scales[pid, h])
                s = max(s, before)
                if s > before:
                    old = (codes[pid, :held, h].to(torch.float32) * torch.tensor(before, dtype=torch.float32)).double()
                    codes[pid, :held, h] = encode(old, s, int8)
            codes[pid, held:held + hi - lo, h] = encode(rows[:, h], s, int8)
            scales[pid, h] = s


def gather(codes, scales, page_ids, n_tokens, page):
    """float64 [n_tokens, H, D] of one sequence."""
    at = torch.arange(n_tokens, device=codes.device)
    pid = torch.as_tensor(page_ids, device=codes.device)[at // page]
    return codes[pid, at % page].double() * scales[pid].double()[:, :, None]


def attend(q, k, v, first_position, causal, scale):
    """q [n, Hq, D] at positions first_position.., k, v float64 [L, H, D] -> o float64 [n, Hq, D], lse [Hq, n], and for error
    bounds: sum_j p_j |v_j| like o, the largest scale * sum_d |q_d k_jd| over visible keys like lse."""
    n, Hq, D = q.shape
    L, H = k.shape[:2]
    o, spread = torch.zeros(2, n, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((Hq, n), -float("inf"), dtype=torch.float64, device=q.device)
    size = torch.zeros(Hq, n, dtype=torch.float64, device=q.device)
    pos = first_position + torch.arange(n, device=q.device)
    seen = torch.arange(L, device=q.device)[None] <= pos[:, None] if causal else torch.ones(n, L, dtype=torch.bool, device=q.device)
    some = seen.any(1) if L else torch.zeros(n, dtype=torch.bool, device=q.device)
    if not bool(some.any()):
        return o, lse, spread, size
    for hq in range(Hq):
        kk, vv, qq = k[:, hq // (Hq // H)], v[:, hq // (Hq // H)], q[:, hq].double()
        s = (qq @ kk.T * scale).masked_fill(~seen, -float("inf"))
        top = torch.where(some, s.max(1).values, torch.zeros_like(s[:, 0]))
        w = torch.exp(s - top[:, None])
        total = w.sum(1)
        lse[hq] = top + torch.log(total)
        p = w / total.clamp(min=1e-300)[:, None]
        o[:, hq], spread[:, hq] = p @ vv, p @ vv.abs()
        size[hq] = (qq.abs() @ kk.abs().T * scale).masked_fill(~seen, 0).max(1).values
    return o, lse, spread, size
