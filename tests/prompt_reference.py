"""The prompt, eviction and 4-bit calls restated in float64 (and, where bits count, in float32 exactly as documented), on
whatever device the inputs are. Test infrastructure; shares no code with the library."""
import math

import torch

EPS32 = 2.0 ** -24                                    # half a step of float32, relative
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: EPS32}


def spans(seq_start):
    s = seq_start.tolist()
    return list(zip(s[:-1], s[1:]))


def attention(q, k, v, seq_start, scale=0.0):
    """out [total, H, dh], lse [H, total], and the parts that tolerances are made of: sum_j p_ij |v_j| (like out) and a bound
    of the float32 rounding of any logit of a row (like lse). Rows outside every sequence stay zero."""
    total, h, dh = q.shape
    group, scale = h // k.shape[1], scale or 1.0 / math.sqrt(dh)
    out = torch.zeros(total, h, dh, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    lse = torch.zeros(h, total, dtype=torch.float64, device=q.device)
    delta = torch.zeros_like(lse)
    for a, b in spans(seq_start):
        i = torch.arange(b - a, device=q.device)
        for head in range(h if b > a else 0):
            x, y, z = q[a:b, head].double(), k[a:b, head // group].double(), v[a:b, head // group].double()
            s = torch.where(i[None] <= i[:, None], x @ y.T * scale, float("-inf"))
            lse[head, a:b] = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[head, a:b, None])
            out[a:b, head], mag[a:b, head] = p @ z, p @ z.abs()
            # dh products summed in any order, the factor, the maximum's subtraction: dh + 4 roundings of the summands' size
            delta[head, a:b] = torch.where(i[None] <= i[:, None], x.abs() @ y.abs().T * abs(scale), 0.0).amax(-1) * (dh + 4) * EPS32
    return out, lse, mag, delta


def received(q, k, lse, seq_start, window=0, scale=0.0):
    """acc [Hk, total] and the bound of its float32 error: every weight's logit error, the exponential and the sum."""
    total, h, dh = q.shape
    hk = k.shape[1]
    group, scale = h // hk, scale or 1.0 / math.sqrt(dh)
    acc = torch.zeros(hk, total, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(acc)
    for a, b in spans(seq_start):
        n = b - a
        i = torch.arange(n, device=q.device)
        first = max(0, n - window) if window else 0
        seen = (i[None] <= i[:, None]) & (i[:, None] >= first)
        for head in range(h if n else 0):
            x, y = q[a:b, head].double(), k[a:b, head // group].double()
            s = x @ y.T * scale
            w = torch.where(seen, torch.exp(s - lse[head, a:b, None].double()), 0.0)
            # logit and its factor, lse and the conversion to powers of 2 (3 roundings of |s| + |lse|), 2 units of the exponential
            d = (x.abs() @ y.abs().T * abs(scale) * (dh + 4) + 3 * (s.abs() + lse[head, a:b, None].double().abs()) + 8) * EPS32
            acc[head // group, a:b] += w.sum(0)
            # rounding of the sums: partial sums of 64 or 128 queries, then their sum
            tol[head // group, a:b] += (w * (torch.expm1(d) + (128 + n / 64 + group) * EPS32)).sum(0)
    return acc, tol


def in_four_bits(rows):
    """The values rows [..., dh] stand for, in float32 arithmetic as adore.h has it; also step and code * step."""
    x = rows.float().unflatten(-1, (-1, 64))
    low = x.amin(-1, keepdim=True).bfloat16().float()
    step = ((x.amax(-1, keepdim=True) - low).clamp(min=0) / 15).bfloat16().float()
    code = torch.where(step > 0, ((x - low) / torch.where(step > 0, step, torch.ones_like(step))).round().clamp(0, 15), torch.zeros_like(x))
    return (code * step + low).flatten(-2), step, (code * step).flatten(-2)


def keep(acc, recent, capacity):
    """Kept positions of one sequence's head, ascending; acc a list of floats."""
    n = len(acc)
    if n <= capacity:
        return list(range(n))
    value = [(-math.inf, 0) if math.isnan(a) else (a, 1) for a in acc]            # NaN below -inf
    older = sorted(range(n - recent), key=lambda t: (-value[t][0], -value[t][1], t))[: capacity - recent]
    return sorted(older + list(range(n - recent, n)))


def step(weights, slot_pos, slot_acc, length, recent):
    """One eviction step on CPU tensors, in place; returns admitted slots and evicted positions."""
    b, hk, c = slot_pos.shape
    group = weights.shape[1] // hk
    admit, evicted = torch.full((b, hk), -1, dtype=torch.int32), torch.full((b, hk), -1, dtype=torch.int32)
    got = weights.double().unflatten(1, (hk, group)).sum(2)
    for i in range(b):
        for g in range(hk):
            n = int(length[i, g])
            if n < 0:
                continue
            taken = slot_pos[i, g] >= 0
            slot_acc[i, g][taken] = (slot_acc[i, g].double() + got[i, g, :c]).float()[taken]
            pos, val = slot_pos[i, g].tolist(), slot_acc[i, g].tolist()
            free = [s for s in range(c) if pos[s] < 0]
            old = sorted((s for s in range(c) if 0 <= pos[s] <= n - recent),
                         key=lambda s: ((0, 0.0) if math.isnan(val[s]) else (1, val[s]), s))
            length[i, g] = n + 1
            if not free and not old:
                continue
            s = free[0] if free else old[0]
            admit[i, g], evicted[i, g] = s, -1 if free else pos[s]
            slot_pos[i, g, s], slot_acc[i, g, s] = n, got[i, g, c].float()
    return admit, evicted


def decode(q, k_rows, v_rows, k_new, v_new, slot_pos, scale=0.0):
    """out [B, H, dh], weights [B, H, C + 1], sum p |v| (like out) and the logits' rounding bound per head (like weights[..., 0]),
    from float64 attention over the occupied slots' rows [B, Hk, C, dh] and the token's own."""
    b, h, dh = q.shape
    hk, c = slot_pos.shape[1:]
    scale = scale or 1.0 / math.sqrt(dh)
    taken = slot_pos >= 0
    k = torch.where(taken[..., None], k_rows.double(), 0.0)
    v = torch.where(taken[..., None], v_rows.double(), 0.0)
    own = torch.full((b, hk, 1), k_new is not None, device=q.device)
    zero = torch.zeros(b, hk, 1, dh, dtype=torch.float64, device=q.device)
    k = torch.cat([k, zero if k_new is None else k_new.double().unsqueeze(2)], 2)
    v = torch.cat([v, zero if v_new is None else v_new.double().unsqueeze(2)], 2)
    taken = torch.cat([taken, own], 2).unsqueeze(2)
    x = q.double().view(b, hk, h // hk, dh)
    s = torch.where(taken, x @ k.transpose(-1, -2) * scale, float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.where(taken, torch.exp(s - torch.where(top.isinf(), 0.0, top)), 0.0)
    norm = p.sum(-1, keepdim=True)
    p = torch.where(norm > 0, p / norm, 0.0)
    delta = (x.abs() @ k.abs().transpose(-1, -2) * abs(scale)).amax(-1) * (dh + 8) * EPS32
    return (p @ v).view(b, h, dh), p.view(b, h, c + 1), (p @ v.abs()).view(b, h, dh), delta.view(b, h)
