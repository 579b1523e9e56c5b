"""Operators around a cache that evicts by accumulated attention weight and holds its rows in 4 bits: what is measured.

A prompt's causal attention, the attention weight its tokens received, the eviction that fills a cache of fixed capacity,
the decode attention over the cache's 4-bit rows and the eviction step after it. `run` computes each in plain torch
operations, or with the library's calls where `own` is true.
"""
import math

import torch

own = False

GROUP = 64      # elements of a row that share a step and a low value
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a chat's first short turns at the smallest parity sizes: latency counts
        dict(name="prompt short", op="prompt_attention", dtype="bf16", heads=8, kv_heads=8, dim=64, lens="1,17,40", pad=0, fused=False),
        # a serving batch of ragged conversations, grouped heads, q/k/v cut out of one projection, unused rows at the end
        dict(name="prompt ragged grouped", op="prompt_attention", dtype="bf16", heads=32, kv_heads=8, dim=128,
             lens="2048,1,513,0,8192,77,3840,300,128", pad=37, fused=True),
        # the float32 correctness shape: 8 heads of 64
        dict(name="prompt float32", op="prompt_attention", dtype="f32", heads=8, kv_heads=8, dim=64, lens="64,1,333,512,1024", pad=3, fused=False),
        # weights that the tokens of 16 prompts of 512 received from all queries (32 heads of 128, as in the decode workloads)
        dict(name="weights of 16 prompts", op="prompt_weights", dtype="bf16", heads=32, kv_heads=32, dim=128,
             lens=",".join(["512"] * 16), pad=0, fused=False, window=0),
        # an observation window of the last 32 queries, float32
        dict(name="weights window float32", op="prompt_weights", dtype="f32", heads=8, kv_heads=4, dim=64, lens="256,31,1000,1", pad=0,
             fused=True, window=32),
        # 16 prompts of 512 cut to a cache of 256 slots, 32 heads
        dict(name="evict 16 prompts", op="evict_prompt", dtype="bf16", heads=32, kv_heads=32, dim=128, lens=",".join(["512"] * 16), pad=0,
             fused=False, capacity=256, recent=64),
        # long ragged prompts, few key/value heads, one sequence shorter than the cache
        dict(name="evict long prompts", op="evict_prompt", dtype="bf16", heads=32, kv_heads=8, dim=128, lens="3840,9,2048,20001", pad=5,
             fused=True, capacity=1024, recent=128),
        # one float32 sequence with 64 slots: latency of a decode step's bookkeeping
        dict(name="evict step small", op="evict_step", dtype="f32", heads=8, kv_heads=8, dim=64, batch=1, capacity=64, fill=1.0, recent=8),
        # a batch of 32 with 1024 slots and 32 heads
        dict(name="evict step batch", op="evict_step", dtype="bf16", heads=32, kv_heads=32, dim=128, batch=32, capacity=1024, fill=0.97,
             recent=128),
        # one float32 sequence with 64 slots
        dict(name="decode small float32", op="q4_attention", dtype="f32", heads=8, kv_heads=8, dim=64, batch=1, capacity=64, fill=0.8,
             weights=True),
        # a batch of 32, 32 heads, 1024 slots, weights wanted for the eviction
        dict(name="decode batch", op="q4_attention", dtype="bf16", heads=32, kv_heads=32, dim=128, batch=32, capacity=1024, fill=1.0,
             weights=True),
        # few sequences with long caches and grouped heads, an odd capacity, no weights wanted
        dict(name="decode long grouped", op="q4_attention", dtype="bf16", heads=32, kv_heads=8, dim=128, batch=3, capacity=40001, fill=0.95,
             weights=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["prompt_attention", "prompt_weights", "evict_prompt", "evict_step", "q4_attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    case = dict(op=op, dtype=dtype, heads=min(32 // kv, group) * kv, kv_heads=kv, dim=rng.choice([64, 128]))
    if op in ("prompt_attention", "prompt_weights", "evict_prompt"):
        longest = 1500 if dtype == "f32" else 6000
        lens = [_log_int(rng, 1, longest) for _ in range(rng.randint(1, 9))]
        while len(lens) > 1 and sum(n * n for n in lens) > (4_000_000 if dtype == "f32" else 60_000_000):
            lens.remove(max(lens))
        if rng.random() < 0.3:
            lens.insert(rng.randrange(len(lens) + 1), 0)
        case.update(lens=",".join(map(str, lens)), pad=rng.choice([0, 0, 1, 50]), fused=rng.random() < 0.5)
    if op == "prompt_weights":
        case["window"] = rng.choice([0, 0, 1, 32, 200])
    if op == "evict_prompt":
        case["capacity"] = _log_int(rng, 16, 2000)
        case["recent"] = rng.randint(1, case["capacity"])
    if op in ("evict_step", "q4_attention"):
        case["batch"] = _log_int(rng, 1, 32)
        case["capacity"] = _log_int(rng, 1, max(1, 1_000_000 // (case["batch"] * kv)))
        case["fill"] = rng.choice([0.0, 0.5, 0.9, 1.0])
    if op == "evict_step":
        case["recent"] = rng.randint(1, case["capacity"])
    if op == "q4_attention":
        case["weights"] = rng.random() < 0.5
    return case


# ---- the 4-bit rows -----------------------------------------------------------------------------
def _padded(capacity):
    return (capacity + 15) // 16 * 16


def _sections(batch, kv_heads, dim, capacity):
    """Byte sizes of the cache's parts: key codes, value codes, key (step, low) pairs, value pairs."""
    rows = batch * kv_heads * _padded(capacity)
    return [rows * dim // 2, rows * dim // 2, rows * (dim // GROUP) * 4, rows * (dim // GROUP) * 4]


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)


def _unpack(cache, batch, kv_heads, dim, capacity):
    """K and V in 32 bits, [batch, kv_heads, capacity, dim], from the cache's bytes."""
    sizes, cp, r = _sections(batch, kv_heads, dim, capacity), _padded(capacity), batch * kv_heads
    kc, vc, kp, vp = torch.split(cache[: sum(sizes)], sizes)
    # a key row: 4 x (dim/32) words of 8 codes, word (t, i) holds elements 32 i + 8 t ..
    k = _nibbles(kc).view(r, cp, 4, dim // 32, 8).permute(0, 1, 3, 2, 4).reshape(r, cp, dim)
    # two neighbouring value rows: 8 x (dim/32) words, word (t, i) holds elements 32 i + 4 t .. of the first, then of the second
    v = _nibbles(vc).view(r, cp // 2, 8, dim // 32, 2, 4).permute(0, 1, 4, 3, 2, 5).reshape(r, cp, dim)
    out = []
    for codes, par in ((k, kp), (v, vp)):
        par = par.view(torch.bfloat16).view(r, cp, dim // GROUP, 2).float()
        x = codes.view(r, cp, dim // GROUP, GROUP).float() * par[..., :1] + par[..., 1:]
        out.append(x.view(batch, kv_heads, cp, dim)[:, :, :capacity])
    return out


def _in_four_bits(x):
    """The values that rows x [..., dim] stand for in 4 bits."""
    g = x.unflatten(-1, (-1, GROUP))
    low = g.amin(-1, keepdim=True).to(torch.bfloat16).to(x.dtype)
    step = ((g.amax(-1, keepdim=True) - low).clamp(min=0) / 15).to(torch.bfloat16).to(x.dtype)
    code = torch.where(step > 0, ((g - low) / torch.where(step > 0, step, 1)).round().clamp(0, 15), 0)
    return (code * step + low).flatten(-2)


# ---- inputs -------------------------------------------------------------------------------------
def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dt, h, hk, d = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case=case)
    if "lens" in case:
        lens = _lens(case)
        used, total = sum(lens), sum(lens) + case["pad"]
        s["lens"] = lens
        s["seq_start"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        # queries twice as long as keys: softmax rows with a few large weights and a long tail
        if case["fused"]:
            rows = normal(total, h + 2 * hk, d)
            rows[:, :h] *= 2.0
            rows[used:] = float("nan")
            rows = rows.to(dt)
            s["q"], s["k"], s["v"] = rows[:, :h], rows[:, h:h + hk], rows[:, h + hk:]
        else:
            s["q"], s["k"], s["v"] = (x.to(dt) for x in (normal(total, h, d) * 2.0, normal(total, hk, d), normal(total, hk, d)))
        if case["op"] == "prompt_attention":
            s["out"], s["lse"] = torch.zeros(total, h, d, dtype=dt, device="cuda"), torch.zeros(h, total, device="cuda")
        elif case["op"] == "prompt_weights":
            s["lse"] = torch.zeros(h, total, device="cuda")
            s["acc"] = torch.zeros(hk, total, device="cuda")
            _plain_attention(s, lse_only=True, into=s["lse"])
        else:
            # weights received: heavy-tailed, some tokens with exactly nothing
            s["acc"] = torch.exp(2 * normal(hk, total)) * (torch.rand(hk, total, generator=g, device="cuda") > 0.05)
            s["slot_pos"] = torch.zeros(len(lens), hk, case["capacity"], dtype=torch.int32, device="cuda")
            s["slot_acc"] = torch.zeros(len(lens), hk, case["capacity"], device="cuda")
            s["length"] = torch.zeros(len(lens), hk, dtype=torch.int32, device="cuda")
            s["cache"] = torch.zeros(sum(_sections(len(lens), hk, d, case["capacity"])), dtype=torch.uint8, device="cuda")
            s["k_rows"], s["v_rows"] = (torch.zeros(len(lens), hk, case["capacity"], d, dtype=dt, device="cuda") for _ in range(2))
        return s
    b, c = case["batch"], case["capacity"]
    codes, _, pairs, _ = _sections(b, hk, d, c)
    # rows of normally distributed keys and values: a low value near -2.4, a step near 0.3
    par = torch.rand(2 * pairs // 4, 2, generator=g, device="cuda")
    par[:, 0] = 0.25 + 0.13 * par[:, 0]
    par[:, 1] = -2.0 - 0.9 * par[:, 1]
    s["cache"] = torch.cat([torch.randint(0, 256, (2 * codes,), generator=g, device="cuda", dtype=torch.uint8),
                            par.to(torch.bfloat16).view(torch.uint8).flatten()])
    # every sequence has decoded 4 C tokens or so; a share of the slots is taken, each by a token of its own
    n = torch.randint(4 * c + 8, 5 * c + 9, (b,), generator=g, device="cuda")
    pos = torch.rand(b, hk, 4 * c + 8, generator=g, device="cuda").argsort(-1)[..., :c] + (n.view(b, 1, 1) - (4 * c + 8))
    s["slot_pos"] = torch.where(torch.rand(b, hk, c, generator=g, device="cuda") < case["fill"], pos, -1).to(torch.int32)
    s["q"], s["k_new"], s["v_new"] = ((normal(b, m, d) * f).to(dt) for m, f in ((h, 2.0), (hk, 1.0), (hk, 1.0)))
    if case["op"] == "evict_step":
        s["length"] = n.to(torch.int32).unsqueeze(1).repeat(1, hk)
        s["slot_acc"] = torch.exp(2 * normal(b, hk, c)) * (s["slot_pos"] >= 0)
        taken = torch.cat([(s["slot_pos"] >= 0).repeat_interleave(h // hk, 1), torch.ones(b, h, 1, dtype=torch.bool, device="cuda")], -1)
        s["weights"] = torch.softmax(torch.where(taken, 2 * normal(b, h, c + 1), float("-inf")), -1)
        s["admit_slot"], s["evicted_pos"] = (torch.zeros(b, hk, dtype=torch.int32, device="cuda") for _ in range(2))
        s["k_row"], s["v_row"] = (torch.zeros(b, hk, 1, d, dtype=dt, device="cuda") for _ in range(2))
    else:
        s["out"] = torch.zeros(b, h, d, dtype=dt, device="cuda")
        s["weights"] = torch.zeros(b, h, c + 1, device="cuda") if case["weights"] else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------
def _plain_attention(s, lse_only=False, into=None):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    out = None if lse_only else torch.zeros_like(s["out"])
    lse = torch.zeros(h, s["q"].shape[0], device="cuda") if into is None else into
    at = 0
    for n in s["lens"]:
        if n:
            q = s["q"][at:at + n].float().view(n, hk, h // hk, d).permute(1, 2, 0, 3)
            k, v = (s[x][at:at + n].float().permute(1, 0, 2).unsqueeze(1) for x in ("k", "v"))
            logits = (q @ k.transpose(-1, -2)).mul_(d ** -0.5)
            logits.masked_fill_(torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1), float("-inf"))
            top = logits.amax(-1, keepdim=True)
            p = logits.sub_(top).exp_()
            norm = p.sum(-1, keepdim=True)
            lse[:, at:at + n] = (top + norm.log()).view(h, n)
            if not lse_only:
                out[at:at + n] = ((p @ v) / norm).permute(2, 0, 1, 3).reshape(n, h, d)
        at += n
    return out, lse


def _plain_weights(s):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    acc, at = torch.zeros_like(s["acc"]), 0
    for n in s["lens"]:
        if n:
            w = min(c["window"] or n, n)
            q = s["q"][at + n - w:at + n].float().view(w, hk, h // hk, d).permute(1, 2, 0, 3)
            k = s["k"][at:at + n].float().permute(1, 0, 2).unsqueeze(1)
            p = (q @ k.transpose(-1, -2)).mul_(d ** -0.5).sub_(s["lse"][:, at + n - w:at + n].view(hk, h // hk, w, 1)).exp_()
            p.masked_fill_(torch.ones(w, n, dtype=torch.bool, device="cuda").triu_(1 + n - w), 0)
            acc[:, at:at + n] = p.sum((1, 2))
        at += n
    return acc


def _plain_evict_prompt(s):
    c = s["case"]
    hk, d, cap, recent = c["kv_heads"], c["dim"], c["capacity"], c["recent"]
    b, dt = len(s["lens"]), s["k"].dtype
    pos = torch.full((b, hk, cap), -1, dtype=torch.int32, device="cuda")
    acc = torch.zeros(b, hk, cap, device="cuda")
    k_rows, v_rows = torch.zeros_like(s["k_rows"]), torch.zeros_like(s["v_rows"])
    at = 0
    for i, n in enumerate(s["lens"]):
        if n:
            a = s["acc"][:, at:at + n]
            a = torch.where(torch.arange(n, device="cuda") >= n - recent, float("inf"), a)
            m = min(n, cap)
            kept = a.sort(dim=-1, descending=True, stable=True)[1][:, :m].sort(-1)[0]
            pos[i, :, :m] = kept.to(torch.int32)
            acc[i, :, :m] = s["acc"][:, at:at + n].gather(1, kept)
            for x, to in (("k", k_rows), ("v", v_rows)):
                rows = s[x][at:at + n].permute(1, 0, 2).gather(1, kept.unsqueeze(-1).expand(hk, m, d)).float()
                to[i, :, :m] = _in_four_bits(rows).to(dt)
        at += n
    length = (s["seq_start"][1:] - s["seq_start"][:-1]).unsqueeze(1).repeat(1, hk)
    return dict(slot_pos=pos, slot_acc=acc, length=length, k=k_rows, v=v_rows)


def _plain_evict_step(s):
    c = s["case"]
    b, h, hk, cap = c["batch"], c["heads"], c["kv_heads"], c["capacity"]
    pos, slots = s["slot_pos"], torch.arange(cap, device="cuda")
    got = s["weights"].view(b, hk, h // hk, cap + 1).double().sum(2)
    acc = torch.where(pos >= 0, (s["slot_acc"].double() + got[..., :cap]).float(), 0.0)
    free = pos < 0
    old = (pos <= s["length"].unsqueeze(-1) - c["recent"]) & ~free
    value = torch.where(free, -1.0, torch.where(old, acc, float("inf")))
    admit = torch.where(value == value.amin(-1, keepdim=True), slots, cap).amin(-1)
    here = slots == admit.unsqueeze(-1)
    evicted = torch.where(here, pos, 0).sum(-1).to(torch.int32)
    s["slot_acc"].copy_(torch.where(here, got[..., cap:].float(), acc))
    s["slot_pos"].copy_(torch.where(here, s["length"].unsqueeze(-1), pos))
    s["length"] += 1
    rows = [_in_four_bits(s[x].float()).to(s[x].dtype).unsqueeze(2) for x in ("k_new", "v_new")]
    return dict(slot_pos=s["slot_pos"], slot_acc=s["slot_acc"], length=s["length"], admit_slot=admit.to(torch.int32), evicted_pos=evicted,
                k=rows[0], v=rows[1])


def _decode_attention(s, kind):
    c = s["case"]
    b, h, hk, d, cap = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["capacity"]
    k, v = (torch.cat([x.to(kind), s[y].to(kind).unsqueeze(2)], 2) for x, y in zip(_unpack(s["cache"], b, hk, d, cap), ("k_new", "v_new")))
    taken = torch.cat([s["slot_pos"] >= 0, torch.ones(b, hk, 1, dtype=torch.bool, device="cuda")], -1).unsqueeze(2)
    logits = s["q"].to(kind).view(b, hk, h // hk, d) @ k.transpose(-1, -2) * d ** -0.5
    logits = torch.where(taken, logits, float("-inf"))
    p = (logits - logits.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    return (p @ v).view(b, h, d), p.view(b, h, cap + 1)


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        from paper_2407_02328_b200 import adore
        if op == "prompt_attention":
            adore.adore_prompt_attention(s["q"], s["k"], s["v"], s["seq_start"], s["out"], s["lse"])
            return dict(out=s["out"], lse=s["lse"])
        if op == "prompt_weights":
            adore.adore_prompt_weights(s["q"], s["k"], s["lse"], s["seq_start"], s["acc"], window=s["case"]["window"])
            return dict(acc=s["acc"])
        if op == "evict_prompt":
            adore.adore_evict_prompt(s["acc"], s["k"], s["v"], s["seq_start"], s["case"]["recent"], s["cache"], s["slot_pos"], s["slot_acc"],
                                     s["length"])
            adore.adore_q4_read(s["cache"], s["case"]["capacity"], None, s["k_rows"], s["v_rows"])
            return dict(slot_pos=s["slot_pos"], slot_acc=s["slot_acc"], length=s["length"], k=s["k_rows"], v=s["v_rows"])
        if op == "evict_step":
            adore.adore_evict_step(s["weights"], s["k_new"], s["v_new"], s["case"]["recent"], s["cache"], s["slot_pos"],
                                   s["slot_acc"], s["length"], s["admit_slot"], s["evicted_pos"])
            adore.adore_q4_read(s["cache"], s["case"]["capacity"], s["admit_slot"], s["k_row"], s["v_row"])
            return dict(slot_pos=s["slot_pos"], slot_acc=s["slot_acc"], length=s["length"], admit_slot=s["admit_slot"],
                        evicted_pos=s["evicted_pos"], k=s["k_row"], v=s["v_row"])
        adore.adore_q4_attention(s["q"], s["k_new"], s["v_new"], s["cache"], s["slot_pos"], s["out"], s["weights"])
        return dict(out=s["out"]) if s["weights"] is None else dict(out=s["out"], weights=s["weights"])
    if op == "prompt_attention":
        out, lse = _plain_attention(s)
        return dict(out=out, lse=lse)
    if op == "prompt_weights":
        return dict(acc=_plain_weights(s))
    if op == "evict_prompt":
        return _plain_evict_prompt(s)
    if op == "evict_step":
        return _plain_evict_step(s)
    out, p = _decode_attention(s, torch.float32)
    return dict(out=out.to(s["q"].dtype)) if s["weights"] is None else dict(out=out.to(s["q"].dtype), weights=p)


def work(case):
    e, h, hk, d = 4 if case["dtype"] == "f32" else 2, case["heads"], case["kv_heads"], case["dim"]
    row = 2 * (d // 2 + d // GROUP * 4)                       # a key and a value row in 4 bits
    if case["op"] in ("prompt_attention", "prompt_weights"):
        lens = _lens(case)
        n = sum(lens)
        if case["op"] == "prompt_attention":
            return dict(bytes=n * d * e * (2 * h + 2 * hk) + n * h * 4, flops=4 * d * h * sum(x * (x + 1) // 2 for x in lens))
        w = [min(case["window"] or x, x) for x in lens]
        seen = sum(y * (x - y) + y * (y + 1) // 2 for x, y in zip(lens, w))
        return dict(bytes=sum(w) * h * (d * e + 4) + n * hk * (d * e + 4), flops=2 * d * h * seen)
    if case["op"] == "evict_prompt":
        lens = _lens(case)
        kept, slots = sum(min(x, case["capacity"]) for x in lens), len(lens) * case["capacity"]
        # weights read, kept rows read, the cache with its maps written, its values read back
        return dict(bytes=hk * (4 * sum(lens) + kept * 2 * d * e + slots * (8 + 2 * row + 2 * d * e)), flops=hk * kept * 2 * d * 6)
    b, c = case["batch"], case["capacity"]
    if case["op"] == "evict_step":
        return dict(bytes=b * (h * (c + 1) * 4 + hk * (c * 12 + 4 * d * e + 3 * row + 16)), flops=b * h * c)
    taken = max(1.0, b * hk * c * case["fill"])
    return dict(bytes=taken * row + b * hk * c * 4 + b * d * e * (2 * h + 2 * hk) + (b * h * (c + 1) * 4 if case["weights"] else 0),
                flops=4 * d * (h // hk) * taken)


# ---- from the definitions, in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    h, hk, d, op = case["heads"], case["kv_heads"], case["dim"], case["op"]
    if op in ("prompt_attention", "prompt_weights"):
        total, at = s["q"].shape[0], 0
        out = torch.zeros(total, h, d, dtype=torch.float64, device="cuda")
        lse = torch.zeros(h, total, dtype=torch.float64, device="cuda")
        acc = torch.zeros(hk, total, dtype=torch.float64, device="cuda")
        for n in s["lens"]:
            mine, i = slice(at, at + n), torch.arange(n, device="cuda")
            for head in range(h if n else 0):
                q, k, v = s["q"][mine, head].double(), s["k"][mine, head // (h // hk)].double(), s["v"][mine, head // (h // hk)].double()
                x = torch.where(i[None, :] <= i[:, None], q @ k.T / math.sqrt(d), float("-inf"))
                if op == "prompt_attention":
                    lse[head, mine] = torch.logsumexp(x, -1)
                    out[mine, head] = torch.exp(x - lse[head, mine, None]) @ v
                else:
                    w = torch.exp(x - s["lse"][head, mine, None].double())
                    acc[head // (h // hk), mine] += w[max(0, n - (case["window"] or n)):].sum(0)
            at += n
        return dict(out=out, lse=lse) if op == "prompt_attention" else dict(acc=acc)
    if op == "evict_prompt":
        b, cap = len(s["lens"]), case["capacity"]
        acc = torch.zeros(b, hk, cap, dtype=torch.float64, device="cuda")
        k, v = (torch.zeros(b, hk, cap, d, dtype=torch.float64, device="cuda") for _ in range(2))
        at = 0
        for i, n in enumerate(s["lens"]):
            for head in range(hk if n else 0):
                a = s["acc"][head, at:at + n].tolist()
                older = sorted(range(max(0, n - case["recent"])), key=lambda t: (-a[t], t))[: cap - min(n, case["recent"])]
                kept = sorted(older + list(range(max(0, n - case["recent"]), n)))
                idx = torch.tensor(kept, device="cuda") + at
                acc[i, head, : len(kept)] = s["acc"][head, idx].double()
                for x, to in (("k", k), ("v", v)):
                    to[i, head, : len(kept)] = _in_four_bits(s[x][idx, head].double())
            at += n
        return dict(slot_pos=None, slot_acc=acc, length=None, k=k, v=v)
    if op == "evict_step":
        acc = s["slot_acc"].double()
        got = s["weights"].double().unflatten(1, (hk, h // hk)).sum(2)
        for b in range(case["batch"]):
            n = int(s["length"][b, 0])
            for head in range(hk):
                pos = s["slot_pos"][b, head].tolist()
                a = torch.where(s["slot_pos"][b, head] >= 0, acc[b, head] + got[b, head, :-1], 0.0)
                acc[b, head] = a
                a = a.tolist()
                free = [i for i, p in enumerate(pos) if p < 0]
                at = free[0] if free else min((i for i, p in enumerate(pos) if p <= n - case["recent"]), key=lambda i: (a[i], i))
                acc[b, head, at] = got[b, head, -1]
        rows = [_in_four_bits(s[x].double()).unsqueeze(2) for x in ("k_new", "v_new")]
        return dict(slot_pos=None, slot_acc=acc, length=None, admit_slot=None, evicted_pos=None, k=rows[0], v=rows[1])
    out, p = _decode_attention(s, torch.float64)
    return dict(out=out) if s["weights"] is None else dict(out=out, weights=p)
