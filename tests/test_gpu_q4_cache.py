"""Eviction by attention weight and the 4-bit cache: the CUDA kernels against float64 and, for rows and choices, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu


def _dt(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _random_cache(b, hk, c, dh, dtype, seed, fill):
    """A cache whose rows were written by the library from random rows, random occupancy, garbage in the empty slots."""
    import torch
    from paper_2407_02328_b200 import adore as lib
    g = torch.Generator("cuda").manual_seed(seed)
    rows = [torch.randn(b * c, hk, dh, generator=g, device="cuda").to(_dt(dtype)) for _ in range(2)]
    start = (torch.arange(b + 1, device="cuda") * c).to(torch.int32)
    cache = torch.randint(0, 256, (lib.adore_q4_bytes(b, hk, dh, c),), generator=g, device="cuda", dtype=torch.uint8)
    pos = torch.zeros(b, hk, c, dtype=torch.int32, device="cuda")
    acc = torch.zeros(b, hk, c, device="cuda")
    length = torch.zeros(b, hk, dtype=torch.int32, device="cuda")
    lib.adore_evict_prompt(torch.zeros(hk, b * c, device="cuda"), *rows, start, c, cache, pos, acc, length)
    k, v = (torch.zeros(b, hk, c, dh, dtype=torch.float32, device="cuda") for _ in range(2))
    lib.adore_q4_read(cache, c, None, k, v)
    taken = torch.rand(b, hk, c, generator=g, device="cuda") < fill
    pos = torch.where(taken, pos, -1 - pos).to(torch.int32).contiguous()
    # empty slots: their pairs become NaN and infinities
    p = (c + 15) // 16 * 16
    codes, pairs = b * hk * p * dh // 2, b * hk * p * (dh // 64) * 4
    tail = cache[2 * codes:].view(torch.bfloat16).view(2, b * hk, p, dh // 64, 2)
    empty = torch.ones(b, hk, p, dtype=torch.bool, device="cuda")
    empty[:, :, :c] = ~taken
    bad = torch.tensor([float("nan"), float("-inf")], dtype=torch.bfloat16, device="cuda")
    tail[:] = torch.where(empty.view(1, b * hk, p, 1, 1), bad.view(1, 1, 1, 1, 2), tail)
    assert tail.numel() * 2 == 2 * pairs
    return cache, pos, k, v


def _attend(b, h, hk, c, dh, dtype, seed=1, fill=0.8, own=True, want=True, scale=0.0, q_scale=2.0, misalign=False):
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    cache, pos, k, v = _random_cache(b, hk, c, dh, dtype, seed, fill)
    g = torch.Generator("cuda").manual_seed(seed + 1000)
    q, kn, vn = ((torch.randn(b, n, dh, generator=g, device="cuda") * f).to(_dt(dtype)) for n, f in ((h, q_scale), (hk, 1.0), (hk, 1.0)))
    if not own:
        kn = vn = None
    out = torch.full_like(q, 7.0)
    w = torch.full((b, h, c + 1), 7.0, device="cuda") if want else None
    lib.adore_q4_attention(q, kn, vn, cache, pos, out, w, scale=scale)
    r, p, mag, delta = ref.decode(q, k, v, kn, vn, pos, scale)
    # sum p (code * step): what the bfloat16 rounding of p * step acts on; |value| + |low| bounds it
    low = torch.where(pos[..., None] >= 0, v.double(), 0.0).unflatten(-1, (-1, 64)).amin(-1, keepdim=True).abs().expand(b, hk, c, dh // 64, 64).flatten(-2)
    lowm = (p[..., :c].view(b, hk, h // hk, c) @ torch.where(pos[..., None] >= 0, low, 0.0)).reshape(b, h, dh)
    half = ref.HALF_STEP[q.dtype]
    f32 = 2 * torch.expm1(delta)[..., None] + (16 + c) * ref.EPS32
    tol = (mag + lowm) * (f32 + (half if dtype == "bf16" else 0)) + 2 * half * r.abs() + 1e-30
    err = (out.double() - r).abs()
    assert (err <= tol).all(), f"out: {(err / tol).max().item():.3f} of the tolerance"
    if want:
        tol = p * f32 + 1e-37
        err = (w.double() - p).abs()
        assert (err <= tol).all(), f"weights: {(err / tol).max().item():.3f} of the tolerance"
        none = torch.full_like(q, 7.0)
        lib.adore_q4_attention(q, kn, vn, cache, pos, none, None, scale=scale)
        assert torch.equal(none, out), "the output depends on whether weights are wanted"
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("c", [1, 2, 15, 16, 17, 31, 64, 255, 1000])
def test_decode_capacities(dtype, dh, c):
    _attend(2, 4, 2, c, dh, dtype)
    _attend(1, 3, 3, c, dh, dtype, seed=2, fill=1.0, own=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,hk", [(1, 1), (7, 1), (8, 1), (9, 1), (16, 1), (17, 1), (40, 2), (32, 32), (64, 8)])
def test_decode_head_groups(dtype, h, hk):
    _attend(2, h, hk, 100, 128, dtype)
    _attend(1, h, hk, 37, 64, dtype, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_with_empty_caches(dtype):
    import torch
    _attend(3, 8, 4, 50, 128, dtype, fill=0.0)                         # the token's own row alone
    out = _attend(3, 8, 4, 50, 128, dtype, fill=0.0, own=False)        # nothing at all
    assert (out == 0).all() and not torch.isnan(out).any()
    _attend(3, 8, 4, 50, 64, dtype, fill=0.05, own=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_scales(dtype):
    _attend(2, 8, 2, 300, 128, dtype, scale=1.0, q_scale=1.0)
    _attend(2, 8, 2, 300, 128, dtype, scale=-0.2)
    _attend(2, 8, 2, 300, 64, dtype, q_scale=40.0)
    _attend(2, 8, 2, 300, 64, dtype, q_scale=1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_many_rows_and_long_caches(dtype):
    _attend(24, 16, 16, 130, 128, dtype)
    _attend(1, 4, 1, 20011, 128, dtype, fill=0.9)
    _attend(1, 2, 2, 5003, 64, dtype, fill=0.5, want=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_rows_in_four_bits(dtype, dh):
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    b, hk, c = 2, 3, 21
    g = torch.Generator("cuda").manual_seed(8)
    k, v = (torch.randn(b * c, hk, dh, generator=g, device="cuda") for _ in range(2))
    k[0] = 0.0                                                        # a row of one value: step 0
    k[1] = 1.25
    k[2] = -3e38 if dtype == "f32" else 1e30
    k[3, :, 5] = 1e4                                                  # one large element
    v[4] = 1e-40                                                      # below the smallest normal number
    v[5] += 1000.0                                                    # a small range far from zero
    v[6, :, ::2] = -0.0
    k, v = k.to(_dt(dtype)), v.to(_dt(dtype))
    start = (torch.arange(b + 1, device="cuda") * c).to(torch.int32)
    cache = torch.zeros(lib.adore_q4_bytes(b, hk, dh, c) + 32, dtype=torch.uint8, device="cuda")
    cache[-32:] = 99
    pos, acc = torch.zeros(b, hk, c, dtype=torch.int32, device="cuda"), torch.zeros(b, hk, c, device="cuda")
    length = torch.zeros(b, hk, dtype=torch.int32, device="cuda")
    lib.adore_evict_prompt(torch.ones(hk, b * c, device="cuda"), k, v, start, 1, cache, pos, acc, length)
    assert (cache[-32:] == 99).all(), "bytes behind the cache were written"
    ko, vo = (torch.zeros(b, hk, c, dh, dtype=_dt(dtype), device="cuda") for _ in range(2))
    lib.adore_q4_read(cache, c, None, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        want = ref.in_four_bits(x.cpu().view(b, c, hk, dh).transpose(1, 2))[0].to(_dt(dtype))
        assert torch.equal(y.cpu(), want)
    slots = torch.tensor([[[3, -1, c, 20, 3]] * hk] * b, dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((b, hk, 5, dh), 7.0, dtype=_dt(dtype), device="cuda") for _ in range(2))
    lib.adore_q4_read(cache, c, slots, kp, vp)
    assert torch.equal(kp[:, :, [0, 3, 4]], ko[:, :, [3, 20, 3]]) and torch.equal(vp[:, :, [0, 3]], vo[:, :, [3, 20]])
    assert (kp[:, :, 1:3] == 0).all() and (vp[:, :, 1:3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_codes_of_rows_full_of_ties_and_of_every_size(dtype, dh):
    """Quotients that are exactly halves of a step, rows of small whole numbers, and magnitudes from subnormal to huge."""
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    g = torch.Generator().manual_seed(dh)
    n, kinds = 400, []
    kinds.append(torch.randint(-20, 21, (n, 1, dh), generator=g).float())                      # short differences
    base = torch.randint(0, 31, (n, 1, dh), generator=g).float() / 2                           # halves of a step of 1
    base[:, :, ::64], base[:, :, 1::64] = 0.0, 15.0
    kinds.append(base * torch.exp2(torch.randint(-60, 60, (n, 1, 1), generator=g).float()))
    kinds.append(torch.randn(n, 1, dh, generator=g) * torch.exp2(torch.randint(-149, 120, (n, 1, 1), generator=g).float()))
    kinds.append(torch.randn(n, 1, dh, generator=g) + 300 * torch.randn(n, 1, 1, generator=g))  # a small range far from zero
    near = base + torch.exp2(torch.randint(-24, -10, (n, 1, dh), generator=g).float()) * torch.sign(torch.randn(n, 1, dh, generator=g))
    kinds.append(near)                                                                         # next to halves
    rows = torch.cat(kinds).to(_dt(dtype)).cuda()
    c = rows.shape[0]
    start = torch.tensor([0, c], dtype=torch.int32, device="cuda")
    cache = torch.zeros(lib.adore_q4_bytes(1, 1, dh, c), dtype=torch.uint8, device="cuda")
    pos, acc = torch.zeros(1, 1, c, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, c, device="cuda")
    length = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    lib.adore_evict_prompt(torch.ones(1, c, device="cuda"), rows, rows.flip(0).contiguous(), start, 1, cache, pos, acc, length)
    k, v = (torch.zeros(1, 1, c, dh, dtype=_dt(dtype), device="cuda") for _ in range(2))
    lib.adore_q4_read(cache, c, None, k, v)
    want = ref.in_four_bits(rows.cpu()[:, 0])[0].to(_dt(dtype))
    assert torch.equal(k.cpu()[0, 0], want) and torch.equal(v.cpu()[0, 0], want.flip(0))


def _evict_prompt(lens, hk, dh, dtype, c, recent, acc, seed=1, pad=0, fused=False):
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    g = torch.Generator("cuda").manual_seed(seed)
    total, b = sum(lens) + pad, len(lens)
    kv = torch.randn(total, 2 * hk + 1, dh, generator=g, device="cuda").to(_dt(dtype))
    kv[sum(lens):] = float("nan")
    k, v = kv[:, :hk], kv[:, hk:2 * hk]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    start = torch.tensor([sum(lens[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda")
    cache = torch.randint(0, 256, (lib.adore_q4_bytes(b, hk, dh, c),), generator=g, device="cuda", dtype=torch.uint8)
    pos, val = torch.full((b, hk, c), 7, dtype=torch.int32, device="cuda"), torch.full((b, hk, c), 7.0, device="cuda")
    length = torch.full((b, hk), 7, dtype=torch.int32, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.adore_evict_prompt(acc, k, v, start, recent, cache, pos, val, length, error_word=word)
    ko, vo = (torch.full((b, hk, c, dh), 7.0, dtype=_dt(dtype), device="cuda") for _ in range(2))
    lib.adore_q4_read(cache, c, None, ko, vo)
    pos, val, ac = pos.cpu(), val.cpu(), acc.cpu()
    for i, n in enumerate(lens):
        at = int(start[i])
        assert (length[i] == n).all()
        for head in range(hk):
            a = ac[head, at:at + n]
            kept = ref.keep(a.tolist(), recent, c)
            m = len(kept)
            assert pos[i, head, :m].tolist() == kept, (i, head)
            assert (pos[i, head, m:] == -1).all() and (val[i, head, m:] == 0).all()
            assert torch.equal(val[i, head, :m].nan_to_num(nan=-77.0), a[kept].nan_to_num(nan=-77.0))
            for x, y in ((k, ko), (v, vo)):
                rows = x[at:at + n, head].cpu()[kept]
                assert torch.equal(y[i, head, :m].cpu(), ref.in_four_bits(rows)[0].to(_dt(dtype)))
                assert (y[i, head, m:] == 0).all()
    assert word.item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c,recent", [(1, 1), (16, 1), (16, 16), (17, 5), (100, 37), (700, 1)])
def test_evict_prompt_keeps_the_most_valuable(dtype, c, recent):
    import torch
    lens = [0, 1, 15, 16, 17, 99, 100, 101, 513, 1100]
    g = torch.Generator("cuda").manual_seed(c)
    acc = torch.exp(2 * torch.randn(3, sum(lens) + 4, generator=g, device="cuda"))
    _evict_prompt(lens, 3, 128 if c % 2 else 64, dtype, c, recent, acc, pad=4, fused=c > 16)


def test_evict_prompt_ties_and_odd_values():
    import torch
    lens = [700, 40, 2000]
    g = torch.Generator("cuda").manual_seed(3)
    acc = torch.randint(0, 4, (2, sum(lens)), generator=g, device="cuda").float()      # few distinct values
    _evict_prompt(lens, 2, 64, "bf16", 100, 10, acc)
    _evict_prompt(lens, 2, 64, "bf16", 100, 10, torch.zeros_like(acc))                  # all alike
    _evict_prompt(lens, 2, 64, "bf16", 100, 100, acc)                                   # only the newest
    acc[0, 5::7] = float("nan")
    acc[0, 6::7] = float("inf")
    acc[1, 5::7] = float("-inf")
    acc[1, 6::7] = -0.0
    acc[1, 4::7] = -1.5
    _evict_prompt(lens, 2, 64, "bf16", 300, 10, acc)
    acc[0] = float("nan")
    _evict_prompt(lens, 2, 64, "f32", 300, 10, acc)


def test_evict_prompt_long_rows():
    import torch
    g = torch.Generator("cuda").manual_seed(4)
    acc = torch.exp(2 * torch.randn(2, 70001, generator=g, device="cuda"))
    _evict_prompt([70001], 2, 64, "bf16", 1000, 100, acc)
    _evict_prompt([60000, 10001], 2, 64, "bf16", 20001, 1, acc)


def test_evict_prompt_one_long_row_among_short_ones():
    import torch
    lens = [6000] + [3, 50] * 6                                       # the average picks the variant for short rows
    g = torch.Generator("cuda").manual_seed(6)
    acc = torch.randint(0, 300, (2, sum(lens)), generator=g, device="cuda").float()
    _evict_prompt(lens, 2, 64, "bf16", 40, 7, acc)
    _evict_prompt(lens, 2, 64, "f32", 5000, 1, acc)


def test_evict_prompt_with_no_tokens():
    import torch
    from paper_2407_02328_b200 import adore as lib
    for total in (0, 6):
        k, acc = torch.zeros(total, 2, 64, device="cuda").bfloat16(), torch.zeros(2, total, device="cuda")
        cache = torch.full((lib.adore_q4_bytes(3, 2, 64, 20),), 255, dtype=torch.uint8, device="cuda")
        pos, val = torch.zeros(3, 2, 20, dtype=torch.int32, device="cuda"), torch.ones(3, 2, 20, device="cuda")
        length = torch.ones(3, 2, dtype=torch.int32, device="cuda")
        lib.adore_evict_prompt(acc, k, k, torch.zeros(4, dtype=torch.int32, device="cuda"), 5, cache, pos, val, length)
        assert (pos == -1).all() and (val == 0).all() and (length == 0).all() and (cache == 0).all()


def test_evict_prompt_skips_bad_sequences():
    import torch
    from paper_2407_02328_b200 import adore as lib
    k = torch.randn(100, 1, 64, device="cuda").bfloat16()
    acc = torch.rand(1, 100, device="cuda")
    cache = torch.zeros(lib.adore_q4_bytes(2, 1, 64, 8), dtype=torch.uint8, device="cuda")
    pos, val = torch.zeros(2, 1, 8, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, 8, device="cuda")
    length = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 50, 101], dtype=torch.int32, device="cuda")
    lib.adore_evict_prompt(acc, k, k, start, 2, cache, pos, val, length, error_word=word)
    assert word.item() == 4 and length.flatten().tolist() == [50, 0]
    assert (pos[1] == -1).all() and (pos[0] >= 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,hk,c,recent", [(4, 4, 1, 1), (8, 2, 16, 3), (7, 1, 33, 33), (4, 2, 300, 40), (2, 1, 5000, 100)])
def test_evict_steps(dtype, h, hk, c, recent):
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    b, dh = 3, 128
    g = torch.Generator("cuda").manual_seed(c)
    cache = torch.randint(0, 256, (lib.adore_q4_bytes(b, hk, dh, c),), generator=g, device="cuda", dtype=torch.uint8)
    n0 = c - min(c, 6)
    pos = torch.where(torch.arange(c, device="cuda") < n0, torch.arange(c, device="cuda"), -1).to(torch.int32).repeat(b, hk, 1).contiguous()
    val = torch.rand(b, hk, c, generator=g, device="cuda") * (pos >= 0)
    length = torch.full((b, hk), n0, dtype=torch.int32, device="cuda")
    length[1] = -1                                                     # a padded sequence
    admit, evicted = (torch.zeros(b, hk, dtype=torch.int32, device="cuda") for _ in range(2))
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    state = [x.cpu().clone() for x in (pos, val, length)]
    for _ in range(20):
        w = torch.rand(b, h, c + 1, generator=g, device="cuda")
        k, v = (torch.randn(b, hk, dh, generator=g, device="cuda").to(_dt(dtype)) for _ in range(2))
        before = cache.clone()
        lib.adore_evict_step(w, k, v, recent, cache, pos, val, length, admit, evicted, error_word=word)
        r_admit, r_evicted = ref.step(w.cpu(), *state, recent)
        assert torch.equal(admit.cpu(), r_admit) and torch.equal(evicted.cpu(), r_evicted)
        for x, y in zip((pos, val, length), state):
            assert torch.equal(x.cpu(), y)
        kr, vr = (torch.zeros(b, hk, c, dh, dtype=_dt(dtype), device="cuda") for _ in range(2))
        kb, vb = kr.clone(), vr.clone()
        lib.adore_q4_read(cache, c, None, kr, vr)
        lib.adore_q4_read(before, c, None, kb, vb)
        hit = torch.nn.functional.one_hot(admit.long().clamp(min=0), c).bool() & (admit >= 0)[..., None]
        for x, old, rows in ((kr, kb, k), (vr, vb, v)):
            assert torch.equal(x[~hit].view(torch.uint8), old[~hit].view(torch.uint8)), "another slot's row changed"
            assert torch.equal(x[hit], ref.in_four_bits(rows.cpu())[0].to(_dt(dtype)).cuda()[admit >= 0])
    assert word.item() == 0 and (length[1] == -1).all()


def test_evict_step_ties_odd_values_and_nothing_to_release():
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    b, h, hk, c, dh = 1, 2, 2, 40, 64
    cache = torch.zeros(lib.adore_q4_bytes(b, hk, dh, c), dtype=torch.uint8, device="cuda")
    k = torch.randn(b, hk, dh, device="cuda").bfloat16()
    for kind in range(4):
        pos = torch.arange(c, dtype=torch.int32, device="cuda").repeat(b, hk, 1).contiguous()
        val = torch.ones(b, hk, c, device="cuda")
        if kind == 1:
            val[0, 0, 7] = val[0, 0, 9] = float("nan")
            val[0, 1, 5] = float("-inf")
        if kind == 2:
            val.fill_(float("inf"))
        if kind == 3:
            pos += 1000                                                # every position newer than the step's own
        length = torch.full((b, hk), 60, dtype=torch.int32, device="cuda")
        admit, evicted = (torch.zeros(b, hk, dtype=torch.int32, device="cuda") for _ in range(2))
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        w = torch.zeros(b, h, c + 1, device="cuda")
        state = [x.cpu().clone() for x in (pos, val, length)]
        lib.adore_evict_step(w, k, k, 1, cache, pos, val, length, admit, evicted, error_word=word)
        r_admit, r_evicted = ref.step(w.cpu(), *state, 1)
        assert torch.equal(admit.cpu(), r_admit) and torch.equal(evicted.cpu(), r_evicted)
        assert torch.equal(pos.cpu(), state[0]) and torch.equal(val.cpu().nan_to_num(nan=-7.0), state[1].nan_to_num(nan=-7.0))
        assert length.flatten().tolist() == [61, 61] and word.item() == (4 if kind == 3 else 0)


def test_decode_across_a_cluster_captured_and_on_two_streams():
    """Long caches are shared by a cluster of CTAs: the same bits from a graph and with another call beside it."""
    import torch
    from paper_2407_02328_b200 import adore as lib
    b, h, hk, c, dh = 2, 8, 2, 9001, 128
    sets = []
    for seed in (1, 2):
        cache, pos, _, _ = _random_cache(b, hk, c, dh, "bf16", seed, 0.9)
        q, kn, vn = (torch.randn(b, n, dh, device="cuda").bfloat16() for n in (h, hk, hk))
        sets.append((q, kn, vn, cache, pos, torch.zeros_like(q), torch.zeros(b, h, c + 1, device="cuda")))
    alone = []
    for s in sets:
        lib.adore_q4_attention(*s)
        alone.append((s[5].clone(), s[6].clone()))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                lib.adore_q4_attention(*s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s in sets:
            lib.adore_q4_attention(*s)
    for s, a in zip(sets, alone):
        assert torch.equal(s[5], a[0]) and torch.equal(s[6], a[1])
        s[5].zero_()
        s[6].zero_()
    graph.replay()
    for s, a in zip(sets, alone):
        assert torch.equal(s[5], a[0]) and torch.equal(s[6], a[1])


@pytest.mark.parametrize("dtype,h,hk,dh", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
def test_prompt_then_decoding_as_a_user_runs_it(dtype, h, hk, dh):
    """Prompt attention, received weights, eviction, then decode steps: every call's result against float64 on the state that the
    calls before it left, once eagerly and once as a replayed graph with the same bits."""
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    lens, c, recent, steps = [90, 7, 200], 48, 8, 60
    b, dt, total = len(lens), _dt(dtype), sum(lens)
    g = torch.Generator("cuda").manual_seed(12)
    q, k, v = (torch.randn(total, n, dh, generator=g, device="cuda").to(dt) for n in (h, hk, hk))
    start = torch.tensor([0, 90, 97, 297], dtype=torch.int32, device="cuda")
    xs = [[torch.randn(b, n, dh, generator=g, device="cuda").to(dt) for n in (h, hk, hk)] for _ in range(steps)]

    def load():
        s = dict(out=torch.zeros_like(q), lse=torch.zeros(h, total, device="cuda"), acc=torch.zeros(hk, total, device="cuda"),
                 cache=torch.zeros(lib.adore_q4_bytes(b, hk, dh, c), dtype=torch.uint8, device="cuda"),
                 pos=torch.zeros(b, hk, c, dtype=torch.int32, device="cuda"), val=torch.zeros(b, hk, c, device="cuda"),
                 length=torch.zeros(b, hk, dtype=torch.int32, device="cuda"))
        lib.adore_prompt_attention(q, k, v, start, s["out"], s["lse"])
        lib.adore_prompt_weights(q, k, s["lse"], start, s["acc"])
        lib.adore_evict_prompt(s["acc"], k, v, start, recent, s["cache"], s["pos"], s["val"], s["length"])
        return s

    def one(s, x, out, w, admit, evicted):
        lib.adore_q4_attention(*x, s["cache"], s["pos"], out, w)
        lib.adore_evict_step(w, x[1], x[2], recent, s["cache"], s["pos"], s["val"], s["length"], admit, evicted)

    s = load()
    assert torch.allclose(s["acc"].double().sum(), torch.tensor(float(total * h), dtype=torch.float64, device="cuda"), rtol=1e-4)
    outs = []
    out, w = torch.zeros(b, h, dh, dtype=dt, device="cuda"), torch.zeros(b, h, c + 1, device="cuda")
    admit, evicted = (torch.zeros(b, hk, dtype=torch.int32, device="cuda") for _ in range(2))
    for x in xs:
        rows = [torch.zeros(b, hk, c, dh, device="cuda") for _ in range(2)]
        c32 = s["cache"]
        lib.adore_q4_read(c32, c, None, *rows)
        r, p, mag, delta = ref.decode(x[0], *rows, x[1], x[2], s["pos"])
        state = [s[n].cpu().clone() for n in ("pos", "val", "length")]
        one(s, x, out, w, admit, evicted)
        assert (out.double() - r).abs().max() <= (0.06 if dtype == "bf16" else 1e-4)
        assert (w.double() - p).abs().max() <= 1e-5
        r_admit, r_evicted = ref.step(w.cpu(), *state, recent)
        assert torch.equal(admit.cpu(), r_admit) and torch.equal(evicted.cpu(), r_evicted)
        for n, y in zip(("pos", "val", "length"), state):
            assert torch.equal(s[n].cpu(), y)
        outs.append(out.clone())
    assert s["length"][0, 0].item() == 90 + steps and (s["pos"] >= 0).all()
    assert (s["pos"].amax(-1) == s["length"] - 1).all()

    t = load()
    x = [y.clone() for y in xs[0]]
    out2, w2 = torch.zeros_like(out), torch.zeros_like(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(t, x, out2, w2, admit, evicted)
    t2 = load()
    for n in t:
        t[n].copy_(t2[n])
    for i in range(steps):
        for y, z in zip(x, xs[i]):
            y.copy_(z)
        graph.replay()
        assert torch.equal(out2, outs[i])
    for n in ("pos", "val", "length", "cache"):
        assert torch.equal(s[n], t[n])
