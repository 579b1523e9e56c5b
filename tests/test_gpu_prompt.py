"""Prompt attention and the attention weights of a prompt: the CUDA kernels against float64."""
import pytest

pytestmark = pytest.mark.gpu


def _seq(lens, lead=0):
    import torch
    at = [lead]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _inputs(lens, h, hk, dh, dtype, seed, pad=0, lead=0, layout="rows", q_scale=2.0):
    """layout: rows (contiguous), fused (parts of one projection), heads (head-major)."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator("cuda").manual_seed(seed)
    total = lead + sum(lens) + pad
    rows = torch.randn(total, h + 2 * hk, dh, generator=g, device="cuda")
    rows[:, :h] *= q_scale
    rows[:lead] = float("nan")                      # rows that belong to no sequence
    rows[lead + sum(lens):] = float("inf")
    rows = rows.to(dt)
    if layout == "heads":
        rows = rows.transpose(0, 1).contiguous().transpose(0, 1)
    parts = rows[:, :h], rows[:, h:h + hk], rows[:, h + hk:]
    return [x.contiguous() for x in parts] if layout == "rows" else list(parts)


def _check(lens, h=4, hk=2, dh=64, dtype="bf16", seed=1, pad=0, lead=0, layout="rows", scale=0.0, q_scale=2.0, window=0, out_layout="rows"):
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    q, k, v = _inputs(lens, h, hk, dh, dtype, seed, pad, lead, layout, q_scale)
    start, total = _seq(lens, lead), q.shape[0]
    if out_layout == "rows":
        out = torch.full((total, h, dh), 7.0, dtype=q.dtype, device="cuda")
    else:
        out = torch.full((h, total, dh), 7.0, dtype=q.dtype, device="cuda").transpose(0, 1)
    lse = torch.full((h, total), 7.0, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.adore_prompt_attention(q, k, v, start, out, lse, scale=scale, error_word=word)
    r_out, r_lse, mag, delta = ref.attention(q, k, v, start, scale)
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    used[lead:lead + sum(lens)] = True
    assert (out[~used] == 7).all() and (lse[:, ~used] == 7).all(), "rows of no sequence were written"
    d = delta.T[used][..., None]
    half = ref.HALF_STEP[q.dtype]
    longest = max(lens)
    # every weight: its logit's error twice (row maximum and logit), 4 units of the exponential, the running sums; in bf16
    # the rounding of the weight to bfloat16; then the rounding of the output
    tol = mag[used] * (2 * torch.expm1(d) + (8 + longest) * ref.EPS32 + (half if dtype == "bf16" else 0)) + r_out[used].abs() * 2 * half + 1e-30
    err = (out.double()[used] - r_out[used]).abs()
    assert (err <= tol).all(), f"out: {(err / tol).max().item():.3f} of the tolerance"
    tol = 2 * d[..., 0].T + (16 + longest) * ref.EPS32 + 4 * ref.EPS32 * r_lse[:, used].abs()
    err = (lse.double()[:, used] - r_lse[:, used]).abs()
    assert (err <= tol).all(), f"lse: {(err / tol).max().item():.3f} of the tolerance"
    for w in {window, 0}:
        acc = torch.full((hk, total), 7.0, device="cuda")
        lib.adore_prompt_weights(q, k, lse, start, acc, window=w, scale=scale, error_word=word)
        r_acc, tol = ref.received(q, k, lse, start, w, scale)
        assert (acc[:, ~used] == 7).all()
        err = (acc.double()[:, used] - r_acc[:, used]).abs()
        tol = tol[:, used] + 1e-30
        assert (err <= tol).all(), f"weights, window {w}: {(err / tol).max().item():.3f} of the tolerance"
        again = torch.zeros_like(acc)
        lib.adore_prompt_weights(q, k, lse, start, again, window=w, scale=scale)
        assert torch.equal(again[:, used], acc[:, used]), "the same inputs gave other bits"
    assert word.item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_lengths_around_the_tiles(dtype, dh):
    _check([1], dh=dh, dtype=dtype)
    _check([1, 0, 2, 63, 64, 65, 0, 127, 128, 129], dh=dh, dtype=dtype, window=64)
    _check([255, 256, 257, 383, 384, 385], h=2, hk=1, dh=dh, dtype=dtype, pad=3, window=100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["fused", "heads"])
def test_strides_and_rows_of_no_sequence(dtype, layout):
    _check([70, 1, 200], h=6, hk=3, dh=128, dtype=dtype, pad=5, lead=7, layout=layout, out_layout=layout, window=33)
    _check([150], h=3, hk=3, dh=64, dtype=dtype, pad=130, lead=1, layout=layout, window=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,hk", [(1, 1), (7, 1), (8, 2), (32, 8)])
def test_head_groups(dtype, h, hk):
    _check([130, 17], h=h, hk=hk, dh=128, dtype=dtype, window=40)


def test_more_sequences_than_lanes():
    _check([(7 * i) % 40 for i in range(100)], h=2, hk=2, dh=64)
    _check([300] * 33 + [5], h=1, hk=1, dh=64, window=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_and_peaked_rows(dtype):
    _check([200, 40], dtype=dtype, scale=0.37, dh=128)
    _check([200, 40], dtype=dtype, scale=-0.1)
    _check([300], dtype=dtype, q_scale=30.0, dh=128)          # one weight near 1, the maximum moves often
    _check([300], dtype=dtype, q_scale=1e-3)                  # all weights alike


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_tiles_than_ctas(dtype):
    _check([200, 130, 300, 1, 64] * 12, h=8, hk=4, dh=64, dtype=dtype, window=90)          # several tiles per persistent CTA
    _check([270, 120] * 12, h=8, hk=8, dh=128, dtype=dtype, pad=9)


def test_empty_batches_and_empty_sequences():
    import torch
    from paper_2407_02328_b200 import adore as lib
    for total in (0, 5):
        q, k = torch.zeros(total, 4, 64, device="cuda").bfloat16(), torch.zeros(total, 2, 64, device="cuda").bfloat16()
        out, lse, acc = torch.full_like(q, 7.0), torch.full((4, total), 7.0, device="cuda"), torch.full((2, total), 7.0, device="cuda")
        start = torch.zeros(4, dtype=torch.int32, device="cuda")
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        lib.adore_prompt_attention(q, k, k, start, out, lse, error_word=word)
        lib.adore_prompt_weights(q, k, lse, start, acc, error_word=word)
        assert (out == 7).all() and (lse == 7).all() and (acc == 7).all() and word.item() == 0


def test_two_streams_at_once():
    import torch
    from paper_2407_02328_b200 import adore as lib
    lens = [900, 300, 77]
    start, sets = _seq(lens), []
    for seed in range(3):
        q, k, v = _inputs(lens, 8, 2, 128, "bf16", seed)
        sets.append((q, k, v, torch.zeros_like(q), torch.zeros(8, sum(lens), device="cuda"), torch.zeros(2, sum(lens), device="cuda")))

    def run(q, k, v, out, lse, acc):
        lib.adore_prompt_attention(q, k, v, start, out, lse)
        lib.adore_prompt_weights(q, k, lse, start, acc)

    alone = []
    for s in sets:
        run(*s)
        alone.append([x.clone() for x in s[3:]])
        for x in s[3:]:
            x.zero_()
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                run(*s)
    torch.cuda.synchronize()
    for s, a in zip(sets, alone):
        for x, y in zip(s[3:], a):
            assert torch.equal(x, y)


def test_long_prompt_bf16():
    _check([2500, 1, 611], h=4, hk=1, dh=128, window=32)


def test_growing_logits_move_the_maximum_in_every_block():
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    n, dh = 1100, 128
    g = torch.Generator("cuda").manual_seed(5)
    q = torch.ones(n, 1, dh, device="cuda").bfloat16()
    k = (torch.arange(n, device="cuda").view(n, 1, 1) * 0.01).expand(n, 1, dh).bfloat16().contiguous()
    v = torch.randn(n, 1, dh, generator=g, device="cuda").bfloat16()
    out, start = torch.zeros_like(q), _seq([n])
    lib.adore_prompt_attention(q, k, v, start, out)
    r, _, mag, delta = ref.attention(q, k, v, start)
    d = delta.T[..., None]
    assert ((out.double() - r).abs() <= mag * (2 * torch.expm1(d) + 2.0 ** -8 + 1200 * ref.EPS32) + 2.0 ** -7 * r.abs()).all()
    out2 = torch.zeros_like(q)
    k2 = k.flip(0).contiguous()                               # and falling ones never do
    lib.adore_prompt_attention(q, k2, v, start, out2)
    r, _, mag, delta = ref.attention(q, k2, v, start)
    d = delta.T[..., None]
    assert ((out2.double() - r).abs() <= mag * (2 * torch.expm1(d) + 2.0 ** -8 + 1200 * ref.EPS32) + 2.0 ** -7 * r.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_sequence_ends_are_skipped_and_reported(dtype):
    import torch
    from paper_2407_02328_b200 import adore as lib
    q, k, v = _inputs([100, 60], 2, 1, 64, dtype, 9)
    for ends, good in (([0, 100, 161], [(0, 100)]), ([-1, 100, 160], [(100, 160)]), ([0, 100, 50], [(0, 100)]),
                       ([5, 2 ** 31 - 1, 160], [])):
        start = torch.tensor(ends, dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(q, 7.0), torch.full((2, 160), 7.0, device="cuda")
        acc = torch.full((1, 160), 7.0, device="cuda")
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        lib.adore_prompt_attention(q, k, v, start, out, lse, error_word=word)
        assert word.item() == 4
        word.zero_()
        lib.adore_prompt_weights(q, k, lse, start, acc, error_word=word)
        assert word.item() == 4
        for t in (0, 99, 100, 159):
            inside = any(a <= t < b for a, b in good)
            assert (lse[0, t].item() != 7) == inside and (acc[0, t].item() != 7) == inside
        lib.adore_prompt_attention(q, k, v, start, out)        # no word to report to


def test_side_stream_and_graph_replay():
    import torch
    from paper_2407_02328_b200 import adore as lib
    from tests import prompt_reference as ref
    q, k, v = _inputs([300, 20], 4, 2, 128, "bf16", 3)
    start = _seq([300, 20])
    out, lse, acc = torch.zeros_like(q), torch.zeros(4, 320, device="cuda"), torch.zeros(2, 320, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def both():
        lib.adore_prompt_attention(q, k, v, start, out, lse)
        lib.adore_prompt_weights(q, k, lse, start, acc, window=50)

    with torch.cuda.stream(side):
        both()
    side.synchronize()
    first = out.clone(), lse.clone(), acc.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    q2, k2, v2 = _inputs([300, 20], 4, 2, 128, "bf16", 4)
    keep = [x.clone() for x in (q, k, v)]
    for x, y in zip((q, k, v), (q2, k2, v2)):
        x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    r, _, _, _ = ref.attention(q, k, v, start)
    assert (out.double() - r).abs().max() < 0.05
    start.copy_(_seq([20, 300]))                               # other lengths within the same total
    graph.replay()
    r, _, _, _ = ref.attention(q, k, v, start)
    assert (out.double() - r).abs().max() < 0.05
    start.copy_(_seq([300, 20]))
    for x, y in zip((q, k, v), keep):
        x.copy_(y)
    graph.replay()
    for a, b in zip(first, (out, lse, acc)):
        assert torch.equal(a, b)
