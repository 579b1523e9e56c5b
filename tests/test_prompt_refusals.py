"""Arguments that the prompt, eviction and 4-bit calls refuse on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

A = 1 << 20          # an address on a 16-byte boundary; nothing is ever read from it here


def _prompt(lib, **kw):
    f = dict(struct_size=C.sizeof(lib.adore_prompt_t), dtype=lib.ADORE_BF16, n_seqs=2, total=100, n_heads=8, n_kv_heads=2, head_dim=128,
             scale=0.0, q_row=1024, q_head=128, k_row=256, k_head=128, v_row=256, v_head=128, out_row=1024, out_head=128)
    f.update(kw)
    return lib.adore_prompt_t(**f)


def _q4(lib, **kw):
    f = dict(struct_size=C.sizeof(lib.adore_q4_t), dtype=lib.ADORE_BF16, batch=2, n_heads=8, n_kv_heads=2, head_dim=128, capacity=40, scale=0.0)
    f.update(kw)
    return lib.adore_q4_t(**f)


@pytest.fixture(scope="module")
def lib():
    from paper_2407_02328_b200 import adore, build
    build.build()
    return adore


BAD_PROMPTS = [
    (dict(struct_size=4), 1), (dict(dtype=2), 1), (dict(n_seqs=0), 1), (dict(total=-1), 1), (dict(n_heads=0), 1), (dict(n_kv_heads=0), 1),
    (dict(n_kv_heads=3), 1), (dict(head_dim=0), 1), (dict(head_dim=96), 8), (dict(head_dim=256), 8), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(q_row=1028), 1), (dict(k_head=4), 1), (dict(k_row=0), 1), (dict(q_head=-128), 1),
    (dict(q_head=64), 1), (dict(total=0x7fff0001), 8), (dict(total=0x7fff0000, k_row=1 << 38), 1), (dict(q_row=1 << 40), 1), (dict(dtype=0, q_row=1026), 1),
]


@pytest.mark.parametrize("change,status", BAD_PROMPTS)
def test_packed_shapes(lib, change, status):
    l, p = lib._lib(), _prompt(lib, **change)
    assert l.adore_prompt_attention(C.byref(p), A, A, A, A, A, A, None, None) == status
    assert l.adore_prompt_weights(C.byref(p), A, A, A, A, 0, A, None, None) == status


def test_packed_pointers(lib):
    l, p = lib._lib(), _prompt(lib)
    assert l.adore_prompt_attention(None, A, A, A, A, A, A, None, None) == 1
    for i in range(5):                                    # seq_start, q, k, v, out missing or off their boundary
        args = [A, A, A, A, A, A, None, None]
        args[i] = None
        assert l.adore_prompt_attention(C.byref(p), *args) == 1
        args[i] = A + 2
        assert l.adore_prompt_attention(C.byref(p), *args) == 1
    assert l.adore_prompt_attention(C.byref(p), A, A, A, A, A, A + 1, None, None) == 1
    assert l.adore_prompt_attention(C.byref(p), A, A, A, A, A, A, A + 2, None) == 1
    for i in (0, 1, 2, 3, 5):
        args = [A, A, A, A, 0, A, None, None]
        args[i] = None
        assert l.adore_prompt_weights(C.byref(p), *args) == 1
    assert l.adore_prompt_weights(C.byref(p), A, A, A, A, -1, A, None, None) == 1
    # rows of the output that overlap, in either order of the strides
    for change in (dict(v_row=100), dict(v_head=8), dict(out_row=512), dict(out_head=128, out_row=128), dict(out_row=128, out_head=1280)):
        q = _prompt(lib, **change)
        assert l.adore_prompt_attention(C.byref(q), A, A, A, A, A, A, None, None) == 1
    # an empty batch needs no pointers but its sequence ends and launches nothing
    q = _prompt(lib, total=0)
    assert l.adore_prompt_attention(C.byref(q), A, None, None, None, None, None, None, None) == 0
    assert l.adore_prompt_weights(C.byref(q), A, None, None, None, 0, None, None, None) == 0
    assert l.adore_prompt_attention(C.byref(q), None, None, None, None, None, None, None, None) == 1


BAD_CACHES = [
    (dict(struct_size=8), 1), (dict(dtype=5), 1), (dict(batch=0), 1), (dict(capacity=0), 1), (dict(n_heads=7), 1), (dict(n_kv_heads=-1), 1),
    (dict(head_dim=80), 8), (dict(scale=float("inf")), 1), (dict(capacity=2 ** 31 - 1), 8), (dict(batch=2 ** 30, n_heads=8), 8),
]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_cache_shapes(lib, change, status):
    l, c = lib._lib(), _q4(lib, **change)
    assert l.adore_q4_bytes(C.byref(c)) == 0
    assert l.adore_q4_attention(C.byref(c), A, A, A, A, A, A, A, None) == status
    assert l.adore_q4_read(C.byref(c), A, A, 1, A, A, None) == status
    assert l.adore_evict_step(C.byref(c), A, A, A, 1, A, A, A, A, A, A, None, None) == status
    assert l.adore_evict_prompt(C.byref(c), C.byref(_prompt(lib)), A, A, A, A, 1, A, A, A, A, None, None) == status


def test_cache_pointers_and_counts(lib):
    l, c, p = lib._lib(), _q4(lib), _prompt(lib)
    for i in range(6):
        if i in (1, 2):
            continue                                      # k_new and v_new may both be missing, not one of them
        args = [A] * 7 + [None]
        if i < 6:
            args[i] = None
        assert l.adore_q4_attention(C.byref(c), *args) == 1
    assert l.adore_q4_attention(C.byref(c), A, None, A, A, A, A, A, None) == 1
    assert l.adore_q4_attention(C.byref(c), A, A, None, A, A, A, A, None) == 1
    for i in (0, 1, 2, 3, 5):
        args = [A] * 7 + [None]
        args[i] = A + 8
        assert l.adore_q4_attention(C.byref(c), *args) == 1
    for recent in (0, -1, 41):
        assert l.adore_evict_step(C.byref(c), A, A, A, recent, A, A, A, A, A, A, None, None) == 1
        assert l.adore_evict_prompt(C.byref(c), C.byref(p), A, A, A, A, recent, A, A, A, A, None, None) == 1
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9):
        args = [A, A, A, 1, A, A, A, A, A, A, None, None]
        if args[i] == 1:
            continue
        args[i] = None
        assert l.adore_evict_step(C.byref(c), *args) == 1
    for change in (dict(n_seqs=3), dict(n_heads=4, n_kv_heads=2), dict(n_kv_heads=4, k_row=512, v_row=512), dict(head_dim=64), dict(dtype=0)):
        assert l.adore_evict_prompt(C.byref(c), C.byref(_prompt(lib, **change)), A, A, A, A, 1, A, A, A, A, None, None) == 1
    for i in (0, 1, 2, 3, 5, 6, 7, 8):
        args = [A, A, A, A, 1, A, A, A, A, None, None]
        if args[i] == 1:
            continue
        args[i] = None
        assert l.adore_evict_prompt(C.byref(c), C.byref(p), *args) == 1
    assert l.adore_q4_read(C.byref(c), A, None, 39, A, A, None) == 1
    assert l.adore_q4_read(C.byref(c), A, A, -1, A, A, None) == 1
    assert l.adore_q4_read(C.byref(c), A, A, 3, None, A, None) == 1
    assert l.adore_q4_read(C.byref(c), A + 4, A, 3, A, A, None) == 1
    assert l.adore_q4_read(C.byref(c), A, A, 0, None, None, None) == 0


def test_bytes_of_a_cache(lib):
    # 16-slot padding, 4 bits an element, a step and a low value of 2 bytes per 64 elements, keys and values
    assert lib.adore_q4_bytes(2, 3, 128, 40) == 2 * 3 * 48 * 2 * (64 + 8)
    assert lib.adore_q4_bytes(1, 1, 64, 1) == 16 * 2 * (32 + 4)
    with pytest.raises(lib.AdoreError) as e:
        lib.adore_q4_bytes(1, 1, 48, 1)
    assert e.value.status == 1


def test_the_binding_refuses_tensors_that_do_not_fit(lib):
    import torch
    bf = torch.bfloat16
    q, k = torch.zeros(10, 4, 64, dtype=bf), torch.zeros(10, 2, 64, dtype=bf)
    start = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: lib.adore_prompt_attention(q, k, k, start, q),                       # on the CPU
                 lambda: lib.adore_prompt_attention(q, k[:9], k, start, q),
                 lambda: lib.adore_prompt_attention(q, k.transpose(1, 2), k, start, q),
                 lambda: lib.adore_prompt_attention(q, k.float(), k, start, q),
                 lambda: lib.adore_prompt_attention(q, k, k, start.long(), q),
                 lambda: lib.adore_prompt_attention(q.half(), k.half(), k.half(), start, q.half()),
                 lambda: lib.adore_prompt_attention(q[0], k, k, start, q),
                 lambda: lib.adore_prompt_weights(q, k, torch.zeros(4, 9), start, torch.zeros(2, 10)),
                 lambda: lib.adore_q4_attention(q, k, k, torch.zeros(1, dtype=torch.uint8), torch.zeros(10, 2, 5, dtype=torch.int32), q),
                 lambda: lib.adore_q4_read(torch.zeros(9, dtype=torch.uint8), 5, None, torch.zeros(1, 1, 5, 64), torch.zeros(1, 1, 5, 64)),
                 lambda: lib.adore_evict_step(torch.zeros(10, 4, 6), k, k, 1, torch.zeros(1, dtype=torch.uint8),
                                              torch.zeros(10, 2, 5, dtype=torch.int32), torch.zeros(10, 2, 5),
                                              torch.zeros(10, 2, dtype=torch.int32), None, None)):
        with pytest.raises(lib.AdoreError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("shape", [dict(batch=65536, n_heads=1, n_kv_heads=1), dict(batch=1, n_heads=65536, n_kv_heads=65536)])
def test_rows_beyond_a_grids_dimensions(lib, shape):
    """Fills and reads refuse what their grids cannot hold, before the selection has written anything."""
    l, c = lib._lib(), _q4(lib, **shape)
    row = 128 * c.n_kv_heads
    p = _prompt(lib, n_seqs=c.batch, n_heads=c.n_heads, n_kv_heads=c.n_kv_heads, k_row=row, v_row=row)
    assert l.adore_evict_prompt(C.byref(c), C.byref(p), A, A, A, A, 1, A, A, A, A, None, None) == 8
    assert l.adore_q4_read(C.byref(c), A, A, 1, A, A, None) == 8
