"""Refusals of the calls around the attention (tables, norms with rotation, 4-bit cache): before anything is launched."""
import ctypes
import random

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    import paper_2503_03588_b200.binding as binding

    return binding


BUF = (ctypes.c_int64 * 64)()
P = (ctypes.addressof(BUF) + 15) // 16 * 16
NULL = ctypes.c_void_p(0)


def _changed(params, **kv):
    bad = type(params).from_buffer_copy(params)
    for k, v in kv.items():
        if k in ("page_stride", "head_stride", "head_dim", "n_kv_heads", "n_pages", "block") and hasattr(bad, "pool"):
            setattr(bad.pool, k, v)
        else:
            setattr(bad, k, v)
    return ctypes.byref(bad)


def test_tables_refusals(b):
    good = b.pa_table_params(4, 64, 8, 100, 256, 100)

    def status(p, at=None, value=0, ws=P, ws_bytes=10 ** 6):
        args = [P] * 10
        if at is not None:
            args[at] = value
        return b.pa_status_string(b.lib.pa_build_block_tables(p, *args, ws, ws_bytes, NULL))

    for bad in (dict(batch=0), dict(max_blocks_per_seq=0), dict(n_pages=0), dict(max_tokens=0), dict(free_capacity=-1)):
        assert status(_changed(good, **bad)) == "PA_ERR_INVALID_ARG", bad
        assert b.lib.pa_build_block_tables_workspace_bytes(_changed(good, **bad)) == 0
    assert status(None) == "PA_ERR_INVALID_ARG"
    assert status(_changed(good, block=128)) == "PA_ERR_SHAPE"
    for bad in (dict(batch=65536), dict(max_tokens=2 ** 30 + 1), dict(free_capacity=2 ** 30 + 1)):
        assert status(_changed(good, **bad)) == "PA_ERR_SHAPE", bad
    for at in range(10):
        assert status(_changed(good), at) == "PA_ERR_INVALID_ARG", at
    assert status(_changed(good), 6, P + 4) == "PA_ERR_ALIGNMENT"      # slots are 8 bytes each
    assert status(_changed(good), 4, P + 2) == "PA_ERR_ALIGNMENT"
    assert status(_changed(good), ws=0) == status(_changed(good), ws_bytes=16) == "PA_ERR_WORKSPACE"
    assert status(_changed(good), ws=P + 4) == "PA_ERR_ALIGNMENT"


def test_rope_refusals(b):
    s, o = b.pa_strides(0, 512, 128), b.pa_strides(4096, 512, 128)
    good = b.pa_rope_params(1, 4, 2, 128, 100, 128, 0, 100, 1e-6, b.PA_BF16, s, s, o, o)

    def forward(p, at=None, value=0):
        args = [P] * 8
        if at is not None:
            args[at] = value
        return b.pa_status_string(b.lib.pa_qk_norm_rope(p, *args, NULL))

    def backward(p, at=None, value=0, dtype=b.PA_F32, ws=P, ws_bytes=10 ** 7):
        args = [P] * 12
        if at is not None:
            args[at] = value
        return b.pa_status_string(b.lib.pa_qk_norm_rope_backward(p, *args[:8], dtype, *args[8:], ws, ws_bytes, NULL))

    for call in (forward, backward):
        for bad in (dict(batch=0), dict(n_q_heads=0), dict(n_kv_heads=0), dict(seq_len=0), dict(max_positions=0), dict(eps=-1.0),
                    dict(eps=float("nan")), dict(eps=float("inf")), dict(w_dtype=7)):
            assert call(_changed(good, **bad)) == "PA_ERR_INVALID_ARG", bad
        for bad in (dict(head_dim=96), dict(rotary_dim=132), dict(rotary_dim=-8), dict(rotary_dim=24), dict(n_q_heads=70000),
                    dict(seq_len=1 << 40), dict(q=b.pa_strides(0, -8, 128))):
            assert call(_changed(good, **bad)) == "PA_ERR_SHAPE", bad
        assert call(_changed(good, k=b.pa_strides(0, 516, 128))) == "PA_ERR_ALIGNMENT"
        assert call(None) == "PA_ERR_INVALID_ARG"
        for at in range(8):
            assert call(_changed(good), at) == "PA_ERR_INVALID_ARG", at
        for at in (0, 1, 2, 3, 4, 6, 7):
            assert call(_changed(good), at, P + 8) == "PA_ERR_ALIGNMENT", at
        assert call(_changed(good), 5, P + 2) == "PA_ERR_ALIGNMENT"
    for bad in (b.pa_strides(0, 512, 0), b.pa_strides(0, 64, 128)):     # rows written over one another
        assert forward(_changed(good, q_out=bad)) == "PA_ERR_SHAPE"
    assert forward(_changed(good, batch=2, k_out=b.pa_strides(0, 512, 128))) == "PA_ERR_SHAPE"
    assert backward(_changed(good), dtype=9) == "PA_ERR_INVALID_ARG"
    for at in range(8, 12):
        assert backward(_changed(good), at) == "PA_ERR_INVALID_ARG", at
    assert backward(_changed(good), 10, P + 2) == "PA_ERR_ALIGNMENT"
    assert backward(_changed(good), ws=0) == backward(_changed(good), ws_bytes=100) == "PA_ERR_WORKSPACE"
    assert backward(_changed(good), ws=P + 4) == "PA_ERR_ALIGNMENT"
    assert b.lib.pa_qk_norm_rope_backward_workspace_bytes(_changed(good)) == 25 * 2 * 128 * 4   # CTAs of eight warps, two warps a token


def test_rope_refuses_outputs_whose_rows_overlap(b):
    """Heads that share a number, whichever axes' strides have them do so; heads that interleave without sharing any are none of
    these.  (A null array stops the calls that are not refused: it is looked at next.)"""
    s, o = b.pa_strides(0, 512, 128), b.pa_strides(1 << 20, 512, 128)

    def status(out, which="q_out", **kv):
        good = b.pa_rope_params(1, 4, 2, 128, 100, 128, 0, 100, 1e-6, b.PA_BF16, s, s, o, o)
        args = [0] + [P] * 7
        return b.pa_status_string(b.lib.pa_qk_norm_rope(_changed(good, **{which: b.pa_strides(*out)}, **kv), *args, NULL))

    assert status((1 << 20, 512, 128)) == status((0, 512, 128)) == "PA_ERR_INVALID_ARG"        # (one batch entry: its stride is not used)
    for out in ((0, 128, 128), (0, 384, 128), (0, 128, 12672), (0, 256, 97 * 256)):   # head h + 1 of a token is head h of another
        assert status(out) == "PA_ERR_SHAPE", out
    for out in ((128, 512, 128), (51072, 512, 128), (512, 512, 128)):
        assert status(out, batch=2) == "PA_ERR_SHAPE", out
    assert status((0, 128, 128), "k_out") == status((512, 512, 128), "k_out", batch=2) == "PA_ERR_SHAPE"
    assert status((51200, 512, 128), batch=2) == status((512, 1024, 128), batch=2) == status((512, 1024, 128), "k_out", batch=2, n_kv_heads=4) == "PA_ERR_INVALID_ARG"
    assert status((0, 128, 12800)) == status((0, 256, 128), n_q_heads=2) == status((0, 256, 97 * 256 + 128)) == "PA_ERR_INVALID_ARG"   # (between others)
    assert status((1 << 62, 1 << 62, 1 << 62), batch=2) == "PA_ERR_SHAPE"                       # (nor beyond 64 bits)
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        sizes = [rng.randint(1, 3), rng.randint(1, 5), rng.randint(1, 4)]
        strides = [8 * rng.randint(0, 60 if rng.random() < 0.5 else 20) for _ in sizes]
        at = sorted(x * strides[0] + y * strides[1] + z * strides[2] for x in range(sizes[0]) for y in range(sizes[1]) for z in range(sizes[2]))
        overlap = any(v - u < 64 for u, v in zip(at, at[1:]))
        seen[overlap] += 1
        got = status(strides, batch=sizes[0], seq_len=sizes[1], n_q_heads=sizes[2], head_dim=64, rotary_dim=64)
        assert got == ("PA_ERR_SHAPE" if overlap else "PA_ERR_INVALID_ARG"), (sizes, strides)
    assert min(seen.values()) > 500


def test_kv4_refusals(b):
    assert b.pa_kv4_page_bytes(128) == 9216 and b.pa_kv4_page_bytes(64) == 4608 and b.pa_kv4_page_bytes(96) == 0
    good = b.pa_kv4_pool(4, 128, 64, 10, 4 * 9216, 9216)
    s = b.pa_strides(0, 512, 128)

    def append(p, n=5, k=P, v=P, ks=s, pool=P, slots=P):
        return b.pa_status_string(b.lib.pa_kv4_append(p, n, k, v, ks, s, pool, slots, NULL))

    def read(p, n=5, pool=P, slots=P, k=P, v=P, dtype=b.PA_F32):
        return b.pa_status_string(b.lib.pa_kv4_read(p, n, pool, slots, k, v, dtype, NULL))

    for call in (append, read):
        for bad in (dict(n_kv_heads=0), dict(n_pages=0)):
            assert call(_changed(good, **bad)) == "PA_ERR_INVALID_ARG", bad
        for bad in (dict(head_dim=96), dict(block=32), dict(n_kv_heads=70000), dict(head_stride=9200), dict(page_stride=0)):
            assert call(_changed(good, **bad)) == "PA_ERR_SHAPE", bad
        assert call(_changed(good, head_stride=9224)) == "PA_ERR_ALIGNMENT"
        for bad in (dict(page_stride=9216), dict(page_stride=4 * 9216 - 16), dict(head_stride=10 * 9216 - 16, page_stride=9216)):   # records over one another
            assert call(_changed(good, **bad)) == "PA_ERR_SHAPE", bad
        assert call(None) == call(_changed(good), n=-1) == "PA_ERR_INVALID_ARG"
        assert call(_changed(good), n=0) == "PA_OK"                      # nothing to do, nothing launched
        assert call(_changed(good), n=1 << 50) == "PA_ERR_SHAPE"
        for name in ("k", "v", "pool"):
            assert call(_changed(good), **{name: 0}) == "PA_ERR_INVALID_ARG"
            assert call(_changed(good), **{name: P + 4}) == "PA_ERR_ALIGNMENT"
        assert call(_changed(good), slots=0) == "PA_ERR_INVALID_ARG"
        assert call(_changed(good), slots=P + 4) == "PA_ERR_ALIGNMENT"
    assert append(_changed(good), ks=b.pa_strides(0, 516, 128)) == "PA_ERR_ALIGNMENT"
    assert append(_changed(good), ks=b.pa_strides(0, -512, 128)) == "PA_ERR_SHAPE"
    assert read(_changed(good), dtype=3) == "PA_ERR_INVALID_ARG"


def test_decode_kv4_refusals(b):
    good = b.pa_kv4_params(2, 28, 5, 1, 64, 0.0, b.PA_BF16, b.pa_kv4_pool(4, 128, 64, 10, 4 * 9216, 9216))

    def status(p, at=None, value=0, ws=P, ws_bytes=10 ** 7):
        args = [P] * 6
        if at is not None:
            args[at] = value
        return b.pa_status_string(b.lib.pa_decode_kv4(p, *args, ws, ws_bytes, NULL))

    for bad in (dict(batch=0), dict(n_q_heads=0), dict(max_blocks_per_seq=0), dict(window_blocks=-1), dict(sink_blocks=-1),
                dict(o_dtype=5), dict(softmax_scale=-1.0), dict(softmax_scale=float("inf")), dict(softmax_scale=float("nan")),
                dict(n_pages=0), dict(n_kv_heads=0)):
        assert status(_changed(good, **bad)) == "PA_ERR_INVALID_ARG", bad
        assert b.lib.pa_decode_kv4_workspace_bytes(_changed(good, **bad)) == 0
    for bad in (dict(n_q_heads=30), dict(n_q_heads=36), dict(head_dim=80), dict(block=16), dict(max_blocks_per_seq=1 << 25),
                dict(batch=70000), dict(window_blocks=5000), dict(sink_blocks=5000), dict(head_stride=9000)):
        assert status(_changed(good, **bad)) == "PA_ERR_SHAPE", bad
    assert status(_changed(good, page_stride=4 * 9216 + 8)) == "PA_ERR_ALIGNMENT"
    for at in range(6):
        assert status(_changed(good), at) == "PA_ERR_INVALID_ARG", at
    for at in (0, 1, 4):
        assert status(_changed(good), at, P + 8) == "PA_ERR_ALIGNMENT", at
    for at in (2, 3, 5):
        assert status(_changed(good), at, P + 2) == "PA_ERR_ALIGNMENT", at
    # a status block of 256 bytes, then two parts of rows per CTA: a number, and (o[128], m, l) of eight heads
    want = 256 + 148 * 2 * (4 + 8 * 130) * 4
    assert b.lib.pa_decode_kv4_workspace_bytes(_changed(good)) == want
    # no range is longer than 384 blocks, rounded to whole rows of up to 1 + 5 + 3 blocks
    rows = (148 * (384 - 18) // 9 + 4) // 4
    assert b.lib.pa_decode_kv4_workspace_bytes(_changed(good, batch=rows)) == 256 + 2 * 148 * 2 * (4 + 8 * 130) * 4
    assert status(_changed(good, batch=65535, n_kv_heads=4096, n_q_heads=4096, max_blocks_per_seq=100, head_stride=9216)) == "PA_ERR_SHAPE"
    assert status(_changed(good), ws=0) == status(_changed(good), ws_bytes=want - 1) == "PA_ERR_WORKSPACE"
    assert status(_changed(good), ws=P + 4) == "PA_ERR_ALIGNMENT"


def test_decode_kv4_workspace_from_tensors(b):
    """The size for what the call takes, pools whose axes of one entry have odd strides among them."""
    q, table = torch.zeros((2, 28, 128), dtype=torch.bfloat16), torch.zeros((2, 64), dtype=torch.int32)
    want = 256 + 148 * 2 * (4 + 8 * 130) * 4
    buf = torch.zeros(64 * 9216, dtype=torch.uint8)
    for pool in (buf.view(16, 4, 9216), buf.view(8, 8, 9216)[:, :4], buf.as_strided((1, 4, 9216), (5, 9216, 1)),
                 buf.as_strided((16, 1, 9216), (9216, 7, 1)), buf.as_strided((1, 1, 9216), (1, 3, 1))):
        heads = 28 // pool.shape[1]
        params = b.kv4_params(q if heads <= 8 else q[:, :8], pool, table, 5, 1)
        assert b.pa_decode_kv4_workspace_bytes(params) == want, pool.stride()
        assert params.n_q_heads == (28 if heads <= 8 else 8) and params.o_dtype == b.PA_BF16
    assert b.pa_decode_kv4_workspace_bytes(b.kv4_params(q, buf.view(16, 4, 9216)[:, :3], table, 5, 1)) == 0     # 28 heads on 3
    assert b.kv4_params(q, buf.view(16, 4, 9216), table, 5, 1, 0.5, torch.float32).o_dtype == b.PA_F32


def test_tensors_that_do_not_fit_are_refused(b):
    """From Python: types, shapes, strides, devices (there is nothing on a GPU here)."""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)    # noqa: E731
    q, k, w, cs, pos = bf(5, 4, 64), bf(5, 2, 64), bf(64), torch.zeros(9, 64), i32(5)
    pool, slots = torch.zeros((3, 2, 4608), dtype=torch.uint8), torch.zeros(5, dtype=torch.int64)
    tab = (i32(2), i32(2), i32(7), i32(1), i32(2, 3), 9, 16)

    def swap(args, **kv):
        args = list(args)
        for name, value in kv.items():
            args[int(name[1:])] = value
        return args

    rope = (q, k, w, w, cs, pos)
    cases = [(b.pa_qk_norm_rope, a) for a in (rope, swap(rope, _0=q.float()), swap(rope, _1=bf(4, 2, 64)), swap(rope, _1=bf(5, 2, 128)),
                                              swap(rope, _2=bf(63)), swap(rope, _2=w.float()), swap(rope, _4=cs.double()),
                                              swap(rope, _4=cs.T), swap(rope, _5=pos.long()), swap(rope, _5=i32(4)),
                                              swap(rope, _0=bf(5, 4, 128)[..., ::2]), rope + (q.float(),), rope + (None, bf(5, 3, 64)))]
    cases += [(b.pa_qk_norm_rope_backward, a) for a in (rope + (q, k), rope + (q, k.float()), rope + (q.half(), k.half()),
                                                        rope + (k, q), rope + (q, k, q.float()))]
    cases += [(b.pa_kv4_append, a) for a in ((k, k, pool, slots), (k.float(), k, pool, slots), (k, bf(4, 2, 64), pool, slots),
                                             (k, k, pool[:, :1], slots), (k, k, pool[..., :4600], slots), (k, k, pool.int(), slots),
                                             (k, k, pool, slots.int()), (k, k, pool, slots[:4]), (q, q, pool, slots))]
    cases += [(b.pa_kv4_read, a) for a in ((pool, slots, 64), (pool, slots, 128), (pool, slots.int(), 64), (pool, slots, 1 << 33),
                                           (pool, slots, 64, k.half(), k.half()), (pool, slots, 64, k, k.float()))]
    dec = (bf(2, 4, 64), pool, i32(2, 3), i32(2), 5, 1)
    cases += [(b.pa_decode_kv4, a) for a in (dec, swap(dec, _0=torch.zeros(2, 4, 64)), swap(dec, _2=i32(3, 3)), swap(dec, _2=i32(3, 2).T),
                                             swap(dec, _3=i32(3)), swap(dec, _3=slots[:2]), swap(dec, _0=bf(2, 4, 128)),
                                             dec + (bf(2, 4, 32),), dec + (bf(2, 4, 64).half(),), dec + (None, i32(2, 4)))]
    cases += [(b.pa_build_block_tables, a) for a in (tab, swap(tab, _0=i32(3)), swap(tab, _1=slots[:2]), swap(tab, _3=i32(2)),
                                                     swap(tab, _4=i32(3, 2).T), swap(tab, _6=-1), tab + (i32(2),), tab + (None, i32(16)))]
    for f, args in cases:
        with pytest.raises(AssertionError):
            f(*args)
    with pytest.raises(OverflowError):
        b.pa_build_block_tables(*swap(tab, _5=1 << 40))
    with pytest.raises(TypeError):
        b.pa_kv4_append(None, k, pool, slots)
