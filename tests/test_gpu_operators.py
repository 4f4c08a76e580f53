"""GPU: block tables, norms with rotation (and gradients), against their plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pa():
    import paper_2503_03588_b200 as pa_

    return pa_


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


# ------------------------------------------------------------------ block tables
def _check_tables(pa, new, cached, free, count, room, n_pages, cap, in_place=False, seed=1):
    rng = np.random.default_rng(seed)
    batch = len(new)
    table = rng.integers(-3, n_pages + 3, (batch, room)).astype(np.int32)   # (entries that stay, some of them no page)
    ref = plain.tables(new, cached, free, count, table, n_pages, cap)
    t, lens, left = _ints(table), _ints(cached), _ints([count])
    out = pa.pa_build_block_tables(_ints(new), lens, _ints(free), left, t, n_pages, cap, lens_out=lens if in_place else None,
                                   free_left=left if in_place else None)
    got = [x.cpu().numpy() for x in out[:5]] + [t.cpu().numpy()]
    for name, a, b in zip(("cu_seqlens", "slot_map", "positions", "lens_out", "free_left", "block_table"), got, ref):
        np.testing.assert_array_equal(a.reshape(np.shape(b)), b, err_msg=name)
    return out


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,cap", [(1, 1), (1, 5), (3, 130), (31, 1000), (700, 900), (1024, 1024), (1024, 1025), (33, 4096), (64, 4097), (1000, 4096), (1024, 9000),
                                       (1025, 100), (2500, 70001), (5, 300000)])
def test_tables(pa, batch, cap, in_place):
    """One and several kernels, turns of 1024 sequences, ragged ends, a padded batch; the stack ends in the middle."""
    rng = np.random.default_rng(batch * 7 + cap)
    for share in (0.3, 1.2):
        new = rng.integers(0, max(2, int(2 * cap * share / batch)), batch)
        cached = np.where(rng.random(batch) < 0.3, 0, rng.integers(0, 700, batch))
        room = int((cached + new).max() + 63) // 64 + 1
        want = int(((cached + new + 63) // 64 - (cached + 63) // 64).sum())
        free = rng.permutation(want + 20).astype(np.int32)
        for count in (want + 20, want // 2, 0):
            _check_tables(pa, new, cached, free, count, room, want + 10, cap, in_place)


def test_tables_of_a_decoding_step(pa):
    """A few tokens each, page boundaries among them; an idle sequence gets nothing; most of the batch is padding."""
    rng = np.random.default_rng(3)
    for batch, cap in ((1000, 1024), (33, 140), (5, 900), (1024, 1000)):
        cached = rng.integers(0, 400, batch)
        _check_tables(pa, rng.integers(-1 if batch > 500 else 0, 2 if batch > 100 else 5, batch), cached, rng.permutation(1100), 1100 if batch < 100 else 6, 8, 1000, cap,
                      in_place=batch % 2 == 0)
    cached = [0, 1, 63, 64, 65, 127, 128, 200]
    _check_tables(pa, [1] * 8, cached, np.arange(50, 70), 20, 5, 100, 8, in_place=True)
    _check_tables(pa, [1, 0, 1, 0, 1, 0, 1, 1], cached, np.arange(50, 70), 2, 5, 100, 64)


def test_tables_refuse_sequences_not_calls(pa):
    """Negative lengths, rows too short, tokens behind the last place, more pages than there are: the others are served."""
    big = 2 ** 31 - 1
    _check_tables(pa, [5, -3, 70, 64, 1], [60, 10, -1, 0, 64], np.arange(9), 9, 2, 50, 300)
    _check_tables(pa, [200, 10, 10], [0, 0, 5], np.arange(30), 30, 2, 50, 300)            # 200 tokens need four pages
    _check_tables(pa, [100, 250, 100], [0, 0, 63], np.arange(30), 30, 8, 50, 300)         # the second ends behind 300
    _check_tables(pa, [100, 250, 10], [0, 0, 3], np.arange(30), 5, 8, 50, 400)            # the second finds no pages, the third needs none
    _check_tables(pa, [big, big, 3], [0, 0, 0], np.arange(30), 30, 8, 50, 400)            # sums beyond 31 bits
    _check_tables(pa, [5, big, 3], [0, 0, 0], np.arange(30), 30, 8, 50, 400)
    _check_tables(pa, [3, 3], [big - 2, big - 3], np.arange(30), 30, 8, 50, 400)
    _check_tables(pa, [70, 70], [0, 0], np.arange(3), 99, 8, 50, 400)                     # a height above the stack
    _check_tables(pa, [70, 70], [0, 0], np.arange(3), -4, 8, 50, 400)
    _check_tables(pa, [70, 70], [0, 0], np.zeros(0), 0, 8, 50, 400)
    _check_tables(pa, [0, 0], [0, 64], np.arange(3), 3, 8, 50, 400)


def test_tables_pages_beyond_32_bits(pa):
    """Slots are 64 times the page."""
    n = 2 ** 31 - 1
    out = _check_tables(pa, [130, 70], [10, 0], [n - 1, 5, n - 2, n, 2 ** 26], 5, 4, n, 256)
    assert int(out[1].max()) > 2 ** 36


def test_tables_captured_and_replayed(pa):
    """Decoding steps from one graph, results in place: pages come off the stack, lengths grow, until no page is left."""
    batch, room, n_pages = 5, 4, 12
    lens, left, t = _ints([60, 0, 63, 64, 10]), _ints([9]), _ints(np.tile(np.arange(room), (batch, 1)) + 100)
    new, free = _ints([1, 1, 1, 1, 0]), _ints(np.arange(12) + 3)
    out = pa.pa_build_block_tables(new, lens, free, left, t, 200, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pa.pa_build_block_tables(new, lens, free, left, t, 200, 8, lens_out=lens, free_left=left)
    ref = (lens.tolist(), int(left), t.cpu().numpy())
    for _ in range(210):
        graph.replay()
        cu, slots, positions, l2, f2, t2 = plain.tables([1, 1, 1, 1, 0], ref[0], np.arange(12) + 3, ref[1], ref[2], 200, 8)
        np.testing.assert_array_equal(out[1].cpu().numpy(), slots)
        np.testing.assert_array_equal(out[2].cpu().numpy(), positions)
        ref = (l2, f2, t2)
    assert lens.tolist() == ref[0] and int(left) == ref[1] == 0 and max(ref[0]) < 256
    np.testing.assert_array_equal(t.cpu().numpy(), ref[2])


def test_small_results_do_not_hold_large_ones(pa):
    """Who keeps the stack's height, the lengths or a weight's gradient keeps no slots, no workspace and no other gradients with
    it: large results have storages of their own, the small ones' is small."""
    t, free = _ints(np.full((300, 40), -1)), _ints(np.arange(12000))
    cu, slots, positions, lens, left, ws = pa.pa_build_block_tables(_ints([2000] * 300), _ints([5] * 300), free, _ints([12000]), t, 12000, 600000)
    assert int(left) == 12000 - 300 * 31       # 2005 tokens are 32 pages, one of which each has
    small = {x.untyped_storage().data_ptr() for x in (cu, lens, left, ws)}
    for x in (cu, lens, left, ws):
        assert x.untyped_storage().nbytes() <= 6 * 65536
    for x in (slots, positions):
        assert x.untyped_storage().nbytes() == x.numel() * x.element_size() and x.untyped_storage().data_ptr() not in small
    args = _inputs(200, 8, 2, 128, 128, 15)
    grads = pa.pa_qk_norm_rope_backward(*args, *(torch.randn((200, h, 128)).cuda() for h in (8, 2)))
    assert grads[0].untyped_storage().nbytes() == grads[0].numel() * 2      # 400 KB
    assert grads[2].untyped_storage().nbytes() <= 5 * 65536
    for a, b in ((0, 1), (0, 2), (0, 4)):
        assert grads[a].untyped_storage().data_ptr() != grads[b].untyped_storage().data_ptr()
    out = pa.pa_qk_norm_rope(*args)
    assert out[0].untyped_storage().nbytes() == out[0].numel() * 2


def test_tables_arrays_off_16_bytes(pa):
    """Slots and positions that start on an odd entry."""
    slots, positions = torch.full((200,), 7, dtype=torch.int64).cuda(), torch.full((200,), 7, dtype=torch.int32).cuda()
    t, free = _ints(np.full((2, 3), -1)), _ints(np.arange(6))
    pa.pa_build_block_tables(_ints([70, 60]), _ints([0, 3]), free, _ints([6]), t, 6, 133, slot_map=slots[3:136], positions=positions[1:134])
    ref = plain.tables([70, 60], [0, 3], range(6), 6, np.full((2, 3), -1), 6, 133)
    np.testing.assert_array_equal(slots.cpu().numpy(), np.concatenate(([7] * 3, ref[1], [7] * 64)))
    np.testing.assert_array_equal(positions.cpu().numpy(), np.concatenate(([7], ref[2], [7] * 66)))


# ------------------------------------------------------------------ norms with rotation
def _angles(n, rot):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    return torch.cat((a.cos(), a.sin()), -1).float().cuda()


def _inputs(tokens, hq, hkv, d, rot, seed, w_dtype=torch.bfloat16, n_pos=500):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((tokens, hq + 2 * hkv, d), generator=g).bfloat16().cuda()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(w_dtype).cuda() for _ in range(2)]
    pos = torch.randint(0, n_pos, (tokens,), generator=g, dtype=torch.int32).cuda()
    return qkv[:, :hq], qkv[:, hq:hq + hkv], *w, _angles(n_pos, rot), pos


def _near_bf16(got, ref, size):
    """A rounding to bf16 is at most 2^-8 of the value.  In fp32: the sum of 128 squares 2^-18 of it, its root half that, a
    root, two products and a rotation of two terms a few 2^-24; the means in the backward pass (sums of 128 products of three
    factors) 2^-17 at most: together below 2^-15 of the terms."""
    err = (got.double() - ref).abs()
    bound = ref.abs() * 2.0 ** -8 * 1.01 + size * 2.0 ** -15 + 1e-37
    assert torch.isfinite(got.float()).all()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot", [(28, 4, 128, 128), (2, 2, 64, 64), (7, 1, 128, 64), (5, 3, 64, 48), (3, 1, 128, 0),
                                          (16, 4, 64, 32), (9, 2, 128, 16)])
def test_norm_rope_and_gradients(pa, hq, hkv, d, rot, interleaved):
    for tokens, w_dtype, d_dtype in ((1, torch.bfloat16, torch.float32), (37, torch.float32, torch.bfloat16),
                                     (1003, torch.bfloat16, torch.float32), (1003, torch.float32, torch.bfloat16)):
        args = _inputs(tokens, hq, hkv, d, rot, tokens + hq, w_dtype)
        g = torch.Generator().manual_seed(5)
        back = [torch.randn((tokens, h, d), generator=g).to(d_dtype).cuda() for h in (hq, hkv)]
        out = pa.pa_qk_norm_rope(*args, eps=1e-5, interleaved=interleaved)
        grads = pa.pa_qk_norm_rope_backward(*args, *back, eps=1e-5, interleaved=interleaved)
        for i in range(2):
            ref, size, dx, dxs, dw, dws = plain.norm_rope(args[i], args[2 + i], args[4], args[5], 1e-5, interleaved, back[i])
            _near_bf16(out[i], ref, size)
            _near_bf16(grads[i], dx, dxs)
            # (fp32 sums: at most 1003 x heads / 16 terms one after the other in a lane, 592 CTAs in turns of 32)
            err = (grads[2 + i].double() - dw).abs()
            assert (err <= dws * 2.0 ** -14).all(), float((err / dws).max())


def test_norm_rope_gradient_is_a_difference_quotient(pa):
    """Along a random direction, in the fp64 plain form whose gradients the kernels are held to: (f(x + e u) - f(x - e u)) / 2 e."""
    q, k, wq, wk, cs, pos = _inputs(5, 3, 2, 64, 64, 9)
    g = torch.Generator().manual_seed(6)
    back = torch.randn((5, 3, 64), generator=g).cuda()
    grads = pa.pa_qk_norm_rope_backward(q, k, wq, wk, cs, pos, back, torch.zeros((5, 2, 64)).cuda())
    u, e = torch.randn((5, 3, 64), generator=g).double().cuda(), 1e-5
    f = lambda x, w: float((plain.norm_rope(x, w, cs, pos, 1e-6, False)[0] * back.double()).sum())  # noqa: E731
    quot = (f(q.double() + e * u, wq) - f(q.double() - e * u, wq)) / (2 * e)
    terms = float((grads[0].double() * u).abs().sum())
    assert abs(quot - float((grads[0].double() * u).sum())) <= 2.0 ** -8 * terms
    v = torch.randn(64, generator=g).double().cuda()
    quot = (f(q, wq.double() + e * v) - f(q, wq.double() - e * v)) / (2 * e)
    assert abs(quot - float((grads[2].double() * v).sum())) <= 1e-4 * float((grads[2].double() * v).abs().sum())
    assert (grads[1] == 0).all() and (grads[3] == 0).all()


@pytest.mark.parametrize("tokens", [6, 900])
def test_norm_rope_leaves_tokens_without_a_position_alone(pa, tokens):
    """Positions -1, beyond the table, of the lowest value: the rows of the outputs keep what they hold, whatever the inputs
    (NaN, infinities) are; gradients are zero and nothing is added.  eps = 0."""
    hq, hkv, d = 6, 2, 128
    q, k, wq, wk, cs, pos = _inputs(tokens, hq, hkv, d, 128, 3)
    q, k = q.clone(), k.clone()
    out = torch.arange(tokens)[:, None] % 6
    bad = (out[:, 0] < 3).cuda()
    pos = torch.where(bad, torch.tensor([-1, 500, -2 ** 31], dtype=torch.int32)[out[:, 0].clamp(max=2)].cuda(), pos)
    q[bad], k[bad] = float("nan"), float("inf")
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    pa.pa_qk_norm_rope(q, k, wq, wk, cs, pos, qo, ko, eps=0.0)
    back = [torch.randn((tokens, h, d)).cuda() for h in (hq, hkv)]
    back[0][bad], back[1][bad] = float("nan"), float("-inf")
    grads = pa.pa_qk_norm_rope_backward(q, k, wq, wk, cs, pos, *back, eps=0.0)
    good = ~bad
    for i, (x, o) in enumerate(((q, qo), (k, ko))):
        assert (o[bad] == 7).all() and (grads[i][bad] == 0).all()
        ref, size, dx, dxs, dw, dws = plain.norm_rope(x[good], (wq, wk)[i], cs, pos[good], 0.0, False, back[i][good])
        _near_bf16(o[good], ref, size)
        _near_bf16(grads[i][good], dx, dxs)
        assert ((grads[2 + i].double() - dw).abs() <= dws * 2.0 ** -14).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens", [6, 1300])
def test_gradients_of_tokens_without_a_position_are_zero_whatever_weights_and_angles_are(pa, tokens, interleaved):
    """Infinite and NaN weights; a row of the table that no token is at holds NaN and infinities."""
    hq, hkv, d = 5, 1, 128
    q, k, wq, wk, cs, pos = _inputs(tokens, hq, hkv, d, 64, 14)
    pos.clamp_(min=1)
    bad = torch.zeros(tokens, dtype=torch.bool).cuda()
    bad[::3], bad[-1] = True, True
    pos[bad] = -1
    back = [torch.randn((tokens, h, d)).cuda() for h in (hq, hkv)]
    ref = pa.pa_qk_norm_rope_backward(q, k, wq, wk, cs, pos, *back, interleaved=interleaved)
    cs[0, ::2], cs[0, 1::2] = float("nan"), float("inf")
    got = pa.pa_qk_norm_rope_backward(q, k, wq, wk, cs, pos, *back, interleaved=interleaved)
    for a, b in zip(got[:4], ref):
        assert torch.equal(a, b)
    wq[3], wk[70], wk[127] = float("inf"), float("nan"), float("-inf")
    got = pa.pa_qk_norm_rope_backward(q, k, wq, wk, cs, pos, *back, interleaved=interleaved)
    assert (got[0][bad] == 0).all() and (got[1][bad] == 0).all()
    for a, b in zip(got[2:4], ref[2:4]):      # (the weights' gradients do not depend on the weights)
        assert torch.equal(a, b)


def test_norm_rope_strides_batches_and_in_place(pa):
    """[batch, N, H, D] views with gaps, a head axis inside out, expanded inputs, outputs over the inputs."""
    b, n, hq, hkv, d = 2, 33, 4, 2, 128
    g = torch.Generator().manual_seed(8)
    big = torch.randn((b, hq, n + 3, d + 8), generator=g).bfloat16().cuda()
    q = big[:, :, :n, :d].transpose(1, 2)                       # [b, n, hq, d], heads far apart
    k = torch.randn((1, 1, hkv, d), generator=g).bfloat16().cuda().expand(b, n, hkv, d)
    w, cs = torch.randn((2, d), generator=g).cuda(), _angles(90, d)
    pos = torch.randint(0, 90, (b, n), generator=g, dtype=torch.int32).cuda()
    flat = lambda x: x.reshape(b * n, -1, d)  # noqa: E731
    ref = [plain.norm_rope(flat(x), w[i], cs, pos.reshape(-1), 1e-6, False) for i, x in enumerate((q, k))]
    kept = big.clone()
    qo, ko = pa.pa_qk_norm_rope(q, k, w[0], w[1], cs, pos, q_out=q)
    assert qo is q
    _near_bf16(flat(qo), *ref[0])
    _near_bf16(flat(ko), *ref[1])
    kept[:, :, :n, :d] = big[:, :, :n, :d]
    assert torch.equal(kept, big)                               # (nothing beside the view was written)
    dq = torch.randn((b, n, 1, d), generator=g).cuda().expand(b, n, hq, d)   # one gradient for all heads
    grads = pa.pa_qk_norm_rope_backward(q, k, w[0], w[1], cs, pos, dq, torch.randn((b, n, hkv, d), generator=g).cuda())
    dx, dxs = plain.norm_rope(flat(q), w[0], cs, pos.reshape(-1), 1e-6, False, flat(dq))[2:4]
    _near_bf16(flat(grads[0]), dx, dxs)


def test_norm_rope_large_and_small_values(pa):
    """Heads of 1e18, of 1e-18 (eps decides) and of zeros."""
    q, k, wq, wk, cs, pos = _inputs(9, 4, 2, 64, 64, 11)
    q = q.float()
    q[:, 0] *= 1e18
    q[:, 1] *= 1e-18
    q[:, 2] = 0
    q = q.bfloat16()
    out = pa.pa_qk_norm_rope(q, k, wq, wk, cs, pos)
    _near_bf16(out[0], *plain.norm_rope(q, wq, cs, pos, 1e-6, False))
    assert (out[0][:, 2] == 0).all()


def test_gradients_are_the_same_every_time(pa):
    args = _inputs(5000, 28, 4, 128, 128, 12)
    back = [torch.randn((5000, h, 128)).cuda() for h in (28, 4)]
    first = pa.pa_qk_norm_rope_backward(*args, *back)
    again = pa.pa_qk_norm_rope_backward(*args, *back, workspace=first[4].fill_(255))
    for a, b in zip(first[:4], again[:4]):
        assert torch.equal(a, b)


def test_norm_rope_captured_and_replayed(pa):
    """Forward and backward in a graph, on another stream, with new values behind the same addresses."""
    args = _inputs(300, 8, 2, 128, 128, 13)
    back = [torch.randn((300, h, 128)).cuda() for h in (8, 2)]
    ws = pa.pa_qk_norm_rope_backward(*args, *back)[4]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = pa.pa_qk_norm_rope(*args)
        grads = pa.pa_qk_norm_rope_backward(*args, *back, workspace=ws)
    args[0].copy_(torch.randn_like(args[0]))
    back[0].mul_(3)
    graph.replay()
    torch.cuda.synchronize()
    ref_out, ref = pa.pa_qk_norm_rope(*args), pa.pa_qk_norm_rope_backward(*args, *back)
    for a, b in zip((*out, *grads[:4]), (*ref_out, *ref[:4])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot", [(28, 4, 128, 128), (16, 4, 64, 32), (5, 3, 64, 48), (9, 2, 128, 16), (3, 1, 128, 0)])
def test_norm_rope_many_tokens(pa, hq, hkv, d, rot, interleaved):
    """Enough tokens for warps that stride over them, in two uneven shares: a batch of views into a projection's output, the
    queries in place; tokens without a position among them keep what they hold, NaN and infinities too."""
    n = 148 * 112 * 256 // d // (hq + hkv) // 2 + 1201
    g = torch.Generator().manual_seed(21)
    qkv = torch.randn((2, n, hq + 2 * hkv, d), generator=g).bfloat16().cuda()
    _, _, wq, wk, cs, _ = _inputs(1, hq, hkv, d, rot, 22)
    pos = torch.randint(0, cs.shape[0], (2, n), generator=g, dtype=torch.int32).cuda()
    bad = (torch.rand((2, n), generator=g) < 0.1).cuda()
    bad[:, -3:] = True
    pos[bad] = torch.tensor([-1, cs.shape[0], -2 ** 31, 2 ** 31 - 1], dtype=torch.int32).cuda().repeat(n)[:int(bad.sum())]
    qkv[bad] = float("nan")
    qkv[0, -3:] = float("inf")
    before = qkv.clone()
    q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv]
    ko = torch.full((2, n, hkv, d), 7.0, dtype=torch.bfloat16).cuda()
    pa.pa_qk_norm_rope(q, k, wq, wk, cs, pos, q_out=q, k_out=ko, eps=1e-5, interleaved=interleaved)
    good = ~bad
    for i, (x, out) in enumerate(((before[:, :, :hq], q), (before[:, :, hq:hq + hkv], ko))):
        _near_bf16(out[good], *plain.norm_rope(x[good], (wq, wk)[i], cs, pos[good], 1e-5, interleaved))
    assert (ko[bad] == 7).all()
    assert torch.equal(q[bad].view(torch.int16), before[:, :, :hq][bad].view(torch.int16))
    assert torch.equal(qkv[:, :, hq:].view(torch.int16), before[:, :, hq:].view(torch.int16))


def test_axes_of_one_entry_have_any_stride(pa):
    """One token, one head, one batch entry: the strides of their axes are never used."""
    g = torch.Generator().manual_seed(23)
    x = torch.randn(4096, generator=g).bfloat16().cuda()
    wq, wk, cs, pos = _inputs(1, 1, 1, 64, 64, 24)[2:]
    odd = x.as_strided((1, 1, 1, 64), (3, 5, 7, 1))
    out = pa.pa_qk_norm_rope(odd, odd, wq, wk, cs, pos)
    ref = pa.pa_qk_norm_rope(odd.contiguous().view(1, 1, 64), odd.contiguous().view(1, 1, 64), wq, wk, cs, pos)
    assert torch.equal(out[0].flatten(), ref[0].flatten()) and torch.equal(out[1].flatten(), ref[1].flatten())


def test_calls_on_two_streams_at_once(pa):
    """Tables, norms and gradients on two streams, each call with a workspace of its own, many times."""
    args = [_inputs(3000, 8, 2, 128, 128, 30 + i) for i in range(2)]
    back = [torch.randn((3000, h, 128)).cuda() for h in (8, 2)]
    new, cached = _ints([40] * 500), _ints([100] * 500)
    free, count = _ints(np.arange(1000)), _ints([900])
    tables = lambda i: pa.pa_build_block_tables(new, cached, free[i:], count, torch.full((500, 4), -1, dtype=torch.int32).cuda(), 1000, 20000)  # noqa: E731
    call = lambda i: (*pa.pa_qk_norm_rope(*args[i]), *pa.pa_qk_norm_rope_backward(*args[i], *back)[:4], *tables(i)[:5])  # noqa: E731
    ref = [[x.clone() for x in call(i)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, call(i)))
    torch.cuda.synchronize()
    for i, outs in got:
        for a, b in zip(outs, ref[i]):
            assert torch.equal(a, b)
