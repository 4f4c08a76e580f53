"""GPU: the 4-bit cache (append, read) and the decode over it, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pa():
    import paper_2503_03588_b200 as pa_

    return pa_


def _randn(*shape, seed=0, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16()


def _pool(pa, pages, heads, d, fill=0):
    return torch.full((pages, heads, pa.pa_kv4_page_bytes(d)), fill, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ append, read
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (7, 4), (300, 3), (5000, 2)])
def test_append_and_read(pa, tokens, heads, d):
    """Values, and the bytes as the header lays them out, to the last bit; slots in any order, some of them none; what else the
    pool holds stays."""
    pages = tokens // 64 + 3
    kv = _randn(tokens, 2 * heads, d, seed=tokens).cuda()
    kv[:, 0] *= 100.0
    k, v = kv[:, :heads], kv[:, heads:]
    slots = torch.randperm(pages * 64, generator=torch.Generator().manual_seed(2))[:tokens].cuda()
    if tokens > 5:
        slots[3], slots[4], slots[5] = -1, pages * 64, -2 ** 40
    good = (slots >= 0) & (slots < pages * 64)
    pool = _pool(pa, pages, heads, d, 0x5A)
    before = plain.page_values(pool, d)
    pa.pa_kv4_append(k, v, pool, slots)
    ref = [torch.where(good[:, None, None], plain.held(x), torch.zeros((), dtype=torch.float64, device="cuda")) for x in (k, v)]
    for got, r in zip(pa.pa_kv4_read(pool, slots, d, dtype=torch.float32), ref):
        assert torch.equal(got.double(), r)
    for got, r in zip(pa.pa_kv4_read(pool, slots, d), ref):
        assert torch.equal(got, r.float().bfloat16())      # (a product of 8 and 4 bits is exact in fp32)
    for now, was, r in zip(plain.page_values(pool, d), before, ref):
        at = slots[good].cpu()
        was[at // 64, :, at % 64] = r[good].cpu()
        assert torch.equal(now, was)
    assert pool.shape[2] == 72 * d


def test_append_ties_zeros_and_wild_values(pa):
    """Values in the middle of two steps go to zero's side; groups below 2^-100 are zeros; NaN and infinities make their group
    NaN and no other; the largest and smallest finite numbers."""
    d = 64
    x = torch.zeros((8, 2, d))
    x[0, 0, :16] = torch.arange(16) * 0.5 - 4       # s = 1 for a largest of 7: halves are ties
    x[0, 0, 20] = 7
    x[0, 1, 32:] = 2.0 ** -101
    x[1, 0, 0], x[1, 0, 40] = float("nan"), 1.0
    x[2, 1, 5], x[2, 1, 50] = float("-inf"), -3.0
    x[3, 0, :] = 3e38
    x[4, 0, :32], x[4, 0, 7] = 2.0 ** -100, 2.0 ** -99
    x[5, 1] = torch.linspace(-1, 1, d)
    x[6, 0, 3] = -5.5
    x = x.bfloat16().cuda()
    pool, slots = _pool(pa, 2, 2, d, 0xFF), torch.arange(60, 68).cuda()
    pa.pa_kv4_append(x, x.flip(2), pool, slots)
    k, v = pa.pa_kv4_read(pool, slots, d, dtype=torch.float32)
    for got, src in ((k, x), (v, x.flip(2))):
        assert torch.equal(torch.nan_to_num(got.double(), nan=1e9), torch.nan_to_num(plain.held(src), nan=1e9))
    assert torch.equal(k[0, 0, :16].cpu(), torch.tensor([-4., -3, -3, -2, -2, -1, -1, 0, 0, 0, 1, 1, 2, 2, 3, 3]))
    assert torch.isnan(k[1, 0, :32]).all() and (k[1, 0, 32:] != 0).sum() == 1


def test_every_quotient_of_two_mantissas(pa):
    """All pairs of 8-bit mantissas of a number and its group's largest, over the exponents that matter: the nearest step."""
    top = torch.arange(128, 256).float()
    x = torch.zeros((128 * 5, 1, 128))
    vals = torch.arange(128, 256).float()
    for e in range(5):                    # numbers 0 .. 4 octaves below; a row holds four groups of 31 numbers and the largest
        for i in range(128):
            y = torch.cat((vals * 2.0 ** -e, torch.zeros(0))).clamp(max=float(top[i]))
            rows = y.unflatten(0, (4, 32)).clone()
            rows[:, 31] = top[i]
            x[e * 128 + i, 0] = rows.flatten()
    x = x.bfloat16().cuda()
    pool, slots = _pool(pa, 10, 1, 128), torch.arange(640).cuda()
    pa.pa_kv4_append(x, -x, pool, slots)
    k, v = pa.pa_kv4_read(pool, slots, 128, dtype=torch.float32)
    assert torch.equal(k.double(), plain.held(x)) and torch.equal(v, -k)


def test_every_quotient_with_no_numerator_left_out(pa):
    """All 128 mantissas of a number against all 128 of its group's largest, 0 to 4 octaves below it: 16 numbers and the largest a
    group, eight groups in two heads."""
    vals = torch.arange(128, 256).float()
    x = torch.zeros((5, 128, 2, 4, 32))
    for e in range(5):
        for i in range(128):
            x[e, i, :, :, :16] = (vals * 2.0 ** -e).clamp(max=float(vals[i])).reshape(2, 4, 16)
    x[..., 31] = vals[None, :, None, None]
    x = x.reshape(640, 2, 128).bfloat16().cuda()
    below = x.view(5, 128, 8, 32)[1:, :, :, :16].reshape(4, 128, 128)
    assert torch.equal(below[3].double() * 16, vals.double().cuda().expand(128, 128))   # (none has been replaced)
    pool, slots = _pool(pa, 10, 2, 128), torch.arange(640).cuda()
    pa.pa_kv4_append(x, -x, pool, slots)
    k, v = pa.pa_kv4_read(pool, slots, 128, dtype=torch.float32)
    assert torch.equal(k.double(), plain.held(x)) and torch.equal(v, -k)


def test_append_strided_pool_and_tensors(pa):
    """A layer's part of a pool of all layers; heads that lie far apart; expanded values; no tokens at all."""
    d, heads = 64, 3
    record = pa.pa_kv4_page_bytes(d)
    everything = torch.full((9, 5, heads, record), 1, dtype=torch.uint8, device="cuda")
    pool = everything[:, 2]
    k = _randn(heads, 100, d + 8, seed=3).cuda()[..., :d].transpose(0, 1)
    v = _randn(1, heads, d, seed=4).cuda().expand(100, heads, d)
    slots = torch.arange(100, 200).cuda()
    kept = everything.clone()
    pa.pa_kv4_append(k, v, pool, slots)
    got = pa.pa_kv4_read(pool, slots, d, dtype=torch.float32)
    assert torch.equal(got[0].double(), plain.held(k)) and torch.equal(got[1].double(), plain.held(v))
    kept[:, 2] = pool
    assert torch.equal(kept, everything)
    pa.pa_kv4_append(k[:0], v[:0], pool, slots[:0])
    assert pa.pa_kv4_read(pool, slots[:0], d)[0].shape == (0, heads, d)
    torch.cuda.synchronize()


def test_pool_beyond_32_bits_of_bytes(pa):
    """A page 5 GB behind the pool's start, for append, read and decode."""
    d, heads = 128, 1
    record = pa.pa_kv4_page_bytes(d)
    pages = 5 * 2 ** 30 // record
    pool = torch.empty((pages, heads, record), dtype=torch.uint8, device="cuda")
    k, v = _randn(70, heads, d, seed=5).cuda(), _randn(70, heads, d, seed=6).cuda()
    table = torch.tensor([[pages - 1, pages - 7]], dtype=torch.int32, device="cuda")
    slots = torch.cat((torch.arange(64) + (pages - 1) * 64, torch.arange(6) + (pages - 7) * 64)).cuda()
    pa.pa_kv4_append(k, v, pool, slots)
    got = pa.pa_kv4_read(pool, slots, d, dtype=torch.float32)
    assert torch.equal(got[0].double(), plain.held(k)) and torch.equal(got[1].double(), plain.held(v))
    q = _randn(1, 3, d, seed=7).cuda()
    o, lse, _ = pa.pa_decode_kv4(q, pool, table, torch.tensor([70], dtype=torch.int32, device="cuda"), 5, 1, o_dtype=torch.float32)
    ref = plain.row_attention(q[0].double(), plain.held(k)[:, 0], plain.held(v)[:, 0], d ** -0.5)
    _near(o[0], lse[0], ref, torch.float32)


# ------------------------------------------------------------------ decode
def _near(o, lse, ref, o_dtype):
    """ref: O, LSE, A = sum p |v|, L = the largest sum of |q k| (scaled) of a row's logits.
    A logit: exact products, 128 of them summed in fp32 (tensor cores: at most 2^-23 of the running sum a step, of the terms'
    sum L 2^-18 at most, taken as 2^-19 L over the four groups' chains of eight), scales and factors 2^-22 L: its weight is off by
    that in relative terms, plus ex2.approx and the sums of weights (4 x 2^-22 and 2^-19).  Twice for the quotient.  Weights for bf16 outputs
    are rounded to bf16, 2^-8, and times their scale once more, (1 + 2^-8)^2 - 1 < 2^-7 + 2^-15; for fp32 outputs in two parts, 2^-16.  The output's rounding: 2^-8."""
    ref_o, ref_lse, size, most = (x.to(o.device) for x in ref)
    logit = 2.0 ** -18 * most + 2.0 ** -18
    assert ((lse.double() - ref_lse).abs() <= logit + ref_lse.abs() * 2.0 ** -22).all(), float(((lse.double() - ref_lse).abs() / logit).max())
    weight = 2 * logit + (2.0 ** -7 + 2.0 ** -15 if o_dtype == torch.bfloat16 else 2.0 ** -16)
    bound = weight[:, None] * size + (ref_o.abs() * 2.0 ** -8 if o_dtype == torch.bfloat16 else 0) + 1e-30
    err = (o.double() - ref_o).abs()
    assert torch.isfinite(o.float()).all()
    assert (err <= bound).all(), float((err / bound).max())


class _Cache:
    """Sequences of the given lengths in scrambled pages; what lies behind a length is 0xFF bytes (NaN scales)."""

    def __init__(self, pa, lens, heads, d, seed=0, k_scale=1.0, v_scale=1.0, room=0):
        self.pa, self.lens, self.heads, self.d = pa, list(lens), heads, d
        blocks = [(max(n, 0) + 63) // 64 for n in self.lens]
        pages = sum(blocks) + 2
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
        self.pool = _pool(pa, pages, heads, d, 0xFF)
        room = max(room, max(blocks), 1)
        table = torch.full((len(blocks), room), -1, dtype=torch.int32)
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(self.lens):
            table[b, :blocks[b]] = order[at:at + blocks[b]]
            at += blocks[b]
            if n <= 0:
                self.k.append(None), self.v.append(None)
                continue
            k, v = _randn(n, heads, d, seed=100 * seed + 2 * b, scale=k_scale).cuda(), _randn(n, heads, d, seed=100 * seed + 2 * b + 1, scale=v_scale).cuda()
            i = torch.arange(n)
            pa.pa_kv4_append(k, v, self.pool, (table[b, i // 64].long() * 64 + i % 64).cuda())
            self.k.append(plain.held(k)), self.v.append(plain.held(v))
        self.table = table.cuda()
        self.lens_d = torch.tensor(self.lens, dtype=torch.int32).cuda()

    def check(self, oracle, hq, W, S, o_dtype=torch.bfloat16, scale=0.0, seed=1, q_scale=1.0, **kw):
        q = _randn(len(self.lens), hq, self.d, seed=seed, scale=q_scale).cuda()
        o, lse, ws = self.pa.pa_decode_kv4(q, self.pool, self.table, self.lens_d, W, S, softmax_scale=scale, o_dtype=o_dtype, **kw)
        self.pa.pa_decode_status(ws)
        for b, n in enumerate(self.lens):
            if n <= 0:
                assert (o[b] == 0).all() and (lse[b] == float("-inf")).all()
                continue
            j = torch.as_tensor(np.asarray(oracle.block_row((n - 1) // 64, W, S))).long()
            keys = (j[:, None] * 64 + torch.arange(64)).flatten()
            keys = keys[keys < n].cuda()
            for h in range(self.heads):
                g = slice(h * hq // self.heads, (h + 1) * hq // self.heads)
                ref = plain.row_attention(q[b, g].double(), self.k[b][keys, h], self.v[b][keys, h], scale or self.d ** -0.5)
                _near(o[b, g], lse[b, g], ref, o_dtype)
        return q, o, lse, ws


@pytest.mark.parametrize("o_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (8, 1, 64), (2, 2, 64), (5, 1, 128), (16, 4, 64), (3, 3, 128)])
def test_decode_kv4(pa, oracle, hq, hkv, d, o_dtype):
    """Lengths around the edges of a warp's 16 keys and of a block; windows that cover all, default ones, none."""
    c = _Cache(pa, [1, 2, 15, 16, 17, 63, 64, 65, 81, 130, 1000, 2049], hkv, d, seed=hq)
    c.check(oracle, hq, 5, 1, o_dtype)
    c.check(oracle, hq, 0, 0, o_dtype, scale=0.21)
    c.check(oracle, hq, 60, 2, o_dtype)


@pytest.mark.parametrize("env", [{}] + [{"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": str(r)} for r in range(1, 9)] +
                         [{"PA_DECODE_PATH": "persist"}] +
                         [{"PA_DECODE_PATH": "cluster", "PA_DECODE_STAGES": s, "PA_DECODE_CLUSTER": r} for s in ("1", "2", "5") for r in ("1", "4")])
@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 128), (4, 1, 64)])
def test_decode_kv4_forms(pa, oracle, pa_env, hq, hkv, d, env):
    """Both kernels, several CTAs per row and ring depths; lengths outside the table among the sequences."""
    pa_env(**env)
    c = _Cache(pa, [9000, 8193, 0, 130, 7, -5], hkv, d, seed=3, k_scale=2.0)
    c.check(oracle, hq, 5, 1)
    c.check(oracle, hq, 30, 2, torch.float32)


def test_decode_kv4_length_beyond_the_table(pa):
    c = _Cache(pa, [100, 64], 2, 64)
    c.lens_d[0] = 129
    q = _randn(2, 4, 64).cuda()
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    assert (o[0] == 0).all() and (lse[0] == float("-inf")).all() and torch.isfinite(lse[1]).all()


def test_decode_kv4_many_rows(pa, oracle, pa_env):
    """Equal ranges: warps with many rows, rows in several warps and CTAs, ranges beyond a block per thread, few blocks for
    all CTAs, more sequences than threads, sequences without a key in between."""
    lens = [int(x) for x in np.random.default_rng(4).integers(1, 1500, 150)]
    c = _Cache(pa, lens, 4, 64, seed=5)
    c.check(oracle, 16, 5, 1)
    c = _Cache(pa, lens, 4, 128, seed=6)
    c.check(oracle, 28, 9, 1, torch.float32)
    pa_env(PA_DECODE_PATH="persist")
    c = _Cache(pa, lens[:40], 1, 64, seed=14)
    c.check(oracle, 1, 5, 1)
    c = _Cache(pa, [300, 0, 64, 1, -1, 129], 1, 128, seed=15)
    c.check(oracle, 8, 5, 1, torch.float32)
    c = _Cache(pa, [0, 0], 2, 64, seed=16)
    c.check(oracle, 8, 5, 1)
    short = [int(x) for x in np.random.default_rng(5).integers(-20, 200, 1000)]
    c = _Cache(pa, short, 1, 64, seed=17)
    c.check(oracle, 3, 5, 1)
    c = _Cache(pa, [1] * 500 + [6000] + [1] * 300, 2, 64, seed=18)
    c.check(oracle, 8, 4096, 1, torch.float32)
    for hq, hkv, d in ((14, 2, 128), (16, 4, 64)):   # rows of up to 60 blocks, of one, without a key
        lens = [int(x) for x in np.random.default_rng(7).integers(1, 4000, 90)]
        lens[3:6] = [0, 1, 64]
        lens[-1] = -7
        c = _Cache(pa, lens, hkv, d, seed=19)
        c.check(oracle, hq, 40, 2)
        c = _Cache(pa, [1] * 70 + [3000] + [64] * 80, hkv, d, seed=20)
        c.check(oracle, hq, 60, 1)


def test_decode_kv4_long_rows_of_few_sequences(pa, oracle):
    """A window of 4096 blocks over 70000 tokens: a row in all CTAs."""
    c = _Cache(pa, [70001], 1, 128, seed=7)
    c.check(oracle, 7, 4096, 0, torch.float32)
    c.check(oracle, 7, 4096, 0)
    c = _Cache(pa, [30000, 700, 21001], 2, 64, seed=8)
    c.check(oracle, 4, 300, 5)


@pytest.mark.parametrize("k_scale,v_scale,q_scale", [(4.0, 1.0, 1.0), (1.0, 1e-12, 1.0), (1.0, 1e20, 1.0), (1e-20, 1.0, 1e20), (1e18, 1.0, 1e-18),
                                                     (1.0, 1e-29, 3.0), (1e-30, 1.0, 1.0)])
def test_decode_kv4_magnitudes(pa, oracle, k_scale, v_scale, q_scale):
    """Queries, keys and values far from 1: the fp16 queries are scaled by powers of two."""
    c = _Cache(pa, [500, 2000], 2, 128, seed=9, k_scale=k_scale, v_scale=v_scale)
    c.check(oracle, 8, 5, 1, torch.float32, q_scale=q_scale)
    c.check(oracle, 8, 5, 1, q_scale=q_scale)


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "3"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 128), (4, 1, 64)])
def test_decode_kv4_weights_lose_less_than_the_output(pa, oracle, pa_env, hq, hkv, d, env):
    """bf16 outputs are off by their own rounding, 2^-8 of them, and little else.  A weight in two bf16 parts is off by 2^-16, its
    product with a scale once more by 2^-15 (the second part holds 2^-7 of it at most): below 2^-14 of the terms, and what the
    logits' errors make of it (as in _near)."""
    pa_env(**env)
    c = _Cache(pa, [2, 9, 30, 64, 200, 1000], hkv, d, seed=26, k_scale=2.0)
    q, o, lse, _ = c.check(oracle, hq, 5, 1)
    for b, n in enumerate(c.lens):
        j = torch.as_tensor(np.asarray(oracle.block_row((n - 1) // 64, 5, 1))).long()
        i = (j[:, None] * 64 + torch.arange(64)).flatten()
        i = i[i < n].cuda()
        for h in range(hkv):
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            ref_o, _, size, most = plain.row_attention(q[b, heads].double(), c.k[b][i, h], c.v[b][i, h], d ** -0.5)
            bound = ref_o.abs() * 2.0 ** -8 + (2 * (2.0 ** -18 * most + 2.0 ** -18) + 2.0 ** -14)[:, None] * size
            err = (o[b, heads].double() - ref_o).abs()
            assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "3"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (8, 1, 64)])
def test_decode_kv4_weights_of_fp32_outputs(pa, pa_env, hq, hkv, d, env):
    """Up to 16 keys and queries of one feature, so that hardly anything but the weights is rounded.  A logit x (in powers of two, below
    2.2) is an exact product times a factor: off by 2^-22 x, its difference to what weights are relative to (below 16) by 2^-21, the
    weight by 2^-22 more: 2^-22 (1 + ln 2 (2 + 2.2)) < 2^-20.  Its product with V's scale is rounded to 2^-24, and all of that is
    summed: 16 terms of at most 2^-24 of the sum each lose 2^-20.  Twice all of it, for the sum of weights: 2^-18."""
    pa_env(**env)
    c = _Cache(pa, [2, 3, 4, 5, 7, 9, 12, 16, 11, 6], hkv, d, seed=29)
    q = torch.zeros((10, hq, d))
    q[:, torch.arange(hq), torch.arange(hq) * 4 % d] = 3.0
    q = q.bfloat16().cuda()
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1, o_dtype=torch.float32, softmax_scale=0.125)
    for b in range(10):
        for h in range(hkv):
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            ref_o, ref_lse, size, most = plain.row_attention(q[b, heads].double(), c.k[b][:, h], c.v[b][:, h], 0.125)
            assert float(most.max()) * 1.443 < 2.2
            err = (o[b, heads].double() - ref_o).abs()
            assert (err <= 2.0 ** -18 * size).all(), float((err / size).max() * 2 ** 18)
            assert ((lse[b, heads].double() - ref_lse).abs() <= 2.0 ** -18).all()


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "3"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 128), (4, 1, 64)])
def test_decode_kv4_values_near_the_largest(pa, oracle, pa_env, hq, hkv, d, env):
    """Values as large as their sum by the weights allows (its magnitudes stay below 3.02e38): finite, and right."""
    pa_env(**env)
    c = _Cache(pa, [1, 3, 64, 700, 3000], hkv, d, seed=22, k_scale=2.0)
    for b, n in enumerate(c.lens):
        i = torch.arange(n)
        slots = (c.table[b].cpu()[i // 64].long() * 64 + i % 64).cuda()
        g = torch.Generator().manual_seed(b)
        v = torch.rand((n, hkv, d), generator=g).bfloat16().float()
        v[torch.rand(v.shape, generator=g) < 0.1] *= -1
        v[0, :, ::32] = 1.0
        v = (v * (3e38 / n)).bfloat16().cuda()
        pa.pa_kv4_append(pa.pa_kv4_read(c.pool, slots, d)[0], v, c.pool, slots)
        c.k[b], c.v[b] = (x.double() for x in pa.pa_kv4_read(c.pool, slots, d, dtype=torch.float32))
        assert torch.equal(c.v[b], plain.held(v))
    for W, S in ((5, 1), (60, 1)):
        c.check(oracle, hq, W, S, torch.float32)
        c.check(oracle, hq, W, S)


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "1"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("o_dtype", [torch.bfloat16, torch.float32])
def test_decode_kv4_large_values_under_a_rising_maximum(pa, pa_env, env, o_dtype):
    """16 blocks of keys, half of them with logits of 4, before or behind those of 0: exp(4) is a factor by which sums must not run
    over where the weighted mean does not."""
    pa_env(**env)
    d, n = 64, 1024
    c = _Cache(pa, [n, n], 1, d, seed=25)
    v = torch.full((n, 1, d), 3e38 / 530, dtype=torch.bfloat16).cuda()     # (512 + 512 exp(-4) weights)
    for b in range(2):
        i = torch.arange(n)
        slots = (c.table[b].cpu()[i // 64].long() * 64 + i % 64).cuda()
        k = torch.zeros((n, 1, d))
        k[(i >= 512) == (b == 0)] = 0.5
        pa.pa_kv4_append(k.bfloat16().cuda(), v, c.pool, slots)
        c.k[b], c.v[b] = plain.held(k.bfloat16().cuda()), plain.held(v)
    q = torch.ones((2, 3, d), dtype=torch.bfloat16).cuda()                # logits of 32 / 8
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 60, 1, o_dtype=o_dtype)
    for b in range(2):
        _near(o[b], lse[b], plain.row_attention(q[b].double(), c.k[b][:, 0], c.v[b][:, 0], d ** -0.5), o_dtype)


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "3"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("q_scale,k_scale", [(1e5, 1e5), (1e9, 1e7), (1e20, 1e15)])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_kv4_logits_beyond_the_range_of_exponents(pa, pa_env, d, q_scale, k_scale, env):
    """Logits of 1e10 and of 1e35 lie so far apart that the largest takes all: its key's values, and it, whatever a step of fp32 is
    there.  (fp32 sums are off by 2^-18 of the products' magnitudes at most, as in _near; a single weight is 1 or two parts of
    it, so its value is exact to 2^-15.)"""
    pa_env(**env)
    c = _Cache(pa, [1, 250, 700], 2, d, seed=27, k_scale=k_scale)
    q = _randn(3, 10, d, seed=28, scale=q_scale).cuda()
    for o_dtype in (torch.float32, torch.bfloat16):
        o, lse, ws = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 60, 1, o_dtype=o_dtype)
        pa.pa_decode_status(ws)
        assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
        taken = 0
        for b in range(3):
            for h in range(2):
                heads = slice(5 * h, 5 * h + 5)
                logits = q[b, heads].double() @ c.k[b][:, h].T * d ** -0.5
                off = 2.0 ** -18 * plain.row_attention(q[b, heads].double(), c.k[b][:, h], c.v[b][:, h], d ** -0.5)[3]
                first = logits.max(-1).values
                assert ((lse[b, heads].double() - first).abs() <= off + first.abs() * 2.0 ** -22).all()
                for g in range(5):
                    rivals = (logits[g] > first[g] - 2 * off[g] - 200).sum()
                    if rivals > 1:
                        continue
                    taken += 1
                    v = c.v[b][int(logits[g].argmax()), h]
                    err = (o[b, 5 * h + g].double() - v).abs()
                    assert (err <= v.abs() * (2.0 ** -7 if o_dtype == torch.bfloat16 else 2.0 ** -15)).all()
        assert taken >= 25


@pytest.mark.parametrize("env", [{}, {"PA_DECODE_PATH": "cluster", "PA_DECODE_CLUSTER": "3"}, {"PA_DECODE_PATH": "persist"}])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_kv4_queries_near_the_largest(pa, pa_env, d, env):
    """Heads of up to 3e38 beside ones of 1 and of 1e-30: over keys of zeros every head gives the mean of V, over keys of 2^-97 the
    large heads' logits are some 2^30, far apart, and the one key with the largest takes all (their fp32 sums are off by 2^-18 of
    the products' magnitudes at most, as in _near)."""
    pa_env(**env)
    c = _Cache(pa, [300, 250, 64], 1, d, seed=23)
    for b, scale in enumerate((0.0, 2.0 ** -97, 2.0 ** -97)):
        n = c.lens[b]
        i = torch.arange(n)
        slots = (c.table[b].cpu()[i // 64].long() * 64 + i % 64).cuda()
        k, v = _randn(n, 1, d, seed=40 + b, scale=scale).cuda(), _randn(n, 1, d, seed=50 + b).cuda()
        pa.pa_kv4_append(k, v, c.pool, slots)
        c.k[b], c.v[b] = plain.held(k), plain.held(v)
    q = torch.rand((3, 5, d), generator=torch.Generator().manual_seed(24)) * 2 - 1
    q *= torch.tensor([3e38, 1.0, 2.0 ** 118, 1e-30, 1e35])[None, :, None]
    q[:, :, 5] = torch.tensor([3.3e38, 1.0, 2.0 ** 118, 1e-30, 1e35])
    q = q.bfloat16().cuda()
    for o_dtype in (torch.float32, torch.bfloat16):
        o, lse, ws = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1, o_dtype=o_dtype)
        pa.pa_decode_status(ws)
        assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
        for b in range(3):
            ref = plain.row_attention(q[b].double(), c.k[b][:, 0], c.v[b][:, 0], d ** -0.5)
            small = torch.tensor([1, 3]).cuda() if b else torch.arange(5).cuda()
            _near(o[b, small], lse[b, small], [x[small] for x in ref], o_dtype)
            if b == 0:
                continue
            logits = q[b].double() @ c.k[b][:, 0].T * d ** -0.5
            for h in (0, 2, 4):
                first, second = logits[h].topk(2).values.tolist()
                off = 2.0 ** -18 * float(ref[3][h])
                assert first - second > 2 * off + 200           # (the inputs are such)
                assert abs(float(lse[b, h]) - first) <= off + abs(first) * 2.0 ** -22
                err = (o[b, h].double() - c.v[b][int(logits[h].argmax()), 0]).abs()
                bound = 2.0 ** -8 if o_dtype == torch.bfloat16 else 2.0 ** -15
                assert (err <= 2 * bound * c.v[b][int(logits[h].argmax()), 0].abs()).all()


def test_decode_kv4_values_of_mixed_magnitude(pa, oracle):
    """A group of V a million times the others, keys whose V is zero, V zero everywhere, a single weight that counts."""
    c = _Cache(pa, [700, 300, 64], 1, 128, seed=10, k_scale=3.0)
    for b, n in enumerate(c.lens):
        i = torch.arange(n)
        slots = (c.table[b].cpu()[i // 64].long() * 64 + i % 64).cuda()
        k, v = pa.pa_kv4_read(c.pool, slots, 128)
        if b == 0:
            v[::3] *= 1e6
            v[1::3, :, :64] = 0
        elif b == 1:
            v[:] = 0
        else:
            v[:, :, 32:64] *= 1e-25
        pa.pa_kv4_append(k, v, c.pool, slots)
        c.k[b], c.v[b] = plain.held(k), plain.held(v)
    for o_dtype in (torch.bfloat16, torch.float32):
        c.check(oracle, 6, 5, 1, o_dtype)
    c.lens_d[1] = 300
    q, o, lse, _ = c.check(oracle, 6, 5, 1)
    assert (o[1] == 0).all() and torch.isfinite(lse).all()


def test_decode_kv4_nan_goes_where_it_belongs(pa):
    """A NaN in a key that is attended to makes its heads' rows NaN, no others; in a masked key, none."""
    c = _Cache(pa, [900, 900], 2, 64, seed=11)
    q = _randn(2, 4, 64).cuda()
    k = torch.zeros((1, 2, 64), dtype=torch.bfloat16).cuda()
    k[0, 1, 3] = float("nan")
    slot = lambda b, pos: (c.table[b, pos // 64].long() * 64 + pos % 64)[None]  # noqa: E731
    fine, fine_lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    pa.pa_kv4_append(k, k, c.pool, slot(1, 400))      # block 6 of a row at block 14: distance 8, a power of two
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    assert torch.equal(o[0], fine[0]) and torch.isfinite(o[1, :2].float()).all()
    assert torch.isnan(o[1, 2:].float()).any(-1).all() and torch.isnan(lse[1, 2:]).all()
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 3, 0)   # the same block, other masks: blocks 12, 13, 14, 10, 6
    assert torch.isnan(lse[1, 2:]).all()
    pa.pa_kv4_append(torch.zeros_like(k), torch.zeros_like(k), c.pool, slot(1, 400))
    pa.pa_kv4_append(k, k, c.pool, slot(1, 500))      # block 7: distance 7, outside the window
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()


def test_decode_kv4_shared_pages_and_bad_entries(pa, oracle):
    """Two sequences on the same pages; entries outside the pool do not fault and leave other sequences alone."""
    c = _Cache(pa, [1500, 1500, 200], 2, 128, seed=12)
    c.table[1] = c.table[0]
    c.k[1], c.v[1] = c.k[0], c.v[0]
    _, o, _, _ = c.check(oracle, 6, 5, 1)
    c.table[0, :] = torch.tensor([-2 ** 31, 2 ** 31 - 1, 10 ** 6, -1], dtype=torch.int32).cuda().repeat(6)[:c.table.shape[1]]
    q = _randn(3, 6, 128, seed=1).cuda()
    o2, _, ws = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    pa.pa_decode_status(ws)
    assert torch.equal(o[1:], o2[1:])


@pytest.mark.parametrize("path,cluster", [("persist", "1"), ("cluster", "1"), ("cluster", "3"), ("cluster", "8")])
def test_decode_kv4_a_wait_that_runs_out_ends_the_kernel(pa, pa_env, path, cluster):
    """Under a limit of one cycle a call ends, with PA_ERR_TIMEOUT or the right result; the calls behind it are right."""
    pa_env(PA_DECODE_PATH=path, PA_DECODE_CLUSTER=cluster, PA_DECODE_STAGES="1")
    c = _Cache(pa, [50 + 40 * i for i in range(150)], 4, 128, seed=13)
    q = _randn(150, 28, 128).cuda()
    ref, ref_lse, ws = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 20, 1)
    pa.pa_decode_status(ws)
    for _ in range(10):
        try:
            pa.pa_set_wait_limit_cycles(1)
            o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 20, 1, workspace=ws)
            pa.pa_decode_status(ws)
            assert torch.equal(o, ref) and torch.equal(lse, ref_lse)
        except pa.PaError as err:
            assert "PA_ERR_TIMEOUT" in str(err)
        finally:
            pa.pa_set_wait_limit_cycles(0)
        o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 20, 1, workspace=ws)
        pa.pa_decode_status(ws)
        assert torch.equal(o, ref) and torch.equal(lse, ref_lse)


def test_decode_kv4_a_wait_that_runs_out_leaves_nothing_to_merge(pa, pa_env):
    """Under a limit of one cycle, on a workspace that never held a result: the kernel that merges rows takes nothing from it."""
    pa_env(PA_DECODE_PATH="persist")
    c = _Cache(pa, [5000 + 300 * i for i in range(30)], 4, 128, seed=14)
    q = _randn(30, 28, 128).cuda()
    ref, ref_lse, ws = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 60, 1)
    guard = torch.full((3, *q.shape), 7.0, dtype=torch.bfloat16).cuda()
    for byte in (0, 1, 127, 255):
        ws.fill_(byte)
        try:
            pa.pa_set_wait_limit_cycles(1)
            pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 60, 1, o=guard[1], workspace=ws)
            pa.pa_decode_status(ws)
        except pa.PaError as err:
            assert "PA_ERR_TIMEOUT" in str(err)
        finally:
            pa.pa_set_wait_limit_cycles(0)
        assert (guard[0] == 7).all() and (guard[2] == 7).all()
    o, lse, _ = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 60, 1, workspace=ws)
    pa.pa_decode_status(ws)
    assert torch.equal(o, ref) and torch.equal(lse, ref_lse)


def test_decode_kv4_heads_of_zeros_under_a_tiny_scale(pa):
    """The powers of two of a head of zeros times a small scale fall below fp32's range: still the mean of the values."""
    c = _Cache(pa, [70, 1, 200], 2, 64, seed=15)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16).cuda()
    ref = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)
    out = pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1, softmax_scale=1e-30)
    assert torch.equal(ref[0], out[0]) and torch.equal(ref[1], out[1]) and torch.isfinite(out[1]).all()


def test_decode_kv4_on_two_streams_at_once(pa):
    """Appends and decodes of two caches on two streams, every call with a workspace of its own."""
    caches = [_Cache(pa, [3000 + 100 * i + 7 * s for i in range(40)], 4, 128, seed=16 + s) for s in range(2)]
    q = _randn(40, 28, 128).cuda()
    ref = [pa.pa_decode_kv4(q, c.pool, c.table, c.lens_d, 5, 1)[:2] for c in caches]
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, pa.pa_decode_kv4(q, caches[i].pool, caches[i].table, caches[i].lens_d, 5, 1)))
    torch.cuda.synchronize()
    for i, (o, lse, ws) in got:
        assert torch.equal(o, ref[i][0]) and torch.equal(lse, ref[i][1])
        pa.pa_decode_status(ws)


def test_appends_reads_and_decodes_on_two_streams_at_once(pa):
    """Two caches on two streams: new tokens in, read back and decoded over, step after step, with nothing in between."""
    caches = [_Cache(pa, [1000 + 90 * i + 7 * s for i in range(30)], 4, 128, seed=30 + s) for s in range(2)]
    q = _randn(30, 28, 128).cuda()
    new = [[_randn(30, 4, 128, seed=60 + 10 * s + i).cuda() for i in range(10)] for s in range(2)]

    def steps(s):
        c, out = caches[s], []
        lens = c.lens_d.clone()
        pages = torch.arange(30).cuda()
        for i in range(10):
            slots = c.table[pages, (lens.long() - 1 - i) // 64].long() * 64 + (lens.long() - 1 - i) % 64   # (over the last tokens)
            pa.pa_kv4_append(new[s][i], new[s][9 - i], c.pool, slots)
            out += [*pa.pa_kv4_read(c.pool, slots, 128), *pa.pa_decode_kv4(q, c.pool, c.table, lens, 5, 1)[:2]]
        return out

    before = [c.pool.clone() for c in caches]
    ref = [steps(s) for s in range(2)]
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(8):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                caches[s].pool.copy_(before[s])
                got.append((s, steps(s)))
    torch.cuda.synchronize()
    for s, outs in got:
        for a, b in zip(outs, ref[s]):
            assert torch.equal(a, b)
    k = [plain.held(x) for x in new[0]]
    for i in range(10):
        assert torch.equal(ref[0][4 * i].double(), k[i].float().bfloat16().double())


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("captured", [False, True])
def test_a_serving_run(pa, oracle, captured):
    """Prompts of several lengths, then decoding steps, the way a server runs them: tables, norms and rotation, prefill of the
    prompts on what the projections gave, append at the slots, decode over the 4-bit pages.  Every step's output against
    64 bits on the values that the cache stands for; one graph replayed for all steps, with a padded place in the batch."""
    hq, hkv, d, W, S, steps = 14, 2, 128, 3, 1, 70
    prompts = [130, 1, 700, 63]
    batch, longest = len(prompts) + 1, 700          # (the last place of the batch is empty)
    g = torch.Generator().manual_seed(20)
    rand = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    wq, wk = 1 + 0.1 * rand(d), 1 + 0.1 * rand(d)
    angle = torch.arange(1000, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    cs = torch.cat((angle.cos(), angle.sin()), -1).float().cuda()
    n_pages = 60
    pool = _pool(pa, n_pages, hkv, d, 0xFF)
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    count = torch.tensor([n_pages], dtype=torch.int32).cuda()
    table = torch.full((batch, 16), -1, dtype=torch.int32).cuda()
    lens = torch.zeros(batch, dtype=torch.int32).cuda()
    new = torch.tensor(prompts + [0], dtype=torch.int32).cuda()
    cap = 1000
    qkv = rand(cap, hq + 2 * hkv, d)

    def project(x):
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def before(x, new, cap):
        cu, slots, positions, *_ = pa.pa_build_block_tables(new, lens, free, count, table, n_pages, cap, lens_out=lens, free_left=count)
        q, k, v = project(x)
        q, k = pa.pa_qk_norm_rope(q, k, wq, wk, cs, positions)
        pa.pa_kv4_append(k, v, pool, slots)
        return cu, slots, positions, q, k, v

    cu, slots, positions, q, k, v = before(qkv, new, cap)
    total = sum(prompts)
    assert cu.tolist() == [0, 130, 131, 831, 894, 894] and (slots[total:] == -1).all() and lens.tolist() == prompts + [0]
    row_ptr, col_idx = pa.pa_build_layout(longest, 64, W, S)
    o, lse, ws = pa.pa_prefill_varlen(q[:total], k[:total], v[:total], cu[:batch].clone(), longest, row_ptr, col_idx)
    pa.pa_prefill_status(ws)
    keys, values, at = [], [], 0
    for n in prompts:
        ref, lref, _ = oracle.prefill(q[at:at + n][None].cpu(), k[at:at + n][None].cpu(), v[at:at + n][None].cpu(), 64, W, S)
        assert np.abs(o[at:at + n].double().cpu().numpy() - ref[0]).max() <= 2e-2
        keys.append(plain.held(k[at:at + n])), values.append(plain.held(v[at:at + n]))
        at += n

    one = torch.tensor([1] * len(prompts) + [0], dtype=torch.int32).cuda()
    x = rand(batch, hq + 2 * hkv, d)
    out = torch.empty((batch, hq, d), dtype=torch.bfloat16, device="cuda")
    out_lse = torch.empty((batch, hq), device="cuda")
    state = {}

    def step():
        _, _, positions, q, k, v = before(x, one, batch)
        _, _, state["ws"] = pa.pa_decode_kv4(q, pool, table, lens, W, S, o=out, lse=out_lse)
        state.update(q=q, k=k, v=v, positions=positions)

    if captured:
        kept = [t.clone() for t in (lens, count, table)]
        step()                                       # (once outside, for what is set up on the first call)
        for t, was in zip((lens, count, table), kept):
            t.copy_(was)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for s in range(steps):
        x.copy_(rand(batch, hq + 2 * hkv, d))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        pa.pa_decode_status(state["ws"])
        assert lens.tolist() == [n + s + 1 for n in prompts] + [0]
        assert state["positions"].tolist() == [n + s for n in prompts] + [-1]
        assert (out[-1] == 0).all() and (out_lse[-1] == float("-inf")).all()
        for b in range(len(prompts)):
            keys[b] = torch.cat((keys[b], plain.held(state["k"][b:b + 1])))
            values[b] = torch.cat((values[b], plain.held(state["v"][b:b + 1])))
            if s % 9 and s != steps - 1:
                continue
            n = len(keys[b])
            j = torch.as_tensor(np.asarray(oracle.block_row((n - 1) // 64, W, S))).long()
            i = (j[:, None] * 64 + torch.arange(64)).flatten()
            i = i[i < n].cuda()
            for h in range(hkv):
                heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
                ref = plain.row_attention(state["q"][b, heads].double(), keys[b][i, h], values[b][i, h], d ** -0.5)
                _near(out[b, heads], out_lse[b, heads], ref, torch.bfloat16)
    held = sum((n + steps + 63) // 64 for n in prompts)
    assert int(count) == n_pages - held and len({int(p) for row in table.tolist() for p in row if p >= 0}) == held
