"""The operators around the attention calls that are timed, in their plain form and as the library's calls.

A case is a dict of plain values.  `kind` says what one pass does:

  tables   pa_build_block_tables: pages, slots and positions for the new tokens of a batch
  rope     pa_qk_norm_rope: the heads' norms and the rotation of queries and keys
  train    the same and its backward pass
  append   pa_kv4_append of a batch's new tokens, read back with pa_kv4_read
  decode   pa_decode_kv4: one token per sequence against pages held in 4 bits

Lengths follow from the case, all other inputs from the seed.  Head counts are those of the repository's workloads and
tests (28 query heads on 4 KV heads of 128 features and smaller ones).

A page of the 4-bit cache holds, for each KV head, 64 tokens' K nibbles, K scales, V nibbles, V scales.  A group is 32
features of a token; its scale s is bf16, a feature's value s (nibble - 8).  Words (8 nibbles, lowest first) of a K row:
features 32 j + 8 t + (0 .. 7) in word t D / 32 + j.  A V row is 8 chunks of D / 8 nibbles: features 32 j + 4 g + (0 .. 3)
at nibble 4 j of chunk g, chunks 0 - 3 and 4 - 7 changing places in tokens with bit 1 set.
"""
import math
import random

import torch

own = False

PAGE = 64       # tokens of a page
GROUP = 32      # features that share a scale
EPS = 1e-6


def _case(name, kind, seq, batch=1, heads=(28, 4, 128), min_seq=0, rot=0, style="halves", window=5, sink=1, out="bf16",
          k_scale=1.0, new=0, grad="f32"):
    hq, hkv, d = heads
    c = {"kind": kind, "batch": batch, "seq": seq, "min_seq": min_seq or seq, "q_heads": hq, "kv_heads": hkv, "head_dim": d,
         "rot": rot or d, "style": style, "window": window, "sink": sink, "out": out, "k_scale": k_scale, "new": new,
         "grad": grad}
    return dict(c, name=name) if name else c


def listed():
    return [
        # A decoding step of a serving batch: one new token each, a page now and then.
        _case("tables_step_b64", "tables", 16384, batch=64, min_seq=100, new=1),
        # Admission of many prompts at once.
        _case("tables_prompts_b500", "tables", 1, batch=500, new=4000),
        # A decoding step of eight users.
        _case("rope_step_b8", "rope", 131072, batch=8, min_seq=65536, new=1),
        # The 32K benchmark prompt.
        _case("rope_prompt_32k", "rope", 1, new=32768),
        # Fine-tuning a small model on ragged samples: heads of 64 features, half of them rotated, in neighbouring pairs.
        _case("train_5x900_d64", "train", 1, batch=5, heads=(16, 4, 64), rot=32, style="pairs", new=901, grad="bf16"),
        # Long-context training.
        _case("train_32k", "train", 1, new=32768),
        # One token for each of a full serving batch, the batch padded.
        _case("append_step_b256", "append", 16384, batch=256, min_seq=4096, new=1),
        # The caches of several prompts of different lengths.
        _case("append_prompts_8x12k", "append", 1, batch=8, new=12000),
        # One user's token against a short chat: nothing but latency.
        _case("decode_b1_4k", "decode", 4001),
        # Eight long contexts, 64K to 128K tokens.
        _case("decode_b8_128k", "decode", 131072, batch=8, min_seq=65536, k_scale=3.0),
        # A full serving batch: bandwidth.
        _case("decode_b256_16k", "decode", 16384, batch=256, min_seq=4096),
        # A small model with a window of 40 blocks, fp32 output.
        _case("decode_b24_d64_w40", "decode", 20000, batch=24, heads=(16, 4, 64), min_seq=300, window=40, sink=2, out="f32"),
    ]


_HEADS = [(28, 4, 128)] * 3 + [(14, 2, 128), (8, 2, 128), (16, 2, 128), (7, 1, 128), (16, 4, 64), (8, 2, 64), (8, 8, 64),
                               (2, 2, 64)]


def _size(rng, lo, hi):
    """Log-uniform in [lo, hi]; one in four a multiple of 64, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n // 64 * 64 if rng.random() < 0.25 else n))


def draw(rng):
    kind = rng.choice(["tables", "rope", "train", "append", "decode", "decode"])
    heads = rng.choice(_HEADS)
    if kind == "tables":
        batch = _size(rng, 1, 1000)
        if rng.random() < 0.5:
            return _case(None, kind, _size(rng, 64, 131072), batch=batch, min_seq=1, new=rng.choice([1, 1, 3]))
        return _case(None, kind, 1, batch=batch, new=_size(rng, 2, min(131072, 2000000 // batch)))
    if kind in ("rope", "train", "append"):
        more = {"heads": heads}
        if kind != "append":
            more |= {"rot": rng.choice([heads[2], heads[2], heads[2] // 2]), "style": rng.choice(["halves", "halves", "pairs"]),
                     "grad": rng.choice(["f32", "bf16"])}
        if kind != "train" and rng.random() < 0.4:
            seq = _size(rng, 64, 131072)
            return _case(None, kind, seq, batch=_size(rng, 1, 256), min_seq=max(1, seq // 8), new=1, **more)
        batch = rng.choice([1, 2, 3, 8])
        return _case(None, kind, 1, batch=batch, new=_size(rng, 2, 32768 // batch), **more)
    window, sink = rng.choice([(5, 1), (5, 1), (5, 1), (9, 1), (1, 1), (3, 2), (40, 1), (0, 0)])
    seq, batch = _size(rng, 1, 131072), _size(rng, 1, 256)
    cost = lambda: batch * heads[1] * heads[2] * (window + 24)  # noqa: E731
    while batch > 1 and (batch * seq * heads[1] * heads[2] > 256 * 16384 * 512 or cost() > 256 * 512 * 29):
        batch //= 2
    return _case(None, kind, seq, batch=batch, heads=heads, min_seq=max(1, seq // rng.choice([1, 2, 8])), window=window, sink=sink,
                 out="f32" if rng.random() < 0.2 else "bf16", k_scale=rng.choice([1.0, 1.0, 2.0, 3.0]))


def _lens(case):
    """(tokens cached, new tokens) of each sequence; decode: the cached ones include the current token."""
    rng = random.Random("%d %d %d %d" % (case["batch"], case["seq"], case["min_seq"], case["new"]))
    b, new = case["batch"], case["new"]
    if new > 3:  # prompts
        return [0] * b, [new] + [rng.randint(max(1, new // 8), new) for _ in range(b - 1)]
    return [case["seq"]] + [rng.randint(case["min_seq"], case["seq"]) for _ in range(b - 1)], [new] * b


# ---------------------------------------------------------------- the 4-bit form, in torch
def _row_order(d, device):
    """Where a feature's nibble stands in a row: K [d], V [64, d]."""
    f = torch.arange(d, device=device)
    j, w = f // GROUP, f % GROUP
    k = (w // 8 * (d // GROUP) + j) * 8 + w % 8
    token = torch.arange(PAGE, device=device)[:, None]
    chunk = (w // 4) ^ (4 * ((token >> 1) & 1))
    return k, chunk * (d // 8) + 4 * j + w % 4


def _quantise(x):
    """x [..., D] bf16 -> (nibbles 0 .. 15 as integers [..., D], scales bf16 [..., D / 32])."""
    g = x.float().unflatten(-1, (-1, GROUP))
    amax = g.abs().amax(-1, keepdim=True)
    s = (amax / 7).to(torch.bfloat16)
    tiny = amax < 2.0 ** -100
    s = torch.where(tiny, torch.zeros_like(s), s)
    quot = g / torch.where(tiny, torch.ones_like(amax), s.float())
    n = torch.where(tiny, torch.zeros_like(g), torch.copysign(torch.ceil(quot.abs() - 0.5), quot))  # (ties to zero)
    return (n.flatten(-2) + 8).to(torch.uint8), s.squeeze(-1)


def _rows(nibbles, order):
    """Nibbles [..., D] to the bytes [..., D / 2] of a row; `order` [..., D] or [D]."""
    put = torch.empty_like(nibbles).scatter_(-1, order.expand(nibbles.shape), nibbles).unflatten(-1, (-1, 2))
    return put[..., 0] | (put[..., 1] << 4)


def _parts(pool, d):
    """Views of a pool [..., record]: K bytes [..., 64, d / 2], K scales [..., 64, d / 16] as bytes, V bytes, V scales."""
    sizes = [PAGE * d // 2, PAGE * d // 16] * 2
    return [p.unflatten(-1, (PAGE, -1)) for p in torch.split(pool, sizes, dim=-1)]


def _values(rows, scales, order):
    """Bytes [..., D / 2] and scales (bytes [..., D / 16]) of rows to fp32 values [..., D]."""
    n = torch.stack((rows & 15, rows >> 4), -1).flatten(-2)
    n = torch.gather(n, -1, order.expand(n.shape)).float() - 8
    s = scales.contiguous().view(torch.bfloat16).float()
    return (n.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def _bytes(scales):
    return scales.contiguous().view(torch.uint8)


class _Draws:
    """Tensors from one seed, drawn on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, *shape, scale=1.0):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=torch.bfloat16)
        return t.mul_(scale) if scale != 1.0 else t

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def prepare(case, seed):
    make = _Draws(seed)
    kind, b, hq, hkv, d = (case[k] for k in ("kind", "batch", "q_heads", "kv_heads", "head_dim"))
    cached, new = _lens(case)
    s = {"case": case}
    if kind == "tables":
        room = max((c + n + PAGE - 1) // PAGE for c, n in zip(cached, new)) + 1
        have = [(c + PAGE - 1) // PAGE for c in cached]
        want = sum((c + n + PAGE - 1) // PAGE - h for c, n, h in zip(cached, new, have))
        pages = sum(have) + want + 16
        order = make.order(pages).to(torch.int32)
        table = torch.full((b, room), -1, dtype=torch.int32, device="cuda")
        held = torch.arange(room, device="cuda")[None, :] < _ints(have)[:, None]
        table[held] = order[:sum(have)]
        s |= {"new": _ints(new), "cached": _ints(cached), "free": order[sum(have):].contiguous(), "count": _ints([pages - sum(have)]),
              "table": table, "pages": pages, "tokens": (sum(new) + 63) // 64 * 64}
        return s
    if kind in ("rope", "train"):
        tokens = sum(new)
        at = [torch.arange(c, c + n, device="cuda") for c, n in zip(cached, new)]
        s["positions"] = torch.cat(at).to(torch.int32)
        rot = case["rot"]
        freq = 1e6 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        angle = torch.arange(max(c + n for c, n in zip(cached, new)), device="cuda", dtype=torch.float64)[:, None] * freq
        s["cos_sin"] = torch.cat((angle.cos(), angle.sin()), -1).float()
        # Queries and keys as a projection leaves them: side by side in a token's row, V behind them.
        qkv = make(tokens, hq + 2 * hkv, d)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
        s["q_weight"], s["k_weight"] = 1 + make(d, scale=0.2), 1 + make(d, scale=0.2)
        if kind == "train":
            dtype = torch.float32 if case["grad"] == "f32" else torch.bfloat16
            s["d_q"], s["d_k"] = make(tokens, hq, d).to(dtype), make(tokens, hkv, d).to(dtype)
        return s
    record = PAGE * (d + d // 8)
    if kind == "append":
        tokens = sum(new)
        blocks = [(c + n + PAGE - 1) // PAGE for c, n in zip(cached, new)]
        # (the last page is in no one's table)
        s["pool"] = torch.zeros((sum(blocks) + 1, hkv, record), dtype=torch.uint8, device="cuda")
        order = make.order(sum(blocks))
        first = [0]
        for n in blocks:
            first.append(first[-1] + n)
        slots = []
        for i in range(b):
            at = torch.arange(cached[i], cached[i] + new[i], device="cuda")
            slots.append(order[first[i] + at // PAGE] * PAGE + at % PAGE)
        slots = torch.cat(slots)
        if case["new"] == 1 and b > 8:  # places of the batch that no request has
            slots[-(b // 16):] = -1
        s["slots"] = slots.contiguous()
        kv = make(tokens, 2 * hkv, d)
        s["k"], s["v"] = kv[:, :hkv], kv[:, hkv:]
        return s
    blocks = [(c + PAGE - 1) // PAGE for c in cached]
    room, pages = max(blocks), sum(blocks)
    order = make.order(pages).to(torch.int32)
    table = torch.full((b, room), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(room, device="cuda")[None, :] < _ints(blocks)[:, None]] = order
    pool = torch.empty((pages, hkv, record), dtype=torch.uint8, device="cuda")
    k_order, v_order = _row_order(d, "cuda")
    for p0 in range(0, pages, 4096):
        part = _parts(pool[p0:p0 + 4096], d)
        shape = (min(4096, pages - p0), hkv, PAGE, d)
        for i, (rows_order, scale) in enumerate(((k_order, case["k_scale"]), (v_order, 1.0))):
            n, sc = _quantise(make(*shape, scale=scale))
            part[2 * i].copy_(_rows(n, rows_order))
            part[2 * i + 1].copy_(_bytes(sc))
    s |= {"pool": pool, "table": table, "lens": _ints(cached), "q": make(b, hq, d)}
    # A decode loop keeps its outputs and scratch.
    s["o"] = torch.empty((b, hq, d), dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")
    s["lse"] = torch.empty((b, hq), dtype=torch.float32, device="cuda")
    s["keep"] = {}
    s["most"] = max(_row_blocks(i, case["window"], case["sink"]) for i in {n - 1 for n in blocks})
    return s


# ---------------------------------------------------------------- the plain forms
def _tables(s):
    new, cached, table = s["new"].long(), s["cached"].long(), s["table"]
    b, room = table.shape
    cap = s["tokens"]
    end = torch.cumsum(new, 0)
    have, need = (cached + 63) // 64, (cached + new + 63) // 64
    fits = (need <= room) & (end <= cap)
    want = torch.where(fits, need - have, torch.zeros_like(need))
    taken = torch.cumsum(want, 0)
    count = s["count"].long()
    served = fits & ((want == 0) | (taken <= count))
    block = torch.arange(room, device=new.device)
    fresh = served[:, None] & (block >= have[:, None]) & (block < need[:, None])
    index = count - 1 - ((taken - want)[:, None] + block - have[:, None])
    table = torch.where(fresh, s["free"][index.clamp(0, s["free"].numel() - 1)], table)
    left = count - torch.where(served, taken * (want > 0), torch.zeros_like(taken)).amax()
    i = torch.arange(cap, device=new.device)
    seq = torch.searchsorted(end, i, right=True)
    inside = seq < b
    seq = seq.clamp(max=b - 1)
    at = cached[seq] + i - (end - new)[seq]
    ok = inside & served[seq]
    page = table[seq, (at // 64).clamp(0, room - 1)].long()
    ok = ok & (page >= 0) & (page < s["pages"])
    slots = torch.where(ok, page * 64 + at % 64, torch.full_like(page, -1))
    positions = torch.where(inside, at, torch.full_like(at, -1)).to(torch.int32)
    cu = torch.cat((torch.zeros_like(end[:1]), end)).to(torch.int32)
    lens = torch.where(served, cached + new, cached).to(torch.int32)
    return cu, slots, positions, lens, left.to(torch.int32), table


def _rotate(x, cos, sin, style, back=False):
    """The first 2 n features of x [tokens, heads, D] by angles whose cosines and sines are cos, sin [tokens, 1, n]."""
    n = cos.shape[-1]
    sin = -sin if back else sin
    if style == "halves":
        a, b = x[..., :n], x[..., n:2 * n]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., :2 * n:2], x[..., 1:2 * n:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y, x[..., 2 * n:]), -1)


def _norm_rope(x, w, cos, sin, style):
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    return _rotate(y, cos, sin, style).to(torch.bfloat16)


def _norm_rope_backward(d_out, x, w, cos, sin, style):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    g = _rotate(d_out.float(), cos, sin, style, back=True)
    xn = x * r
    h = g * w.float()
    dx = r * (h - xn * (h * xn).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (g * xn).sum((0, 1))


def _append(s):
    slots, pool, (hkv, d) = s["slots"], s["pool"], s["k"].shape[1:]
    spare = (pool.shape[0] - 1) * PAGE
    at = torch.where(slots < 0, torch.full_like(slots, spare), slots)
    page, place = at // PAGE, at % PAGE
    k_order, v_order = _row_order(d, pool.device)
    v_order = v_order[place][:, None, :]
    kn, ks = _quantise(s["k"])
    vn, vs = _quantise(s["v"])
    part = _parts(pool, d)
    for where, what in zip(part, (_rows(kn, k_order), _bytes(ks), _rows(vn, v_order), _bytes(vs))):
        where[page, :, place] = what
    kb, ks, vb, vs = (where[page, :, place] for where in part)
    none = (slots < 0)[:, None, None]
    k, v = _values(kb, ks, k_order), _values(vb, vs, v_order)
    return k.masked_fill(none, 0.0), v.masked_fill(none, 0.0)


def _decode(s):
    case, table, lens, q = s["case"], s["table"], s["lens"].long(), s["q"].float()
    b, hq, d = q.shape
    hkv = case["kv_heads"]
    row = ((lens - 1) // PAGE)[:, None]
    j = torch.arange(table.shape[1], device=q.device)
    far = row - j
    listed_ = (far >= 0) & ((far < case["window"]) | ((far & (far - 1)) == 0) | (j < case["sink"]))
    block = torch.sort(torch.where(listed_, j, torch.full_like(far, table.shape[1])), -1).values[:, :s["most"]]
    there = block < table.shape[1]
    block = block.clamp(max=table.shape[1] - 1)
    page = torch.where(there, torch.gather(table, 1, block).long(), torch.zeros_like(block))
    k_order, v_order = _row_order(d, q.device)
    kb, ks, vb, vs = _parts(s["pool"][page], d)  # [b, blocks, hkv, 64, ...]
    token = block[..., None] * PAGE + torch.arange(PAGE, device=q.device)
    seen = (there[..., None] & (token < lens[:, None, None]))[:, :, None, None, :]
    k = _values(kb, ks, k_order)
    logits = torch.einsum("bhgd,bnhtd->bnhgt", q.view(b, hkv, hq // hkv, d), k) / math.sqrt(d)
    del k
    logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax((1, 4), keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum((1, 4), keepdim=True)
    v = _values(vb, vs, v_order)
    o = torch.einsum("bnhgt,bnhtd->bhgd", p, v) / total[:, 0]
    lse = (top + torch.log(total))[:, 0, :, :, 0].reshape(b, hq)
    return o.reshape(b, hq, d).to(s["o"].dtype), lse


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        import paper_2503_03588_b200 as pa
    if kind == "tables":
        if own:
            cu, slots, positions, lens, left, _ = pa.pa_build_block_tables(
                s["new"], s["cached"], s["free"], s["count"], s["table"], s["pages"], s["tokens"])
            return cu, slots, positions, lens, left, s["table"]
        return _tables(s)
    if kind in ("rope", "train"):
        pairs = case["style"] == "pairs"
        args = (s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos_sin"], s["positions"])
        if own:
            out = pa.pa_qk_norm_rope(*args, eps=EPS, interleaved=pairs)
            if kind == "train":
                out += pa.pa_qk_norm_rope_backward(*args, s["d_q"], s["d_k"], eps=EPS, interleaved=pairs)[:4]
            return out
        cos, sin = s["cos_sin"][s["positions"].long()][:, None, :].chunk(2, -1)
        turn = (cos, sin, case["style"])
        out = (_norm_rope(s["q"], s["q_weight"], *turn), _norm_rope(s["k"], s["k_weight"], *turn))
        if kind == "train":
            dq, dwq = _norm_rope_backward(s["d_q"], s["q"], s["q_weight"], *turn)
            dk, dwk = _norm_rope_backward(s["d_k"], s["k"], s["k_weight"], *turn)
            out += (dq, dk, dwq, dwk)
        return out
    if kind == "append":
        if own:
            pa.pa_kv4_append(s["k"], s["v"], s["pool"], s["slots"])
            return pa.pa_kv4_read(s["pool"], s["slots"], case["head_dim"], dtype=torch.float32)
        return _append(s)
    if own:
        o, lse, s["keep"]["ws"] = pa.pa_decode_kv4(s["q"], s["pool"], s["table"], s["lens"], case["window"], case["sink"], o=s["o"],
                                                   lse=s["lse"], workspace=s["keep"].get("ws"), o_dtype=s["o"].dtype)
        return o, lse
    return _decode(s)


def _row_blocks(i, window, sink):
    """How many key blocks query block i lists (distances below the window, powers of two, sink blocks)."""
    w = max(window, 1)
    return sum(1 for j in range(min(sink, i + 1)) if i - j >= w) + min(i + 1, w) + sum(
        1 for e in range(32) if w <= 1 << e <= i and i - (1 << e) >= sink)


def work(case):
    hq, hkv, d = (case[k] for k in ("q_heads", "kv_heads", "head_dim"))
    cached, new = _lens(case)
    tokens = sum(new)
    kind = case["kind"]
    if kind == "tables":
        # Lengths in and out, cu_seqlens; a page number read and written; a slot and a position a token.
        pages = sum((c + n + 63) // 64 - (c + 63) // 64 for c, n in zip(cached, new))
        return {"bytes": 16 * case["batch"] + 8 * pages + 12 * tokens, "flops": 10 * tokens}
    if kind in ("rope", "train"):
        n = tokens * (hq + hkv) * d
        size, flops = 4 * n + tokens * (4 + 4 * case["rot"]), 8 * n
        if kind == "train":  # the gradients of the outputs in, those of the inputs out
            size += n * ((4 if case["grad"] == "f32" else 2) + 2)
            flops += 16 * n
        return {"bytes": size, "flops": flops}
    if kind == "append":
        # K and V in; their 4-bit form out, and in again; fp32 values out.
        n = 2 * tokens * hkv * d
        return {"bytes": 2 * n + 2 * (9 * n // 16) + 4 * n + 16 * tokens, "flops": 6 * n}
    size = flops = 0
    for n in cached:
        keys = (_row_blocks((n - 1) // PAGE, case["window"], case["sink"]) - 1) * PAGE + (n - 1) % PAGE + 1
        size += keys * hkv * (d + d // 8) + hq * (d * (6 if case["out"] == "f32" else 4) + 4)
        flops += 4 * keys * hq * d
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _held(x):
    """The value that a number of a group has in 4 bits, in fp64: whole multiples of a seventh of the largest, rounded to bf16."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().max(-1, keepdim=True).values
    unit = (top / 7).to(torch.bfloat16).double()
    unit = unit * (top >= 2.0 ** -100)
    safe = unit + (unit == 0)
    low = torch.floor(g.abs() / safe)
    steps = low + (g.abs() / safe - low > 0.5)
    return (torch.sign(g) * steps * unit).reshape(x.shape)


def _nibble_at(pool, d, page, head, token, feature, v):
    """The value at (page, head, token of the page, feature) of a pool, by its byte's address; index tensors that broadcast."""
    record = pool.shape[-1]
    group, within = feature // 32, feature % 32
    if v:
        nib = ((within // 4) ^ (((token // 2) % 2) * 4)) * (d // 8) + group * 4 + within % 4
    else:
        nib = (within // 8) * (d // 4) + group * 8 + within % 8
    base = (page * pool.shape[1] + head) * record + (record // 2 if v else 0)
    flat = pool.reshape(-1)
    byte = flat[base + token * (d // 2) + nib // 2].int()
    u = torch.where(nib % 2 == 0, byte % 16, byte // 16)
    sc = flat.view(torch.bfloat16)[(base + 64 * (d // 2)) // 2 + token * (d // 32) + group]
    return (u - 8).double() * sc.double()


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "tables":
        new, cached = s["new"].tolist(), s["cached"].tolist()
        table, free, left = s["table"].cpu(), s["free"].tolist(), int(s["count"])
        slots, positions = [-1] * s["tokens"], [-1] * s["tokens"]
        cu, lens, i = [0], [], 0
        for b, (c, n) in enumerate(zip(cached, new)):  # (there are pages and places for all)
            for block in range(-(-c // 64), -(-(c + n) // 64)):
                left -= 1
                table[b, block] = free[left]
            row = table[b].tolist()
            for at in range(c, c + n):
                slots[i], positions[i] = row[at // 64] * 64 + at % 64, at
                i += 1
            cu.append(i)
            lens.append(c + n)
        return (_ints(cu), _ints(slots, torch.int64), _ints(positions), _ints(lens), _ints([left]), table.cuda())
    if kind in ("rope", "train"):
        table = s["cos_sin"].double()[s["positions"].long()]
        n = case["rot"] // 2
        turn = torch.complex(table[:, :n], table[:, n:])[:, None, :]

        def pairs(x):
            first, second = (x[..., :n], x[..., n:2 * n]) if case["style"] == "halves" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
            return torch.complex(first.contiguous(), second.contiguous())

        def turned(x, by):
            z, y = pairs(x) * by, x.clone()
            if case["style"] == "halves":
                y[..., :n], y[..., n:2 * n] = z.real, z.imag
            else:
                y[..., 0:2 * n:2], y[..., 1:2 * n:2] = z.real, z.imag
            return y

        def both(x, w, d_out):
            x, w = x.double(), w.double()
            length = torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS)
            unit = x / length
            out = turned(unit * w, turn)
            if d_out is None:
                return out, None, None
            g = turned(d_out.double(), turn.conj())
            along = torch.mean(g * w * unit, -1, keepdim=True)
            return out, (g * w - unit * along) / length, torch.sum(g * unit, (0, 1))

        q, dq, dwq = both(s["q"], s["q_weight"], s.get("d_q"))
        k, dk, dwk = both(s["k"], s["k_weight"], s.get("d_k"))
        return (q, k, dq, dk, dwq, dwk) if kind == "train" else (q, k)
    if kind == "append":
        kept = (s["slots"] >= 0).double()[:, None, None]
        return _held(s["k"]) * kept, _held(s["v"]) * kept
    hq, hkv, d = (case[k] for k in ("q_heads", "kv_heads", "head_dim"))
    lens = s["lens"].tolist()
    o = torch.zeros((len(lens), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((len(lens), hq), dtype=torch.float64, device="cuda")
    f, head = torch.arange(d, device="cuda"), torch.arange(hkv, device="cuda")[:, None, None]
    for b, n in enumerate(lens):
        last = (n - 1) // 64
        blocks = [j for j in range(last + 1)
                  if last - j < case["window"] or bin(last - j).count("1") <= 1 or j < case["sink"]]
        token = torch.tensor([64 * j + t for j in blocks for t in range(64) if 64 * j + t < n], device="cuda")
        page = s["table"][b].long()[token // 64][:, None]
        at = (s["pool"], d, page, head, (token % 64)[:, None], f)
        keys, values = _nibble_at(*at, v=False), _nibble_at(*at, v=True)
        q = s["q"][b].double().reshape(hkv, hq // hkv, d)
        logits = q @ keys.transpose(1, 2) / d ** 0.5
        lse[b] = torch.logsumexp(logits, -1).reshape(hq)
        o[b] = (torch.softmax(logits, -1) @ values).reshape(hq, d)
    return o, lse
