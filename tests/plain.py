"""Plain forms, in 64 bits, of the operators around the attention calls: block tables, norms with rotation, the 4-bit cache."""
import numpy as np
import torch


def tables(new, cached, free, count, table, n_pages, cap):
    """Sequence by sequence, token by token.  Returns (cu, slots, positions, lens, left, table)."""
    table = np.array(table, dtype=np.int64)
    count = max(0, min(int(count), len(free)))
    slots, positions = np.full(cap, -1, dtype=np.int64), np.full(cap, -1, dtype=np.int64)
    cu, lens, end, wanted, left = [0], [], 0, 0, count
    for b, (n_, c) in enumerate(zip(map(int, new), map(int, cached))):
        n, start = max(n_, 0), end
        end += n
        have, need = -(-max(c, 0) // 64), -(-(c + n) // 64)
        fits = c >= 0 and n_ >= 0 and need <= table.shape[1] and end <= cap and c + n < 2 ** 31
        want = need - have if fits else 0
        wanted += want
        served = fits and (want == 0 or wanted <= count)
        if served and want:
            for i in range(want):
                table[b, have + i] = free[count - 1 - (wanted - want + i)]
            left = count - wanted
        for i in range(n):
            if start + i >= cap:
                break
            at = c + i
            positions[start + i] = min(at, 2 ** 31 - 1)
            if served and 0 <= table[b, at // 64] < n_pages:
                slots[start + i] = table[b, at // 64] * 64 + at % 64
        cu.append(min(end, 2 ** 31 - 1))
        lens.append(c + n if served else c)
    return cu, slots, positions, lens, left, table


def norm_rope(x, w, cos_sin, pos, eps, interleaved, back=None):
    """x [tokens, heads, D], w [D], cos_sin [n, rot], pos [tokens] (inside the table).  Returns (out, size) in fp64, `size`
    bounding the terms that out was summed from; with `back` (the outputs' gradient) also dx, its terms, dw, its terms."""
    x, w, table = x.double(), w.double(), cos_sin.double()[pos.long()]
    rot = table.shape[1]
    c, s = table[:, None, :rot // 2], table[:, None, rot // 2:]
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))

    def turn(y, s):
        z = y.clone()
        z[..., one], z[..., two] = y[..., one] * c - y[..., two] * s, y[..., two] * c + y[..., one] * s
        return z

    def size(y):
        z = y.abs().clone()
        z[..., one] = z[..., two] = (y[..., one].abs() + y[..., two].abs())
        return z

    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xn = x * r
    if back is None:
        return turn(xn * w, s), size(xn * w)
    g, gs = turn(back.double(), -s), size(back.double())
    h, hs = g * w, gs * w.abs()
    dx = r * (h - xn * (h * xn).mean(-1, keepdim=True))
    dxs = r * (hs + xn.abs() * (hs * xn.abs()).mean(-1, keepdim=True))
    return turn(xn * w, s), size(xn * w), dx, dxs, (g * xn).sum((0, 1)), (gs * xn.abs()).sum((0, 1))


def held(x):
    """What a group of 32 numbers is held as, fp64 [..., D]."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    s = (top / 7).to(torch.bfloat16).double()
    q = g.abs() / torch.where(s > 0, s, torch.ones_like(s))
    n = torch.where(q - q.floor() > 0.5, q.floor() + 1, q.floor())
    y = torch.sign(g) * n * s
    y = torch.where(top < 2.0 ** -100, torch.zeros_like(y), y)
    return torch.where(torch.isfinite(top), y, torch.full_like(y, float("nan"))).flatten(-2)


def page_values(pool, d):
    """Every value of a pool [pages, heads, 72 d] uint8 as the header describes it: K, V fp64 [pages, heads, 64, d]."""
    raw = pool.cpu().numpy()
    out = []
    for v in (False, True):
        half = raw[..., 36 * d:] if v else raw[..., :36 * d]
        rows = half[..., :32 * d].reshape(*raw.shape[:2], 64, d // 2)
        nib = np.stack((rows & 15, rows >> 4), -1).reshape(*raw.shape[:2], 64, d)
        scales = torch.from_numpy(half[..., 32 * d:].copy()).view(torch.bfloat16).double().numpy().reshape(*raw.shape[:2], 64, d // 32)
        y = np.empty(nib.shape)
        for f in range(d):
            j, w = f // 32, f % 32
            if v:
                for token in range(64):
                    at = ((w // 4) ^ (4 if token & 2 else 0)) * (d // 8) + 4 * j + w % 4
                    y[..., token, f] = (nib[..., token, at].astype(int) - 8) * scales[..., token, j]
            else:
                y[..., f] = (nib[..., (w // 8 * (d // 32) + j) * 8 + w % 8].astype(int) - 8) * scales[..., j]
        out.append(torch.from_numpy(y))
    return out


def row_attention(q, k, v, scale):
    """q [heads, D], k, v [keys, D] fp64.  Returns O, LSE, sum p |v|, and the largest sum of |q k| in a logit."""
    s = q @ k.T * scale
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[:, None])
    return p @ v, lse, p @ v.abs(), (q.abs() @ k.abs().T * scale).amax(-1)
