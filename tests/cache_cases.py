"""The operators of include/respec_cache.h in 64 bits, and batches for them; everything is evaluated on the host."""
import math
from dataclasses import dataclass
from fractions import Fraction

import torch

import prompt_cases as pc

F64 = torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
NAN_CODE = 0x7F


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

_TURN = 2 * Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


def angle(p, w):
    """p w, less whole turns: exact but for pi's 50 digits and the float."""
    a = Fraction(p) * Fraction(w)
    return float(a - round(a / _TURN) * _TURN)


def rotary(x, pos, w, rotary_dim, half, amplitude=1.0):
    """(rows, tolerance) of x [T][H][D] at positions [T] (ints) for frequencies w (floats).

    With e = 2^-24 a cosine or sine is off by: its argument, at most pi / 4 and rounded twice, 1.57 e; three
    roundings of its polynomial, 3 e; what the polynomial leaves out, e / 2; the angle itself, 2^-31 of a turn, e / 20;
    the amplitude's product, e.  A product and the sum round by e each of their size.  In all under 2^-20 (16 e) of
    amplitude (|x_a| + |x_b|), and the result's rounding.
    """
    u = torch.finfo(x.dtype).eps / 2
    y = x.to(F64)
    turned = torch.tensor([[angle(p, f) for f in w] for p in pos], dtype=F64)
    c, s = turned.cos()[:, None] * amplitude, turned.sin()[:, None] * amplitude
    r = rotary_dim
    a, b = (y[..., :r // 2], y[..., r // 2:r]) if half else (y[..., :r:2], y[..., 1:r:2])
    pair = (a * c - b * s, b * c + a * s)
    size = amplitude * (a.abs() + b.abs())
    join = (lambda t: torch.cat(t, -1)) if half else (lambda t: torch.stack(t, -1).flatten(-2))
    out = torch.cat([join(pair), y[..., r:]], -1)
    tol = torch.cat([join((size, size)) * 2 ** -20 + join(pair).abs() * u + 1e-30, torch.full_like(y[..., r:], 1e-300)], -1)
    return out, tol


# ---------------------------------------------------------------------------
# the 8-bit cache
# ---------------------------------------------------------------------------

def power(top: float) -> int:
    """The least k from -126 on with top <= 448 2^k."""
    k = -126
    if top > 0:
        k = max(k, math.floor(math.log2(top / 448)) - 1)
        while top > math.ldexp(448.0, k):
            k += 1
    return k


def codes(x, k):
    """Nearest e4m3 values (ties to even) of x 2^-k, float64 in, bytes out; what is not finite is a NaN."""
    fine = x.isfinite()
    y = torch.where(fine, x, 0.0) * 2.0 ** -k
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.round(y / step) * step
    assert float(y.abs().max() if y.numel() else 0) <= 448
    return torch.where(fine, y.float().to(E4M3).view(torch.uint8), torch.tensor(NAN_CODE, dtype=torch.uint8))


def values(code, byte):
    return code.view(E4M3).to(F64) * torch.exp2(byte.to(F64) - 127)


@dataclass
class Q8:
    """A chunk batch over an 8-bit cache: its state before the new rows go in (k, v, ks, vs) and after (want_*)."""
    c: pc.Chunk
    block: int
    before: list   # codes of K, V and exponent bytes of K, V
    after: list


def q8(sizes, *, block=16, edit=None, front=1.0, stale=NAN_CODE, **kw):
    """A batch as prompt_cases.make's, its rows in front quantised block by block (``front`` times as large), blocks that are
    nobody's with bytes of any kind.  edit(c): changes the new rows before they are appended.  c.rows hold what
    the cache stands for after the append."""
    c = pc.make(sizes, **kw)
    if edit:
        edit(c)
    gen = torch.Generator().manual_seed(7 + kw.get("seed", 0))
    n_pages, hkv, page, d = c.k_pages.shape
    assert page % block == 0
    before, after = [], []
    for which in (0, 1):
        code = torch.full((n_pages, hkv, page, d), stale, dtype=torch.uint8)
        byte = torch.randint(0, 255, (n_pages, hkv, page // block), generator=gen, dtype=torch.uint8)
        news, done = (c.k_new, c.v_new)[which], 0
        for b, (n, l) in enumerate(c.sizes):
            rows = c.rows[b][which][:l].to(F64) * front
            for r0 in range(0, l, block):
                at, within = int(c.table[b, r0 // page]), r0 % page
                part = rows[r0:r0 + block].transpose(0, 1)
                k = torch.tensor([power(x) for x in part.abs().amax((1, 2)).tolist()])
                byte[at, :, within // block] = (k + 127).to(torch.uint8)
                code[at, :, within:within + part.shape[1]] = codes(part, k[:, None, None])
        before += [code.clone(), byte.clone()]
        for b, (n, l) in enumerate(c.sizes):
            append(code, byte, news[done:done + n].to(F64), c.table[b], l, page, block)
            done += n
        after += [code, byte]
        for b, (n, l) in enumerate(c.sizes):
            out = torch.empty(n + l, hkv, d, dtype=F64)
            for r in range(n + l):
                at, within = int(c.table[b, r // page]), r % page
                out[r] = values(code[at, :, within], byte[at, :, within // block, None])
            c.rows[b] = (out, c.rows[b][1]) if which == 0 else (c.rows[b][0], out)
    order = (0, 2, 1, 3)
    return Q8(c, block, [before[i] for i in order], [after[i] for i in order])


def append(code, byte, new, table, length, page, block):
    """The definition of an append of rows `new` [n][Hkv][D] behind `length` rows, in place."""
    n = len(new)
    for blk in range(length // block, (length + n - 1) // block + 1 if n else 0):
        lo, hi = max(blk * block, length), min((blk + 1) * block, length + n)
        at, sub, r0 = int(table[blk * block // page]), blk * block % page // block, blk * block % page
        for h in range(code.shape[1]):
            part = new[lo - length:hi - length, h]
            k = power(float(torch.where(part.isfinite(), part.abs(), 0.0).max()))
            if lo > blk * block:
                was = int(byte[at, h, sub]) - 127
                k = max(k, was)
                old = slice(r0, r0 + lo - blk * block)
                if k > was:
                    code[at, h, old] = codes(values(code[at, h, old], torch.tensor(was + 127)), k)
            byte[at, h, sub] = k + 127
            code[at, h, r0 + lo - blk * block:r0 + hi - blk * block] = codes(part, k)


def same_codes(got, want):
    """Equal bytes, NaNs of either sign alike."""
    nan = (got & 0x7F) == NAN_CODE
    return bool(((got == want) | (nan & ((want & 0x7F) == NAN_CODE))).all())
