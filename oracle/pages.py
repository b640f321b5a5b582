"""Writing, reading and sharing a decoding batch's pages, in float64 and plain Python straight from the definitions.

The decode stage of the paper (Section 2.1) appends every token's key and value to the cache; a server also keeps them in 8 bits and
lets several sequences (samples, beams) go on from one.
"""
import numpy as np

PAGE = 16


def e4m3_values():
    """What the 256 bytes stand for (4 exponent bits, bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    v = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = np.nan if (b & 127) == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = -x if b >= 128 else x
    return v


VALUES = e4m3_values()


def to_e4m3(x):
    """Bytes nearest to x, ties to the even mantissa, magnitudes above 448 to 448, NaN to 0x7f (its sign is not kept)."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    up = np.searchsorted(VALUES[:127], mag)                # first value not below
    up = np.minimum(up, 126)
    down = np.maximum(up - 1, 0)
    d_up, d_down = VALUES[up] - mag, mag - VALUES[down]
    b = np.where((d_up < d_down) | ((d_up == d_down) & (up % 2 == 0)), up, down).astype(np.uint8)
    b = np.where(VALUES[up] == mag, up, b).astype(np.uint8)
    return np.where(np.isnan(x), 127, b | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def scale_exponent(amax):
    """The least e in -32 .. 32 with amax <= 448 * 2^e."""
    for e in range(-32, 32):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return 32


def norm_rotate(x, gain, eps, table):
    """x [rows, heads, d]; gain [d] or None; table [rows, d / 2, 2] (cosine, sine) or None."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        if gain is not None:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
        if table is not None:
            h = x.shape[-1] // 2
            c, s = table[:, None, :, 0], table[:, None, :, 1]
            x = np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)
    return x


def fill_page(raw, scale, lo, new):
    """One head's keys or values of a page: raw uint8 [16, d], scale, first new slot, new values [n, d].  Returns (raw, scale, values), values
    [16, d]: what the new slots hold before their rounding."""
    raw, n = raw.copy(), len(new)
    finite = np.abs(new[np.isfinite(new)])
    s = 2.0 ** scale_exponent(finite.max(initial=0.0))
    if lo > 0:
        if scale >= s:
            s = scale
        else:
            raw[:lo] = to_e4m3(VALUES[raw[:lo]] * (scale / s))
    raw[lo:lo + n] = to_e4m3(new / s)
    return raw, s


def fork(table, held, length, parent, width_out, refs, free, room, n_pages):
    """Plain lists in and out.  Returns table_out, held_out, length_out, refs, free, missing, copies [(source, destination)]."""
    refs, free = list(refs), list(free)
    n = len(held)
    held = [min(max(h, 0), len(table[0]) if table else 0) for h in held]
    length = [min(max(x, 0), h * PAGE) for x, h in zip(length, held)]
    pages = [list(table[s][:held[s]]) for s in range(n)]
    kids = [[i for i, p in enumerate(parent) if p == s] for s in range(n)]
    out, lengths, copies, missing, taken = [], [], [], 0, set()
    for i, p in enumerate(parent):
        if not 0 <= p < n:
            out.append([]); lengths.append(0)
            continue
        full = length[p] // PAGE
        mine = (pages[p] if kids[p][0] == i else pages[p][:full])[:width_out]
        have = len(mine)
        want = min(-(-(length[p] + room) // PAGE), width_out)
        while len(mine) < want and free:
            page = free.pop()
            taken.add(page)
            if kids[p][0] != i and len(mine) == full and length[p] % PAGE and 0 <= pages[p][full] < n_pages:
                copies.append((pages[p][full], page))
            mine.append(page)
        missing += max(want - len(mine), 0)
        assert len(mine) >= have
        out.append(mine); lengths.append(min(length[p], len(mine) * PAGE))
    freed = set()
    for s in range(n):
        for j, page in enumerate(pages[s]):
            if not 0 <= page < n_pages:
                continue
            if not kids[s]:
                refs[page] -= 1
                if refs[page] == 0:
                    freed.add(page)
            elif j < length[s] // PAGE:
                refs[page] += len(kids[s]) - 1
    for page in taken:
        refs[page] = 1
    return out, [len(x) for x in out], lengths, refs, free + sorted(freed), missing, copies
