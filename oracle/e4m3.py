"""Numbers in 8 bits and the blocks of a cache that share a scale, in plain Python and float64, from the format's definition: sign, 4 bits of
exponent with bias 7, 3 of fraction; exponent 0 without the leading one; 0x7f and 0xff NaN.  A scale s stands for 2^(s - 127)."""
import numpy as np

_CODES = np.arange(256)
_EXP, _FRAC = (_CODES >> 3) & 15, _CODES & 7
VALUES = np.where(_EXP > 0, (8 + _FRAC) * 2.0 ** (_EXP - 10), _FRAC * 2.0 ** -9) * np.where(_CODES & 128, -1.0, 1.0)
VALUES[[0x7f, 0xff]] = np.nan


def decode(codes, scale):
    """codes uint8 [...], scale [...] or one number."""
    return VALUES[codes] * 2.0 ** (np.clip(np.asarray(scale, np.float64), 1, 254) - 127)


def encode(x):
    """Nearest code, ties to the even one; what no number is near to (over 464), and NaN, as 0x7f."""
    x = np.asarray(x, np.float64)
    grid, size = VALUES[:0x7f], np.abs(x)
    hi = np.clip(np.searchsorted(grid, np.where(np.isnan(size), 0, size)), 1, 0x7e)   # grid[hi - 1] < size <= grid[hi]
    up, down = grid[hi] - size, size - grid[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    code = np.where(size <= 464, code, 0x7f)
    return (code | np.where(np.signbit(x) & (size <= 464), 0x80, 0)).astype(np.uint8)


def least_scale(x):
    """The least scale, from 10 on, of a block whose values are x."""
    x = np.abs(np.asarray(x, np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    s = 10
    while top > 448 * 2.0 ** (s - 127):
        s += 1
    return s


def append(pagemap, k_scale, v_scale, block, seqs, cu, k_new, v_new, status, layer=0, n_tokens=None):
    """PagedMap.append for codes (pagemap.k, pagemap.v uint8) and their scales [layers, pages, blocks, hkv], changed in place."""
    page = pagemap.page
    for i, s in enumerate(seqs):
        if s < 0 or s >= len(pagemap.length) or status[i] != 0:
            continue
        n = int(cu[i + 1] - cu[i])
        by_block = {}
        for j in range(n):
            pos = int(pagemap.length[s]) - n + j
            if pos >= 0 and (n_tokens is None or cu[i] + j < n_tokens):
                by_block.setdefault(pos // block, []).append((pos, cu[i] + j))
        for b, tokens in by_block.items():
            p, first = pagemap.table[s, b * block // page], b * block % page
            older = range(first, tokens[0][0] % page)
            rows = [t for _, t in tokens]
            for codes, scales, new in ((pagemap.k, k_scale, k_new), (pagemap.v, v_scale, v_new)):
                for h in range(codes.shape[3]):
                    at = (layer, p, first // block, h)
                    had = int(scales[at])
                    scales[at] = max(least_scale(new[rows, h]), min(max(had, 1), 254) if len(older) else 0)
                    for slot in older:
                        if scales[at] != had:
                            codes[layer, p, slot, h] = encode(decode(codes[layer, p, slot, h], had) / 2.0 ** (float(scales[at]) - 127))
                    for pos, t in tokens:
                        codes[layer, p, pos % page, h] = encode(np.asarray(new[t, h], np.float64) / 2.0 ** (float(scales[at]) - 127))
