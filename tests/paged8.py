"""Caches in 8 bits for the tests, and the comparison with the 64-bit oracle."""
import numpy as np

import paper_2510_10620_amd as P
from oracle import e4m3
from oracle import paged as OP

NAN = float("nan")


def dtype_of(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def f64(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def ints(x):
    import torch
    return torch.tensor([int(y) for y in x], dtype=torch.int32, device="cuda")


def randn(shape, io, seed, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype_of(io)).cuda()


def make_cache(lens, page, block, hkv, d, io="bf16", layers=1, spare=3, extra_seqs=1, width=None, seed=0, layout="token"):
    """A cache whose sequences lie on pages in any order; slots without a token hold NaN, blocks without one scales that are no scales.  layout as
    in the tests of the other dtypes, or "mixed": K as "token", V as "head".  -> (Cache, sequences of `lens`)"""
    import torch
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in lens]
    n_pages, n_seqs, blocks = sum(used) + spare, len(lens) + extra_seqs, page // block
    width = width or max(1, max(used))
    where, names = rng.permutation(n_pages), rng.permutation(n_seqs)[:len(lens)]
    table, ref, length = np.full((n_seqs, width), -1, np.int32), np.zeros(n_pages, np.int32), np.zeros(n_seqs, np.int32)
    filled = np.zeros((n_pages, page), bool)
    at = 0
    for s, n in enumerate(lens):
        table[names[s], : used[s]] = where[at: at + used[s]]
        length[names[s]] = n
        for x, p in enumerate(where[at: at + used[s]]):
            filled[p, : n - x * page] = True
        at += used[s]
    ref[where[:at]] = 1
    tensors = []
    for which in range(2):
        x = rng.standard_normal((layers, n_pages, page, hkv, d)) * 100
        codes = np.where(filled[None, :, :, None, None], e4m3.encode(np.clip(x, -448, 448)), 0x7f).astype(np.uint8)
        scales = np.where(filled.reshape(n_pages, blocks, block).any(2)[None, :, :, None], rng.integers(118, 122, (layers, n_pages, blocks, hkv)),
                          rng.choice([0, 255], (layers, n_pages, blocks, hkv))).astype(np.uint8)
        codes = torch.from_numpy(codes)
        if layout == "head" or (layout == "mixed" and which):
            y = torch.empty((layers, n_pages, hkv, page, d), dtype=torch.uint8, device="cuda").transpose(2, 3)
        elif layout == "gaps":
            y = torch.full((layers, n_pages, page, hkv + 1, d + 16), 0x7f, dtype=torch.uint8, device="cuda")[:, :, :, :hkv, :d]
        else:
            y = torch.empty(codes.shape, dtype=torch.uint8, device="cuda")
        tensors.append((y.copy_(codes).view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda()))
    (k, ks), (v, vs) = tensors
    return P.Cache(k, v, *(torch.from_numpy(a).cuda() for a in (ref, table, length)), k_scale=ks, v_scale=vs, io_dtype=dtype_of(io)), names


def infinite_at(cache, s, pos):
    """Token `pos` of sequence s stands for infinities in number 3 (+) and 4 (-) of V and in number 5 (+) of K, and for zeros else; so do the others of its block."""
    import torch
    page, block = cache.k.shape[2], cache.k.shape[2] // cache.k_scale.shape[2]
    p, slot = int(cache.page_table[s, pos // page]), pos % page
    at = slice(slot // block * block, slot // block * block + block)
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    k[0, p, at], v[0, p, at] = 0, 0
    cache.k_scale[0, p, slot // block], cache.v_scale[0, p, slot // block] = 247, 247
    k[0, p, slot, :, 5], v[0, p, slot, :, 3], v[0, p, slot, :, 4] = 0x7e, 0x7e, 0xfe
    return p, slot


class Held:
    """A cache's contents on the host: codes, scales and the page map."""

    def __init__(self, cache):
        import torch
        self.page, self.block = cache.k.shape[2], cache.k.shape[2] // cache.k_scale.shape[2]
        self.k, self.v = (x.view(torch.uint8).cpu().numpy().copy() for x in (cache.k, cache.v))
        self.ks, self.vs = (x.cpu().numpy().copy() for x in (cache.k_scale, cache.v_scale))
        self.table, self.length, self.ref = (x.cpu().numpy().copy() for x in (cache.page_table, cache.seq_len, cache.page_ref))

    def map(self):
        return OP.PagedMap(self.page, self.ref, self.table, self.length, self.k, self.v)

    def values(self, s, j, layer=0):
        """K and V of the tokens j of sequence s: (those whose page exists, k, v)"""
        j = np.asarray(j, np.int64)
        p = self.table[s][j // self.page] if len(j) else j
        real = (p >= 0) & (p < self.k.shape[1])
        j, p = j[real], p[real]
        slot = j % self.page
        return j, *(e4m3.decode(c[layer, p, slot], sc[layer, p, slot // self.block][:, :, None]) for c, sc in ((self.k, self.ks), (self.v, self.vs)))


def check_rows(cache, q, out, lse, scale, rows, window=0, sink=0, layer=0, weights=2.0 ** -15, held=None):
    """rows: (row of q, sequence, position) of every token; the other rows must hold NaN, as they did before the call.

    With u the half step of fp32 (2^-24), r that of the outputs' type, L keys of D dimensions: a score is off by at most (D + 4) u
    scale sum|q k| (the products and their sum, the scale, and log2 e in it; keys and queries go in without a rounding), the exponential by 4 u more, so a weight
    by e = 2 ((D + 4) u size + 4 u) of itself (its own score and the maximum's); the sums by L u; bf16: weights are held to `weights`.  The
    output is a quotient of two such sums over |v| and is rounded once."""
    held = held or Held(cache)
    bf16 = q.element_size() == 2
    u, r, d = 2.0 ** -24, 2.0 ** -8 if bf16 else 2.0 ** -24, q.shape[2]
    o, l, qq = f64(out), f64(lse), f64(q)
    others = np.setdiff1d(np.arange(q.shape[0]), [i for i, _, _ in rows])
    assert np.isnan(o[others]).all() and np.isnan(l[:, others]).all(), "a row that no place has was written"
    worst = 0.0
    for i, s, pos in rows:
        j, k, v = held.values(s, OP.seen_keys(pos + 1, window, sink), layer)
        ref, ref_l, mean, size = OP.attend(qq[i], k, v, scale)
        if not len(j):
            assert (o[i] == 0).all() and (l[:, i] == -np.inf).all(), f"row {i} sees no key"
            continue
        e = 2 * ((d + 4) * u * size + 4 * u) + 2 * len(j) * u + (weights if bf16 else 0)
        bad = np.abs(o[i] - ref) / (r * np.abs(ref) + 1.01 * (2 * e[:, None] * mean))
        assert bad.max() <= 1, f"row {i} (sequence {s}, position {pos}, {len(j)} keys): out is {bad.max():.2f} times its bound off"
        e = e - (weights if bf16 else 0)
        bad_l = np.abs(l[:, i] - ref_l) / (e + 2 * u * np.abs(ref_l) + 4 * u)
        assert bad_l.max() <= 1, f"row {i} (sequence {s}, position {pos}, {len(j)} keys): LSE is {bad_l.max():.2f} times its bound off"
        worst = max(worst, bad.max(), bad_l.max())
    return worst
