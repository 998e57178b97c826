"""The operators of a paged key-value cache held in 8 bits, as cases whose time and results can be measured.

The cache is that of perf/operators.py with keys and values as e4m3 numbers: `block` neighbouring tokens of a page share a scale for each
KV head, a power of two that is kept as its biased exponent in one byte, [layers, pages, page / block, KV heads]; a number stands for
code x 2^(exponent - 127).  Queries, new keys and values and outputs are bf16 or fp32.  A case is one pass through

  attend    attention of one new token per sequence over its pages
  chunk     attention of the last tokens of every sequence (a piece of a prompt, tokens to be verified) over its pages, causal
  extend    room for new tokens, their keys and values rounded into the pages, and the tail of every sequence read back
  read      the last tokens of every sequence read out of the pages, packed

in its plain form, or, with `own`, through the entry points of paper_2510_10620_amd.  Head counts, lengths, masks and page sizes are those
of the package's workloads, tests and benchmark.
"""
import math

import numpy as np
import torch

own = False

# Fields of a case.
#   rows     sequences that hold tokens; the tokens before the new ones are drawn from [lo, hi], evenly or (median > 0) log-normally
#   new      chunk, extend, read: most new (read) tokens of a sequence (1: one token each; else from a quarter of it up to it)
#   pad      places of the batch that name no sequence (a batch padded to a fixed size)
#   block    tokens that share a scale
#   window, sink   sliding window (0: none) and attention sink
_BASE = dict(do="attend", rows=32, lo=512, hi=8192, median=2048, len_seed=2, pad=0, page=64, block=64, new=1, hq=32, hkv=8, d=128, io="bf16",
             window=0, sink=0)


def _case(name, **kw):
    return dict(_BASE, name=name, **kw)


def listed():
    return [
        # one chat with a few hundred tokens, two small heads: all latency
        _case("attend_one_short", rows=1, lo=300, hi=300, median=0, page=16, block=16, hq=4, hkv=2, d=64),
        # an ordinary batch of chats of mixed lengths, padded to a fixed size
        _case("attend_batch", pad=3),
        # many chats at once: the largest call
        _case("attend_many", rows=224, lo=64, hi=16384, median=4096, page=32, block=32),
        # one document of the largest length under fp32 activations
        _case("attend_long_f32", rows=1, lo=131067, hi=131067, median=0, page=256, block=128, io="f32"),
        # drafted tokens of a batch of chats, verified in one pass
        _case("chunk_verify", do="chunk", rows=16, new=5, page=16, block=16, pad=1),
        # a piece of a long prompt behind the pieces before it
        _case("chunk_prompt", do="chunk", rows=1, lo=30720, hi=30720, median=0, new=2048),
        # prompts of a batch, some of them behind earlier turns, under a sliding window with a sink
        _case("chunk_ragged_window", do="chunk", rows=7, lo=0, hi=6000, median=0, new=1500, page=20, block=10, hq=16, hkv=4, d=64, window=1024, sink=64),
        # a small model's drafted tokens, fp32
        _case("chunk_few_f32", do="chunk", rows=4, lo=1, hi=900, median=0, new=7, hq=8, hkv=2, d=64, page=32, block=8, io="f32"),
        # a decoding step of a batch: one token each
        _case("extend_step", do="extend", rows=64, pad=2, page=16, block=16, lo=16, hi=2048, median=512),
        # prompts put into the cache after their prefill, some of them behind earlier turns
        _case("extend_prompts", do="extend", rows=9, lo=0, hi=3000, median=0, new=8192),
        # the tails of a few sequences, for a kernel that wants them packed
        _case("read_few", do="read", rows=8, lo=0, hi=300, median=0, new=33, page=16, block=16, hkv=2, d=64, io="f32"),
        # whole contexts taken out of the cache
        _case("read_many", do="read", rows=24, lo=0, hi=0, median=0, new=8192, page=128, block=64),
    ]


def _loguniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["attend", "attend", "attend", "chunk", "chunk", "chunk", "extend", "extend", "read"])
    heads = [(32, 8), (32, 8), (16, 4), (8, 2), (4, 1), (24, 6), (16, 16), (16, 1), (1, 1), (64, 2)]
    hq, hkv = rng.choice(heads)
    page = rng.choice([8, 16, 16, 20, 32, 64, 64, 100, 128, 256])
    block = rng.choice([b for b in (1, 2, 5, 8, 16, 16, 32, 32, 64, 64, 100, 128, 256) if page % b == 0])
    c = dict(_BASE, do=do, hq=hq, hkv=hkv, d=rng.choice([128, 128, 128, 64, 32]), io=rng.choice(["bf16", "bf16", "bf16", "f32"]),
             len_seed=rng.randrange(1 << 20), page=page, block=block, pad=rng.choice([0, 0, 1, 3]), median=0)
    if do == "attend":
        c["hi"] = _loguniform(rng, 1, 131072)
        most = max(1, min(256, 1000000000 // (c["hi"] * 2 * hkv * c["d"])))
        c.update(rows=_loguniform(rng, 1, most), lo=rng.choice([0, max(1, c["hi"] // 3), c["hi"]]))
    elif do == "chunk":
        c["new"] = _loguniform(rng, 2, 2048)
        room = 1 << 30                                             # padded scores of the plain form
        c["hi"] = _loguniform(rng, 1, max(1, min(32768, room // (hq * c["new"]) - c["new"])))
        longest = c["hi"] + c["new"]
        most = min(64, room // (hq * c["new"] * longest), 1000000000 // (2 * hkv * c["d"] * longest))
        c.update(lo=rng.choice([0, c["hi"] // 2, c["hi"]]), rows=_loguniform(rng, 1, max(1, most)))
    elif do == "extend":
        c.update(rows=_loguniform(rng, 1, 256), lo=0, hi=_loguniform(rng, 1, 4096))
        if rng.random() < 0.5:
            c.update(rows=_loguniform(rng, 1, 9), new=_loguniform(rng, 2, 65536 // max(8, hkv)))
    else:
        c.update(rows=_loguniform(rng, 1, 24), lo=0, hi=_loguniform(rng, 1, 2048), new=_loguniform(rng, 1, 65536 // max(8, hkv)))
    if do in ("attend", "chunk") and rng.random() < 0.25:
        c.update(window=_loguniform(rng, 1, 8192), sink=rng.choice([0, 1, 16, 64, 200]))
    return c


def _sizes(c):
    """(tokens held, new tokens, pages in use, pages of the cache, entries of a row of the table, sequences of the cache)
    attend, chunk, read: the new tokens are held already."""
    r = np.random.default_rng(c["len_seed"])
    if c["median"]:
        lens = np.clip(np.round(np.exp(r.normal(math.log(c["median"]), 1.0, c["rows"]))), c["lo"], c["hi"]).astype(np.int64)
    else:
        lens = r.integers(c["lo"], c["hi"] + 1, c["rows"])
    new = np.ones(c["rows"], dtype=np.int64) if c["new"] == 1 else r.integers(max(1, c["new"] // 4), c["new"] + 1, c["rows"])
    last = lens + (new if c["do"] != "attend" else 0)
    held = lens if c["do"] == "extend" else last
    used = -(-held // c["page"])
    n_pages = int((-(-last // c["page"])).sum()) + max(4, int(used.sum()) // 4)
    return held, new, used, n_pages, max(1, int((-(-last // c["page"])).max())), c["rows"] + 1


def _tail(c):
    """extend: how many tokens of every sequence are read back: the new ones and those that share a scale with the first of them."""
    held, new = _sizes(c)[:2]
    return new + held % c["block"]


def prepare(case, seed):
    c = case
    held, new, used, n_pages, width, n_seqs = _sizes(c)
    page, block, hkv, d = c["page"], c["block"], c["hkv"], c["d"]
    dtype = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)

    def randn(*shape):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)

    def stored():
        """Keys or values as a cache holds them: tokens of different sizes, scales that reach 448 units in the largest."""
        x = torch.empty((n_pages, page // block, block, hkv, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        x *= torch.empty((n_pages, page // block, 1, hkv, 1), dtype=torch.bfloat16, device="cuda").uniform_(0.5, 1.5, generator=gen)
        e = _exponent(x.abs().amax((2, 4)))
        codes = (x * _two_to(-e[:, :, None, :, None])).to(torch.float8_e4m3fn).view(1, n_pages, page, hkv, d)
        return codes, (e + 127).to(torch.uint8).view(1, n_pages, page // block, hkv).contiguous()

    # the cache as it is after some time: a sequence's pages lie anywhere
    where = rng.permutation(n_pages)[: int(used.sum())]
    names = rng.permutation(n_seqs)[: c["rows"]]
    table = np.full((n_seqs, width), -1, dtype=np.int32)
    ref = np.zeros(n_pages, dtype=np.int32)
    length = np.zeros(n_seqs, dtype=np.int32)
    ref[where] = 1
    length[names] = held
    at = np.concatenate([[0], np.cumsum(used)])
    for i, s in enumerate(names):
        table[s, : used[i]] = where[at[i]: at[i + 1]]
    # the page map in one allocation, so that a pass can start from the same map as the one before
    ints0 = torch.from_numpy(np.concatenate([ref, length, table.reshape(-1)])).cuda()
    ints = ints0.clone()
    (k, ks), (v, vs) = stored(), stored()
    s = dict(c, ints=ints, ints0=ints0, k=k, v=v, k_scale=ks, v_scale=vs, ref=ints[:n_pages], length=ints[n_pages: n_pages + n_seqs],
             table=ints[n_pages + n_seqs:].view(n_seqs, width), longest=int(held.max()), scale=1.0 / math.sqrt(d))

    def on_gpu(x):
        return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()

    def begins(x):
        return on_gpu(np.concatenate([[0], np.cumsum(x), np.full(c["pad"], x.sum())]))

    n = c["rows"] + c["pad"]
    s["seqs"] = on_gpu(np.concatenate([names, np.full(c["pad"], -1)]))
    tokens = n if c["do"] == "attend" else int(new.sum())
    s["n_new"], s["cu_new"], s["most"] = on_gpu(np.concatenate([new, np.zeros(c["pad"])])), begins(new), int(new.max())
    if c["do"] in ("attend", "chunk"):
        s["q"] = randn(tokens, c["hq"], d)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((c["hq"], tokens), dtype=torch.float32, device="cuda")
    else:
        if c["do"] == "extend":
            s["k_new"], s["v_new"] = randn(tokens, hkv, d), randn(tokens, hkv, d)
            s["status"] = torch.zeros(n, dtype=torch.int32, device="cuda")
            s["cu_tail"], tokens = begins(_tail(c)), int(_tail(c).sum())
        else:
            s["cu_tail"] = s["cu_new"]
        s["k_out"], s["v_out"] = (torch.zeros((tokens, hkv, d), dtype=dtype, device="cuda") for _ in range(2))
    if own:
        import paper_2510_10620_amd as P
        s["P"], s["cache"] = P, P.Cache(k, v, s["ref"], s["table"], s["length"], k_scale=ks, v_scale=vs, io_dtype=dtype)
        if c["do"] == "attend":
            s["ws"] = torch.empty(P.dcp_paged_attn_workspace_bytes(s["cache"], n, c["hq"]), dtype=torch.uint8, device="cuda")
        elif c["do"] == "chunk":
            s["ws"] = torch.empty(P.dcp_paged_attn_chunk_workspace_bytes(s["cache"], n, tokens, c["hq"]), dtype=torch.uint8, device="cuda")
    return s


def run(state):
    s = state
    do = s["do"]
    if do == "attend":
        if own:
            s["P"].dcp_paged_attn_fwd(s["cache"], s["q"], s["out"], s["lse"], s["scale"], s["ws"], seqs=s["seqs"], window=s["window"], sink=s["sink"])
        else:
            _attend(s, torch.arange(s["seqs"].shape[0] + 1, device="cuda"), 1)
        return {"out": s["out"], "lse": s["lse"]}
    if do == "chunk":
        if own:
            s["P"].dcp_paged_attn_chunk_fwd(s["cache"], s["q"], s["out"], s["lse"], s["scale"], s["ws"], s["cu_new"], seqs=s["seqs"],
                                            window=s["window"], sink=s["sink"])
        else:
            _attend(s, s["cu_new"].long(), s["most"])
        return {"out": s["out"], "lse": s["lse"]}
    got = {"k": s["k_out"], "v": s["v_out"]}
    if do == "extend":
        s["ints"].copy_(s["ints0"])
        got.update(status=s["status"], ref=s["ref"], length=s["length"], table=s["table"])
        if own:
            s["P"].dcp_cache_reserve(s["cache"], s["seqs"], s["status"], n_new=s["n_new"])
            s["P"].dcp_cache_append(s["cache"], s["k_new"], s["v_new"], seqs=s["seqs"], cu_new=s["cu_new"], status=s["status"])
        else:
            _reserve(s)
            _append(s)
    if own:
        s["P"].dcp_cache_read(s["cache"], s["k_out"], s["v_out"], seqs=s["seqs"], cu_new=s["cu_tail"])
    else:
        _read(s)
    return got


# ------------------------------------------------------------------------------------------------- plain forms
def _two_to(e):
    """2^e from its bits, e from -126 to 127 (a power computed on the GPU is not exact)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponent(top):
    """The least e from -117 on with top <= 448 x 2^e."""
    m, x = torch.frexp(top.float())
    return torch.where(m == 0, -117, torch.where(m <= 0.875, x - 9, x - 8)).clamp(min=-117).to(torch.int32)


def _attend(s, cu, most):
    """Attention of the tokens [cu[i], cu[i + 1]) of q, the last ones of place i's sequence (at most `most`)."""
    seqs, page, block, hkv, d, hq = s["seqs"], s["page"], s["block"], s["hkv"], s["d"], s["hq"]
    row, n, per = seqs.clamp(min=0).long(), seqs.shape[0], s["hq"] // s["hkv"]
    keys = max(1, s["longest"])
    width = -(-keys // page)
    at = s["table"][row, :width].clamp(min=0).long()

    def gathered(codes, exponents):                                # [n, KV heads, keys, D]
        x = codes[0].view(torch.uint8)[at].view(torch.float8_e4m3fn).float().view(n, width * page // block, block, hkv, d)
        x = x * _two_to(exponents[0][at].view(n, -1, 1, hkv, 1).int() - 127)
        return x.view(n, width * page, hkv, d).transpose(1, 2)

    length = torch.where(seqs >= 0, s["length"][row], torch.zeros_like(seqs)).long()
    t = torch.arange(most, device=seqs.device)
    count = cu[1:] - cu[:-1]
    mine = (t < count[:, None]) & (seqs >= 0)[:, None]             # [n, most]: the query is there
    index = (cu[:-1, None] + t).clamp(max=s["q"].shape[0] - 1)
    pos = (length - count)[:, None] + t if s["do"] == "chunk" else (length - 1)[:, None]
    j = torch.arange(width * page, device=seqs.device)
    seen = (j <= pos[:, :, None]) & (j < length[:, None, None])    # [n, most, keys]
    if s["window"]:
        seen &= (j > pos[:, :, None] - s["window"]) | (j < s["sink"])
    q = s["q"][index].float().view(n, most, hkv, per, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, per * most, d)
    score = torch.matmul(q * s["scale"], gathered(s["k"], s["k_scale"]).transpose(2, 3).contiguous()).view(n, hkv, per, most, width * page)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, hkv, per * most, -1), gathered(s["v"], s["v_scale"]).contiguous()).view(n, hkv, per, most, d)
    out = (out / torch.where(total == 0, torch.ones_like(total), total)).permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(n, most, hq)
    s["out"][index[mine]] = out[mine].to(s["out"].dtype)
    s["lse"][:, index[mine]] = lse[mine].t()


def _reserve(s):
    seqs, page, table, length, ref = s["seqs"], s["page"], s["table"], s["length"], s["ref"]
    row, named = seqs.clamp(min=0).long(), seqs >= 0
    new = torch.where(named, s["n_new"], torch.zeros_like(seqs))
    first = (length[row] + page - 1) // page
    need = torch.where(named, (length[row] + new + page - 1) // page - first, torch.zeros_like(seqs))
    free = torch.argsort((ref > 0).to(torch.int32), stable=True)   # the free pages first
    last = need.cumsum(0)
    served = (need == 0) | (last <= (ref <= 0).sum())
    k = torch.arange(s["most"] // page + 2, device=seqs.device)
    takes = served[:, None] & (k < need[:, None])
    got = free[((last - need)[:, None] + k).clamp(max=free.shape[0] - 1)][takes]
    table.view(-1)[(row[:, None] * table.shape[1] + first[:, None] + k)[takes]] = got.to(torch.int32)
    ref[got] = 1
    length.index_add_(0, row, torch.where(served, new, torch.zeros_like(new)))
    s["status"].copy_(torch.where(served, 0, 1))


def _token_places(s, cu, n_tokens):
    """(token exists, its page, its slot, its number in the sequence, its place's first token) for rows that end the sequences."""
    seqs, page = s["seqs"], s["page"]
    t = torch.arange(n_tokens, device=seqs.device)
    i = torch.searchsorted(cu, t, right=True) - 1
    row = seqs[i].clamp(min=0).long()
    pos = s["length"][row].long() - cu[i + 1] + t
    return (seqs[i] >= 0) & (pos >= 0), s["table"][row, pos.clamp(min=0) // page].long(), pos % page, pos, pos - t + cu[i]


def _append(s):
    page, block = s["page"], s["block"]
    goes, to, slot, pos, first = _token_places(s, s["cu_new"].long(), s["k_new"].shape[0])
    unit = to * (page // block) + slot // block                    # the token's block, of all blocks of the layer
    held = first - first // block * block                          # tokens that the place's first block holds already
    old_in = goes & (pos // block == first // block) & (held > 0)  # tokens that share a block with older ones
    for_all = torch.arange(page // block * s["k"].shape[1], device=to.device)
    older = torch.zeros_like(for_all).index_copy_(0, unit[old_in], held[old_in])         # older tokens of every block
    fresh = torch.zeros_like(for_all).index_fill_(0, unit, 1) > 0                        # blocks that get new tokens
    _append_one(s, s["k"], s["k_scale"], s["k_new"], unit, slot, older, fresh)
    _append_one(s, s["v"], s["v_scale"], s["v_new"], unit, slot, older, fresh)


def _append_one(s, codes, exponents, x, unit, slot, older, fresh):
    block, hkv, d = s["block"], s["hkv"], s["d"]
    x = x.float()
    size = x.abs().amax(-1)                                        # [tokens, KV heads]
    top = torch.zeros((older.shape[0], hkv), device=x.device).index_reduce_(0, unit, size, "amax")
    e = exponents.view(-1, hkv).int() - 127
    want = torch.where(older[:, None] > 0, torch.maximum(_exponent(top), e), _exponent(top))
    now = torch.where(fresh[:, None], want, e)
    units = codes.view(torch.uint8).view(-1, block, hkv, d)
    changed = torch.nonzero((older > 0) & (now > e).any(1)).squeeze(1)
    was = units[changed].view(torch.float8_e4m3fn).float()
    again = (was * _two_to((e - now)[changed][:, None, :, None])).to(torch.float8_e4m3fn).view(torch.uint8)
    stays = torch.arange(block, device=x.device)[:, None, None] >= older[changed][:, None, None, None]
    units[changed] = torch.where(stays, units[changed], again)
    units[unit, slot % block] = (x * _two_to(-now[unit][:, :, None])).to(torch.float8_e4m3fn).view(torch.uint8)
    exponents.view(-1, hkv).copy_((now + 127).to(torch.uint8))


def _read(s):
    cu = s["cu_tail"].long()
    there, page, slot, _, _ = _token_places(s, cu, s["k_out"].shape[0])
    for_one = there[:, None, None]

    def numbers(codes, exponents):
        x = codes[0].view(torch.uint8)[page, slot].view(torch.float8_e4m3fn).float()
        return x * _two_to(exponents[0][page, slot // s["block"]][:, :, None].int() - 127)

    s["k_out"].copy_(torch.where(for_one, numbers(s["k"], s["k_scale"]).to(s["k_out"].dtype), s["k_out"]))
    s["v_out"].copy_(torch.where(for_one, numbers(s["v"], s["v_scale"]).to(s["v_out"].dtype), s["v_out"]))


# ------------------------------------------------------------------------------------------------- the least work
def work(case):
    c = case
    held, new, used, n_pages, width, n_seqs = _sizes(c)
    e = 2 if c["io"] == "bf16" else 4
    token, d, hq, page = c["hkv"] * c["d"], c["d"], c["hq"], c["page"]        # bytes of K or of V, one token
    if c["do"] in ("attend", "chunk"):
        count = np.minimum(1, held) if c["do"] == "attend" else new
        keys = pairs = 0
        for n, q in zip(held.tolist(), count.tolist()):
            if not n or not q:
                continue
            w, k = c["window"] or n, c["sink"]
            pos = np.arange(n - q, n)
            lo = np.maximum(pos + 1 - w, 0)
            pairs += int((pos + 1 - lo + np.minimum(k, lo)).sum())
            keys += n - int(lo[0]) + min(k, int(lo[0]))
        scales = 2 * keys * c["hkv"] / c["block"]
        rows = c["rows"] if c["do"] == "attend" else int(new.sum())
        return {"bytes": float(2 * keys * token + scales + rows * hq * (2 * d * e + 4) + 4 * keys / page), "flops": 4.0 * pairs * hq * d}
    tail = int(new.sum() if c["do"] == "read" else _tail(c).sum())
    moved = 2 * tail * token * (1 + e) + 2 * tail * c["hkv"] / c["block"]     # read back
    if c["do"] == "extend":
        taken = int((-(-(held + new) // page) - used).sum())
        n = int(new.sum())
        moved += 2 * n * token * (1 + e) + 2 * n * c["hkv"] / c["block"]      # written
        moved += 4.0 * (2 * n_pages + 2 * n_seqs + 2 * n_seqs * width) + 4.0 * n_pages + 8.0 * taken + 16.0 * c["rows"]
    return {"bytes": float(moved), "flops": 0.0}


# ------------------------------------------------------------------------------------------------- 64 bits
def _power(e):
    """2^e from its bits, in 64."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid(x):
    """x on the grid of e4m3: steps of 2^-3 of the power of two below it, of 2^-9 below 2^-6; half a step goes to the even neighbour."""
    power = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60)))
    power = torch.where(_power(power) > x.abs(), power - 1, power)
    power = torch.where(_power(power + 1) <= x.abs(), power + 1, power).clamp(min=-6)
    return torch.round(x / _power(power - 3)) * _power(power - 3)


def _values(codes, exponents, table, length, page, block):
    """The tokens of one sequence as 64-bit numbers [tokens, KV heads, D]."""
    j = torch.arange(length, device="cuda")
    pages = torch.from_numpy(table.astype(np.int64)).cuda()[torch.div(j, page, rounding_mode="floor")]
    x = codes[0].view(torch.uint8)[pages, j % page].view(torch.float8_e4m3fn).double()
    return x * _power(exponents[0][pages, torch.div(j % page, block, rounding_mode="floor")].int() - 127)[:, :, None]


def exact(case, seed):
    s = prepare(case, seed)
    page, block, per = s["page"], s["block"], s["hq"] // s["hkv"]
    table, length, names, cu = s["table"].cpu().numpy().copy(), s["length"].tolist(), s["seqs"].tolist(), s["cu_new"].tolist()
    if s["do"] in ("attend", "chunk"):
        out, lse = s["out"].double(), s["lse"].double()
        for i, r in enumerate(names):
            if r < 0:
                continue
            n = length[r]
            a, b = (i, i + 1) if s["do"] == "attend" else (cu[i], cu[i + 1])
            k, v = (_values(s[x], s[x + "_scale"], table[r], n, page, block) for x in "kv")
            key, pos = torch.arange(n, device="cuda")[None], torch.arange(n - (b - a), n, device="cuda")[:, None]
            hidden = key > pos
            if s["window"]:
                hidden |= (pos - key >= s["window"]) & (key >= s["sink"])
            for h in range(s["hq"]):
                if n == 0:
                    out[a:b, h], lse[h, a:b] = 0.0, -math.inf
                    continue
                z = (s["q"][a:b, h].double() @ k[:, h // per].t().contiguous()) * s["scale"]
                z[hidden] = -math.inf
                lse[h, a:b] = torch.logsumexp(z, 1)
                out[a:b, h] = torch.softmax(z, 1) @ v[:, h // per].contiguous()
        return {"out": out, "lse": lse}
    got = {}
    if s["do"] == "extend":
        ref, status, was = s["ref"].tolist(), [], list(length)
        free, full = [p for p in range(len(ref)) if ref[p] == 0], False
        for i, r in enumerate(names):
            status.append(0)
            if r < 0:
                continue
            have, new = -(-length[r] // page), cu[i + 1] - cu[i]
            need = -(-(length[r] + new) // page) - have
            if need and (full or need > len(free)):
                status[-1], full = 1, True
                continue
            table[r, have: have + need] = free[:need]
            for p in free[:need]:
                ref[p] = 1
            del free[:need]
            length[r] += new
        got = dict(status=torch.tensor(status, dtype=torch.int32), ref=torch.tensor(ref, dtype=torch.int32),
                   length=torch.tensor(length, dtype=torch.int32), table=torch.from_numpy(table))
    tails = s["cu_tail"].tolist()
    for name in "kv":
        x = s[name + "_out"].double()
        for i, r in enumerate(names):
            a, b = tails[i], tails[i + 1]
            if r < 0 or a == b:
                continue
            if s["do"] == "read":
                x[a:b] = _values(s[name], s[name + "_scale"], table[r], length[r], page, block)[length[r] - (b - a):]
                continue
            if status[i]:
                return None
            older = (b - a) - (cu[i + 1] - cu[i])                  # they fill a block with the first new ones
            all_of = s[name + "_new"][cu[i]: cu[i + 1]].double()
            least = torch.full((-(-(b - a) // block), s["hkv"]), -117.0, dtype=torch.float64, device="cuda")
            if older:
                before = _values(s[name], s[name + "_scale"], table[r], was[r], page, block)[was[r] - older:]
                all_of = torch.cat([before, all_of])
                least[0] = s[name + "_scale"][0, table[r, was[r] // page], was[r] % page // block].double() - 127
            for y in range(least.shape[0]):                        # block by block, from the first one's begin
                part = all_of[y * block: (y + 1) * block]
                size = part[older if y == 0 else 0:].abs().amax((0, 2))
                e = least[y].clone()
                while bool((size > 448 * _power(e)).any()):
                    e = torch.where(size > 448 * _power(e), (e + 1).maximum(torch.floor(torch.log2(size / 449))), e)
                x[a + y * block: a + y * block + part.shape[0]] = _grid(part / _power(e)[None, :, None]) * _power(e)[None, :, None]
        got[name] = x
    return got
