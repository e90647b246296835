"""The attention block ahead of a synchronisation, as measurable cases: keys and values held in 4 bits.

A tensor-parallel device computes attention over its own heads, multiplies by its rows of the output projection and
synchronises the partial sums.  The operators here are what comes before that product:

  append     a step's keys and values go into the pages of the cache in 4 bits, queries and keys rotated to their
             positions on the way; then the batch's own rows are read back, which is what the cache now holds
  attention  the step's queries attend to the pages: causal, optionally only to a window of recent positions and to
             the first few positions of the sequence

The cache (one layer) is [pages][kv heads][page size / 16] blocks of 16 positions; a block is 16 rows of dim/2 bytes of
key codes (code d of a row is the low nibble of byte d/2 if d is even, else the high one), 16 rows of value codes, 16
words for the keys and 16 for the values.  A word holds BF16 `step` (low half) and BF16 `low` (high half), and a code c
stands for low + step * c.  Position t of a sequence is position t % page size of page table[t // page size].
A step brings n new positions of every sequence, the last ones of its `length`: rows start[s] .. start[s+1] - 1.

Head counts are those of the repository's workloads (5120 features = 40 heads of 128 over 4 devices, 32 query and 16
key heads of 128 over 8, 8192 features = 64 heads) and the ranges around them.
"""
import math

import numpy as np
import torch

own = False     # set by whoever measures: False, the plain forms; True, the framework's calls

BLOCK = 16              # positions of a block of the cache
MIN_STEP = 2.0 ** -60   # smallest step, and the smallest in relation to the vector's largest magnitude
REL_STEP = 2.0 ** -16


def _case(name, op, heads, kv_heads, dim, page, seqs, new, length, window=0, first=0, rot=0, interleaved=False, pad=0):
    """new, length: (smallest, largest) over the sequences.  rot: rotated values of a head.  pad: rows behind the last sequence."""
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "seqs": seqs, "new_lo": new[0], "new_hi": new[1],
         "len_lo": length[0], "len_hi": length[1], "window": window, "first": first, "rot": rot, "interleaved": interleaved, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one generated token of one conversation, on one of 4 devices: nothing but latency
        _case("append_token", "append", 10, 10, 128, 16, 1, (1, 1), (777, 777), rot=128),
        # the decode batch of 64 sequences on one of 8 devices
        _case("append_decode", "append", 4, 2, 128, 32, 64, (1, 1), (64, 8000), rot=128),
        # the headline prompt on one of 4 devices
        _case("append_prompt", "append", 10, 10, 128, 64, 1, (2048, 2048), (2048, 2048), rot=128),
        # a ragged batch of prompts on one device that holds all heads; adjacent pairs rotated, the rest of a head left alone
        _case("append_ragged", "append", 64, 8, 128, 16, 13, (1, 1300), (500, 4000), rot=64, interleaved=True, pad=5),
        # one conversation, one token: latency
        _case("decode_token", "attention", 10, 10, 128, 16, 1, (1, 1), (777, 777)),
        # the decode batch of 64 on one of 8 devices, ragged
        _case("decode_batch", "attention", 4, 2, 128, 32, 64, (1, 1), (64, 8000)),
        # long contexts on a device that holds all heads: the largest cache
        _case("decode_long", "attention", 64, 8, 128, 64, 32, (1, 1), (16384, 32768)),
        # the same batch where a layer sees a window and the first positions; pages that left the window are gone
        _case("decode_window", "attention", 32, 16, 128, 32, 64, (1, 1), (2000, 16384), window=4096, first=4),
        # four drafted tokens a sequence to verify, heads of 64
        _case("verify_drafts", "attention", 32, 4, 64, 16, 24, (2, 4), (300, 9000)),
        # the headline prompt on one of 4 devices
        _case("prompt", "attention", 10, 10, 128, 64, 1, (2048, 2048), (2048, 2048)),
        # a chunk of a long prompt beside sequences that decode
        _case("chunk_and_decode", "attention", 32, 8, 128, 32, 9, (1, 700), (900, 12000), pad=3),
        # long prompts, window and first positions: the most arithmetic
        _case("prompt_window", "attention", 32, 16, 128, 128, 2, (8000, 8191), (8000, 8191), window=4096, first=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 5, 8, 10, 16])
    group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 12, 16]) if kv <= 4 else rng.choice([1, 2, 4, 5, 8])
    heads, page = kv * group, rng.choice([16, 32, 64, 128])
    if rng.random() < 0.35:
        seqs = _log(rng, 1, 200)
        new = _log(rng, 1, max(1, min(4000, 16000 // seqs)))
        hi = new + _log(rng, 1, 8000)
        lo = rng.randint(max(1, hi // 3), hi)
        return _case("", "append", heads, kv, dim, page, seqs, (rng.randint(1, new), new), (lo, hi),
                     rot=rng.choice([16, dim // 2, dim, dim]), interleaved=rng.random() < 0.4, pad=rng.choice([0, 0, 7]))
    window = rng.choice([0, 0, 1, _log(rng, 5, 5000)])
    first = rng.choice([0, 1, 4, 77]) if window else 0
    kind = rng.random()
    if kind < 0.55:                      # decoding, at most the largest listed cache
        seqs = _log(rng, 1, 128)
        new = rng.choice([1, 1, 1, 2, 5])
        hi = _log(rng, 10, min(40000, 24 * 32768 * 8 // (seqs * kv)))
        return _case("", "attention", heads, kv, dim, page, seqs, (1, new), (max(1, hi // rng.choice([1, 2, 9])), hi), window, first, pad=rng.choice([0, 0, 2]))
    seqs = _log(rng, 1, 6)               # prompts and chunks
    new = _log(rng, 6, 5000 // seqs)
    hi = min(new + rng.choice([0, 0, _log(rng, 1, 6000)]), 9000)
    return _case("", "attention", heads, kv, dim, page, seqs, (rng.randint(1, new), new), (new, hi), window, first, pad=rng.choice([0, 0, 2]))


def _sizes(c):
    """New positions and lengths of the sequences: spread over their ranges, both ends among them where there are two."""
    i = np.arange(c["seqs"])
    spread = lambda lo, hi, step, at: np.where(i == at, hi, lo + np.floor((hi - lo + 1) * np.modf(i * step)[0])).astype(np.int64)  # noqa: E731
    new = spread(c["new_lo"], c["new_hi"], 0.7548776662466927, 0)
    length = np.maximum(spread(c["len_lo"], c["len_hi"], 0.5698402909980532, min(1, c["seqs"] - 1)), new)
    return new, length


def _visible(c):
    """Per sequence: visible (query, position) pairs and positions that any query sees."""
    pairs, seen = [], []
    for n, ln in zip(*_sizes(c)):
        p = np.arange(ln - n, ln)
        lo = np.maximum(0, p - c["window"] + 1) if c["window"] else np.zeros_like(p)
        pairs.append(int((p + 1 - lo).sum() + np.minimum(lo, c["first"]).sum()))
        seen.append(int(ln - lo[0] + min(lo[0], c["first"])))
    return sum(pairs), sum(seen)


def work(case):
    new, _ = _sizes(case)
    T, D, hq, hk = int(new.sum()), case["dim"], case["heads"], case["kv_heads"]
    entry = hk * (D + 8)          # bytes of a position: codes and words of keys and values
    if case["op"] == "append":
        # keys, values and queries in, rotated queries and cache entries out; the entries in again, their values out
        return {"bytes": T * (4 * hq * D + 4 * hk * D + 2 * entry + 4 * hk * D + 4 * case["rot"]), "flops": T * (6 * (hq + hk) * case["rot"] + 16 * hk * D)}
    pairs, seen = _visible(case)
    return {"bytes": seen * entry + 4 * T * hq * D, "flops": 4 * pairs * hq * D}


def _bf16(x):
    return x.to(torch.bfloat16)


def _quantised(x):
    """x [..., dim] float32 -> codes (uint8), step and low (both BF16) of each vector: 16 levels between its ends.  A vector that holds a
    NaN or whose range is beyond float32 becomes step 1, low NaN, codes 0."""
    lo, hi, top = x.amin(-1), x.amax(-1), x.abs().amax(-1)
    low = _bf16(lo)
    d = hi - low.float()
    bad = ~(d < math.inf) | ~torch.isfinite(low.float())
    step = _bf16(torch.maximum(torch.maximum(d * torch.tensor(1.0 / 15.0, device=x.device), top * REL_STEP), torch.tensor(MIN_STEP, device=x.device)))
    step, low = torch.where(bad, 1.0, step), torch.where(bad, math.nan, low)
    u = (x - low.float()[..., None]) / step.float()[..., None]
    codes = torch.where(bad[..., None], 0.0, u.round().clamp(0, 15)).to(torch.uint8)
    return codes, step, low


def _packed(codes, step, low):
    """Rows of dim/2 bytes, and words as 4 bytes each."""
    rows = codes[..., 0::2] | (codes[..., 1::2] << 4)
    return rows, torch.stack([step, low], -1).view(torch.uint8).reshape(*step.shape, 4)


def _views(c, cache):
    """Key rows, value rows, key words and value words of a cache, each [pages, kv heads, blocks, 16, bytes], sharing its memory."""
    half = c["dim"] // 2
    n = BLOCK * half
    b = cache.view(-1, c["kv_heads"], c["page"] // BLOCK, 2 * n + 8 * BLOCK)
    split = lambda x, w: x.unflatten(-1, (BLOCK, w))  # noqa: E731
    return split(b[..., :n], half), split(b[..., n:2 * n], half), split(b[..., 2 * n:2 * n + 4 * BLOCK], 4), split(b[..., 2 * n + 4 * BLOCK:], 4)


def _values(rows, words):
    """float32 values of rows of codes and their words."""
    codes = torch.stack([rows & 15, rows >> 4], -1).flatten(-2).float()
    w = words.contiguous().view(torch.bfloat16).float()
    return w[..., 1:2] + w[..., 0:1] * codes


def prepare(case, seed):
    c, g = case, torch.Generator("cuda").manual_seed(int(seed))
    dev, D, hq, hk, ps = "cuda", c["dim"], c["heads"], c["kv_heads"], c["page"]
    new, length = _sizes(c)
    T = int(new.sum()) + c["pad"]
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(dev)
    lengths = torch.from_numpy(length.astype(np.int32)).to(dev)
    per = -(-int(length.max()) // ps)                     # pages of a row of the table
    n_pages = int((-(-length // ps)).sum()) + 3           # some pages belong to nobody
    normal = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    # a head's channels differ in size, a few keep an offset or are large, as keys' do
    k_size = torch.exp(0.4 * normal(hk, D)) * torch.where(torch.rand(hk, D, generator=g, device=dev) < 0.02, 6.0, 1.0)
    k_off = normal(hk, D) * 0.3
    v_size = torch.exp(0.3 * normal(hk, D))
    # the pages of a sequence lie anywhere
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    have = torch.from_numpy((np.arange(per)[None] < (-(-length // ps))[:, None])).to(dev)
    table = torch.full((c["seqs"], per), -1, dtype=torch.int32, device=dev)
    table[have] = order[: int((-(-length // ps)).sum())]
    if c["window"]:                                       # and pages that no query sees any more are gone
        seen_from = torch.from_numpy(np.maximum(0, length - new - c["window"] + 1)).to(dev)
        last = (torch.arange(per, device=dev)[None] + 1) * ps
        gone = (last <= seen_from[:, None]) & (torch.arange(per, device=dev)[None] * ps >= c["first"])
        table[gone] = -1
    cache = torch.empty(n_pages * hk * (ps // BLOCK) * (BLOCK * (D + 8)), dtype=torch.uint8, device=dev)
    views = _views(c, cache)
    chunk = max(1, (1 << 27) // (hk * ps * D))
    for at in range(0, n_pages, chunk):                   # what the positions hold so far
        m = min(chunk, n_pages - at)
        k, v = normal(m, hk, ps // BLOCK, BLOCK, D), normal(m, hk, ps // BLOCK, BLOCK, D)
        k, v = k * k_size[:, None, None] + k_off[:, None, None], v * v_size[:, None, None]
        for x, rows, words in ((k, views[0], views[2]), (v, views[1], views[3])):
            r, w = _packed(*_quantised(_bf16(x).float()))
            rows[at:at + m], words[at:at + m] = r, w
        del k, v, x, r, w
    state = {"case": c, "T": T, "cache": cache, "n_pages": n_pages, "table": table, "start": start, "lengths": lengths, "max_new": int(new.max())}
    if c["op"] == "append":
        qkv = torch.cat([normal(T, hq * D), (normal(T, hk, D) * k_size + k_off).flatten(1), (normal(T, hk, D) * v_size).flatten(1)], 1).to(torch.bfloat16)
        # the layer's projection in one buffer: rows of queries, keys and values side by side
        state |= {"q": qkv[:, : hq * D], "k": qkv[:, hq * D: (hq + hk) * D], "v": qkv[:, (hq + hk) * D:], "qkv": qkv}
        inv = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=dev) / c["rot"])
        angle = torch.arange(per * ps, dtype=torch.float64, device=dev)[:, None] * inv
        state["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        state |= {"q_out": torch.zeros(T, hq * D, dtype=torch.bfloat16, device=dev), "k_out": torch.zeros(T, hk * D, dtype=torch.bfloat16, device=dev),
                  "v_out": torch.zeros(T, hk * D, dtype=torch.bfloat16, device=dev)}
    else:
        state |= {"q": normal(T, hq * D).to(torch.bfloat16), "out": torch.zeros(T, hq * D, dtype=torch.bfloat16, device=dev)}
    if own:
        from paper_2411_07942_b200 import binding

        kv = binding.TpqKv(hq, hk, D, ps)
        batch = binding.KvBatch(cache.data_ptr(), n_pages, table.data_ptr(), per, start.data_ptr(), lengths.data_ptr(), c["seqs"], state["max_new"], T)
        state |= {"kv": kv, "batch": batch}
        if c["op"] == "append":
            state["rope"] = binding.KvRotation(state["rotation"].data_ptr(), per * ps, c["rot"], int(c["interleaved"]), None)
        else:
            state["workspace"] = torch.empty(kv.attention_workspace_bytes(batch), dtype=torch.uint8, device=dev)
    return state


def _own_run(s):
    c, kv, stream = s["case"], s["kv"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "append":
        kv.append(s["batch"], s["k"].data_ptr(), s["v"].data_ptr(), k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), rotation=s["rope"],
                  q_ptr=s["q"].data_ptr(), q_stride=s["q"].stride(0), q_out_ptr=s["q_out"].data_ptr(), stream=stream)
        kv.read(s["batch"], s["k_out"].data_ptr(), s["v_out"].data_ptr(), stream=stream)
        return {"q": s["q_out"], "keys": s["k_out"], "values": s["v_out"]}
    kv.attention(s["batch"], s["q"].data_ptr(), s["out"].data_ptr(), s["workspace"].data_ptr(), s["workspace"].numel(), scale=1 / math.sqrt(c["dim"]),
                 window=c["window"], first=c["first"], stream=stream)
    return {"out": s["out"]}


def _rows(s):
    """Of every row: its sequence, its place among that sequence's new positions, its position, and whether it belongs to one."""
    row = torch.arange(s["T"], device="cuda")
    seq = (torch.searchsorted(s["start"], row.to(torch.int32), right=True) - 1).clamp(max=s["case"]["seqs"] - 1)
    at = row - s["start"][seq]
    n = (s["start"][1:] - s["start"][:-1])[seq]
    return seq, at, s["lengths"][seq] - n + at, at < n


def _rotated(x, table, pos, rot, interleaved):
    """x [rows, heads, dim] float32."""
    cos, sin = table[pos, None, : rot // 2], table[pos, None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2: rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), x[..., rot:]], -1)


def run(state):
    s, c = state, state["case"]
    if own:
        return _own_run(s)
    D, hq, hk, ps = c["dim"], c["heads"], c["kv_heads"], c["page"]
    seq, at, pos, real = _rows(s)
    key_rows, value_rows, key_words, value_words = _views(c, s["cache"])
    if c["op"] == "append":
        rotated = lambda x: _rotated(x.float().unflatten(1, (-1, D)), s["rotation"], torch.where(real, pos, 0), c["rot"], c["interleaved"])  # noqa: E731
        k, v = _packed(*_quantised(rotated(s["k"]))), _packed(*_quantised(s["v"].float().unflatten(1, (hk, D))))
        # a row behind the last sequence goes to a page that belongs to nobody
        spare = s["n_pages"] - 1
        n = s["T"] - c["pad"]
        p = pos[:n].long()
        place = (s["table"][seq[:n], p // ps].long(), slice(None), p % ps // BLOCK, p % BLOCK)
        key_rows[place], key_words[place], value_rows[place], value_words[place] = k[0][:n], k[1][:n], v[0][:n], v[1][:n]
        out = []
        for rows, words in ((key_rows, key_words), (value_rows, value_words)):
            x = torch.zeros(s["T"], hk * D, dtype=torch.bfloat16, device="cuda")
            x[:n] = _bf16(_values(rows[place], words[place])).flatten(1)
            out.append(x)
        return {"q": torch.where(real[:, None], _bf16(rotated(s["q"])).flatten(1), 0), "keys": out[0], "values": out[1]}
    L = s["table"].shape[1] * ps
    pages = s["table"].clamp(min=0).long()
    gather = lambda rows, words: _values(rows[pages], words[pages]).permute(0, 2, 1, 3, 4, 5).reshape(c["seqs"], hk, L, D)  # noqa: E731
    q_at = (s["start"][:-1, None] + torch.arange(s["max_new"], device="cuda")).clamp(max=s["T"] - 1).long()
    q = s["q"].float().view(s["T"], hk, hq // hk, D)[q_at].permute(0, 2, 3, 1, 4)          # [seqs, kv heads, group, new, dim]
    first_pos = s["lengths"] - (s["start"][1:] - s["start"][:-1])
    p = (first_pos[:, None] + torch.arange(s["max_new"], device="cuda"))[:, :, None]       # [seqs, new, 1]
    t = torch.arange(L, device="cuda")[None, None]
    see = t <= p
    if c["window"]:
        see = see & ((t > p - c["window"]) | (t < c["first"]))
    see = (see & (t < s["lengths"][:, None, None]))[:, None]                                # [seqs, 1, new, positions]
    scores = torch.matmul(q.flatten(2, 3), gather(key_rows, key_words).transpose(-1, -2)).unflatten(2, (hq // hk, s["max_new"]))
    scores = torch.where(see[:, :, None], scores / math.sqrt(D), -math.inf)
    weights = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-1e30))
    del scores
    total = weights.sum(-1, keepdim=True)
    o = torch.matmul(weights.flatten(2, 3), gather(value_rows, value_words)).unflatten(2, (hq // hk, s["max_new"])) / total.clamp(min=1e-37)
    o = o.permute(0, 3, 1, 2, 4)[seq, at.clamp(max=s["max_new"] - 1).long()].flatten(1)
    return {"out": torch.where(real[:, None], _bf16(o), 0)}


def exact(case, seed):
    """The same from the definitions in 64 bits, sequence by sequence."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    D, hq, hk, ps = c["dim"], c["heads"], c["kv_heads"], c["page"]
    new, length = _sizes(c)
    starts = np.concatenate([[0], np.cumsum(new)])
    f64 = torch.float64

    def turned(x, pos):
        cs = s["rotation"][pos].to(f64)
        z = torch.complex(cs[:, : c["rot"] // 2], cs[:, c["rot"] // 2:])[:, None]
        head = x[..., : c["rot"]]
        pair = head.unflatten(-1, (c["rot"] // 2, 2)) if c["interleaved"] else head.unflatten(-1, (2, c["rot"] // 2)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
        return torch.cat([y.flatten(-2) if c["interleaved"] else y.transpose(-1, -2).flatten(-2), x[..., c["rot"]:]], -1)

    def held(x):
        low = x.amin(-1, keepdim=True).to(torch.bfloat16).to(f64)
        step = torch.stack([(x.amax(-1, keepdim=True) - low) / 15, x.abs().amax(-1, keepdim=True) * REL_STEP, torch.full_like(low, MIN_STEP)]).amax(0).to(torch.bfloat16).to(f64)
        return low + step * ((x - low) / step).round().clamp(0, 15)

    if c["op"] == "append":
        got = {"q": torch.zeros(s["T"], hq * D, dtype=f64, device="cuda")}
        got |= {n: torch.zeros(s["T"], hk * D, dtype=f64, device="cuda") for n in ("keys", "values")}
        for i in range(c["seqs"]):
            r = slice(int(starts[i]), int(starts[i + 1]))
            pos = torch.arange(int(length[i] - new[i]), int(length[i]), device="cuda")
            x = {n: s[n][r].to(f64).unflatten(1, (-1, D)) for n in ("q", "k", "v")}
            got["q"][r], got["keys"][r], got["values"][r] = turned(x["q"], pos).flatten(1), held(turned(x["k"], pos)).flatten(1), held(x["v"]).flatten(1)
        return got
    out = torch.zeros(s["T"], hq, D, dtype=f64, device="cuda")
    half, entry = D // 2, BLOCK * (D + 8)
    blocks = s["cache"].view(-1, hk, ps // BLOCK, entry)
    for i in range(c["seqs"]):
        n, ln = int(new[i]), int(length[i])
        page = s["table"][i, : -(-ln // ps)].clamp(min=0).long()
        mine = blocks[page].transpose(0, 1).flatten(1, 2)                                   # [kv heads, blocks, bytes]
        kv = []
        for which in (0, 1):
            b = mine[..., which * BLOCK * half: (which + 1) * BLOCK * half].reshape(hk, -1, half)
            word = mine[..., 2 * BLOCK * half + which * 4 * BLOCK:][..., : 4 * BLOCK].reshape(hk, -1, 4).contiguous().view(torch.bfloat16).to(f64)
            x = torch.empty(hk, b.shape[1], D, dtype=f64, device="cuda")
            x[..., 0::2], x[..., 1::2] = (b % 16).to(f64), (b // 16).to(f64)
            kv.append((word[..., 1:] + word[..., :1] * x)[:, :ln])
        t = torch.arange(ln, device="cuda")
        for a in range(0, n, 1024):
            m = min(1024, n - a)
            p = torch.arange(ln - n + a, ln - n + a + m, device="cuda")[:, None]
            hide = t > p
            if c["window"]:
                hide |= (t <= p - c["window"]) & (t >= c["first"])
            q = s["q"][int(starts[i]) + a: int(starts[i]) + a + m].to(f64).view(m, hk, hq // hk, D)
            for h in range(hk):
                score = (q[:, h].transpose(0, 1) @ kv[0][h].T) / math.sqrt(D)
                out[int(starts[i]) + a: int(starts[i]) + a + m, h * (hq // hk): (h + 1) * (hq // hk)] = (score.masked_fill(hide, -math.inf).softmax(-1) @ kv[1][h]).transpose(0, 1)
    return {"out": out.flatten(1)}
