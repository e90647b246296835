"""A device's own work around the synchronisations of a step, as measurable cases: feed-forward, 4-bit weights, answers.

A tensor-parallel device computes its share of the feed-forward block ahead of the second synchronisation of a layer (its
columns of the gate and up projections, the activation, the product, then its rows of the down projection) and, behind the
last one, its slice of the vocabulary's logits, from which the log probabilities of an answer come.  The operators:

  quantize   a weight matrix [outputs][K] in BF16 becomes one in 4 bits, and is read back
  linear     x W^T with W in 4 bits: the down projection's partial sums in BF16, or a head's logits in FP32
  gated      act(x Wg^T) * (x Wu^T), both matrices in BF16 or both in 4 bits
  answers    of every row of logits (split over devices by columns): the log probability of a given token, the entropy and
             the n most likely tokens

A weight in 4 bits: codes -8 .. 7, one step for every `group` adjacent values of a row, w = step * code.  A row's steps
have 5 significant bits and lie within 2^15 of each other: with a the largest magnitude of a group, its step is 2a/15 rounded up to 5
significant bits, but at least 2^(e - 15), where e is the exponent of the row's largest step.

Sizes are the repository's workloads (5120 and 4608 features over 4 and 8 devices, feed-forward widths of 13824 and 36864,
a vocabulary of 32000) and the ranges around them.
"""
import math

import torch

own = False     # set by whoever measures: False, the plain forms; True, the framework's calls

ACTS = ("silu", "gelu_tanh", "gelu_erf")


def _weights(name, op, T, n, K, group=0, act="", out="bf16", pad=0):
    """n outputs of K inputs each; group 0: BF16 weights.  pad: elements between the rows of x and of the output."""
    c = {"op": op, "T": T, "n": n, "K": K, "group": group, "act": act, "out": out, "pad": pad}
    return {"name": name, **c} if name else c


def _answers(name, T, vocab, devices=1, top=0, logits="bf16", masked=0.0):
    """vocab: columns over all devices.  masked: share of the columns that a grammar or a padded vocabulary leaves out (-inf)."""
    c = {"op": "answers", "T": T, "vocab": vocab, "devices": devices, "top": top, "logits": logits, "masked": masked}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a down projection on one of 8 devices is brought into 4 bits when a model is loaded; and a head
        _weights("quantize_down", "quantize", 0, 5120, 1728, 64),
        _weights("quantize_head", "quantize", 0, 32000, 5120, 128),
        # one generated token, one of 8 devices: the smallest product of a layer, nothing but latency
        _weights("linear_token", "linear", 1, 5120, 1728, 64),
        # one token's logits on a device that holds the whole head
        _weights("head_token", "linear", 1, 32000, 5120, 32, out="fp32"),
        # the down projection of the headline prompt on one of 4 devices
        _weights("linear_prompt", "linear", 2048, 5120, 3456, 128),
        # one generated token, weights in BF16, one of 8 devices
        _weights("gated_token", "gated", 1, 1728, 5120, act="silu"),
        # a decode batch of odd size on one of 8 devices of the wider model, weights in 4 bits
        _weights("gated_batch_int4", "gated", 61, 4608, 4608, 128, act="gelu_tanh"),
        # the headline prompt on one of 4 devices
        _weights("gated_prompt", "gated", 2048, 3456, 5120, act="silu"),
        # a ragged prompt on one of 4 devices, weights in 4 bits
        _weights("gated_prompt_int4", "gated", 1999, 3456, 5120, 32, act="silu", pad=8),
        # the answer to one token: its probability and 20 alternatives
        _answers("answers_token", 1, 32000, top=20),
        # scoring of given text: log probabilities and entropy of 2048 tokens
        _answers("answers_score", 2048, 32000),
        # a decode batch over a large vocabulary that 4 devices share, part of it masked, FP32 logits
        _answers("answers_shards", 61, 256000, devices=4, top=20, logits="fp32", masked=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["quantize", "linear", "gated", "answers"], [1, 4, 4, 3])[0]
    if op == "answers":
        vocab = _log(rng, 300, 260000)
        return _answers("", _log(rng, 1, max(1, min(4096, 2048 * 32000 // vocab))), vocab, devices=rng.choice([1, 1, 1, 2, 4, 8]),
                        top=rng.choice([0, 0, 1, 5, 20, 32]), logits=rng.choice(["bf16", "bf16", "fp32"]), masked=rng.choice([0.0, 0.0, 0.5]))
    K = _log(rng, 100, 14000) if rng.random() < 0.5 else 128 * _log(rng, 1, 100)
    group = rng.choice([32, 64, 128])
    if op == "quantize":
        return _weights("", op, 0, _log(rng, 50, 32000 * 5120 // K), K, group)
    n = _log(rng, 50, min(33000, 32000 * 5120 // K))
    n = n if rng.random() < 0.5 else max(64, n // 64 * 64)
    T = rng.choice([1, 1, 2, 3]) if rng.random() < 0.25 else _log(rng, 1, max(1, min(4096, 2048 * 3456 * 5120 // (n * K))))
    if op == "linear":
        return _weights("", op, T, n, K, group, out=rng.choice(["bf16", "bf16", "fp32"]), pad=rng.choice([0, 0, 24]))
    return _weights("", op, T, n, K, rng.choice([0, group]), act=rng.choice(ACTS), pad=rng.choice([0, 0, 24]))


def _groups(c):
    return -(-c["K"] // c["group"])


def work(case):
    c = case
    if c["op"] == "answers":
        cells = c["T"] * c["vocab"]
        # logits and tokens in; probability, entropy and alternatives out; an exponential, a maximum and two sums a cell
        return {"bytes": cells * (2 if c["logits"] == "bf16" else 4) + c["T"] * (4 + 8 + 8 * c["top"]), "flops": 6 * cells}
    weight = c["n"] * (c["K"] / 2 + _groups(c) + 4) if c["group"] else 2 * c["n"] * c["K"]
    if c["op"] == "quantize":
        # BF16 in, 4 bits out; 4 bits in again, BF16 out
        return {"bytes": int(4 * c["n"] * c["K"] + 2 * weight), "flops": 5 * c["n"] * c["K"]}
    two = 2 if c["op"] == "gated" else 1
    return {"bytes": int(two * weight + 2 * c["T"] * c["K"] + (4 if c["out"] == "fp32" else 2) * c["T"] * c["n"]),
            "flops": 2 * two * c["T"] * c["n"] * c["K"]}


def _quantised(w, group):
    """w [outputs][K] float32 -> codes (int8) [outputs][K] and steps (float32) [outputs][groups]."""
    n, K = w.shape
    padded = torch.nn.functional.pad(w, (0, -K % group)).view(n, -1, group)
    # (a division by a plain number would be a product with its rounded reciprocal, which can end up a step higher)
    bound = padded.abs().amax(-1) * 2 / torch.tensor(15.0, device=w.device)
    mantissa, exponent = torch.frexp(bound)                       # mantissa in [0.5, 1): 5 significant bits are multiples of 1/32
    two = lambda e: (e + 127 << 23).view(torch.float32)  # noqa: E731   (2^e: ldexp and pow are an ulp off for some e)
    step = torch.ceil(mantissa * 32) * two(exponent - 5)
    top = torch.frexp(step.amax(-1, keepdim=True)).exponent - 1
    step = torch.maximum(step, two(top - 15))
    step = torch.where(step.amax(-1, keepdim=True) > 0, step, 1.0)
    return (padded / step[..., None]).round().clamp(-8, 7).to(torch.int8).view(n, -1)[:, :K], step


def _values(codes, step, group):
    return codes.float() * step.repeat_interleave(group, 1)[:, : codes.shape[1]]


def _act(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))


def _shares(c):
    """Columns of each device: as equal as they get in multiples of 8, the rest on the last one."""
    d, v = c["devices"], c["vocab"]
    each = v // d // 8 * 8
    return [each] * (d - 1) + [v - each * (d - 1)]


def prepare(case, seed):
    c, g = case, torch.Generator("cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    state = {"case": c}
    if own:
        from paper_2411_07942_b200 import binding

        state |= {"binding": binding, "block": binding.TpqBlock()}
    if c["op"] == "answers":
        kind = torch.bfloat16 if c["logits"] == "bf16" else torch.float32
        spread = 1.0 + 2.0 * torch.rand(c["T"], 1, generator=g, device="cuda")      # sure rows and unsure ones
        out = torch.rand(c["vocab"], generator=g, device="cuda") < c["masked"]
        allowed = torch.nonzero(~out).flatten() if c["masked"] else torch.arange(c["vocab"], device="cuda")
        state["logits"] = []
        for n in _shares(c):
            # a device's logits: rows padded to a multiple of 8 values, as its product leaves them
            buf = torch.full((c["T"], -(-n // 8) * 8), math.nan, dtype=kind, device="cuda")
            buf[:, :n] = normal(c["T"], n) * spread
            at = sum(x.shape[1] for x in state["logits"])
            buf[:, :n].masked_fill_(out[at:at + n], -math.inf)
            state["logits"].append(buf[:, :n])
        state["tokens"] = allowed[torch.randint(0, allowed.numel(), (c["T"],), generator=g, device="cuda")].to(torch.int32)
        if own:
            bytes_ = binding.token_record_bytes(c["T"], c["top"])
            state["records"] = [torch.empty(bytes_, dtype=torch.uint8, device="cuda") for _ in range(c["devices"])]
            state |= {"logprob": torch.empty(c["T"], device="cuda"), "entropy": torch.empty(c["T"], device="cuda"),
                      "top": torch.empty(c["T"], c["top"], dtype=torch.int32, device="cuda"), "top_logprob": torch.empty(c["T"], c["top"], device="cuda")}
        return state
    n, K = c["n"], c["K"]

    def weight():
        # outputs differ in size, and so do inputs (what the layer norm ahead scales by); a few weights stand out
        w = normal(n, K).mul_(torch.exp(0.3 * normal(n, 1)) / math.sqrt(K)).mul_(torch.exp(0.2 * normal(1, K)))
        w[torch.randint(0, n, (max(1, n // 16),), generator=g, device="cuda"), torch.randint(0, K, (max(1, n // 16),), generator=g, device="cuda")] *= 6
        return w.to(torch.bfloat16)

    if c["op"] == "quantize":
        state["w"] = weight()
        if own:
            state |= {"w4": torch.empty(binding.weight4_bytes(n, K, c["group"]), dtype=torch.uint8, device="cuda"),
                      "values": torch.empty(n, K, dtype=torch.bfloat16, device="cuda")}
        return state
    wide = -(-K // 8) * 8 + c["pad"]
    state["x"] = torch.full((c["T"], wide), math.nan, dtype=torch.bfloat16, device="cuda")[:, :K]
    state["x"].copy_(normal(c["T"], K) * torch.exp(0.3 * normal(1, K)))
    out_wide = -(-n // 8) * 8 + c["pad"]
    state["out"] = torch.zeros(c["T"], out_wide, dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16, device="cuda")[:, :n]
    state["weights"], state["keep"] = [], []
    for _ in range(2 if c["op"] == "gated" else 1):
        w = weight()
        wide_w = -(-K // 8) * 8
        if not own:
            state["weights"].append(_quantised(w.float(), c["group"]) if c["group"] else w)
        elif c["group"]:
            w4 = torch.empty(binding.weight4_bytes(n, K, c["group"]), dtype=torch.uint8, device="cuda")
            state["block"].quantize_weight(w.data_ptr(), n, K, c["group"], w4.data_ptr(), w4.numel(), stream=torch.cuda.current_stream().cuda_stream)
            state["keep"].append(w4)
            state["weights"].append(binding.Weight(w4.data_ptr(), n, K, 0, binding.TPQ_WEIGHT_INT4, c["group"]))
            del w
        else:
            w = torch.nn.functional.pad(w, (0, wide_w - K))
            state["keep"].append(w)
            state["weights"].append(binding.Weight(w.data_ptr(), n, K, wide_w, binding.TPQ_WEIGHT_BF16, 0))
    if own:
        state["act"] = {"silu": binding.TPQ_ACT_SILU, "gelu_tanh": binding.TPQ_ACT_GELU_TANH, "gelu_erf": binding.TPQ_ACT_GELU_ERF}.get(c["act"])
    return state


def _own_run(s):
    c, block, stream = s["case"], s["block"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "quantize":
        block.quantize_weight(s["w"].data_ptr(), c["n"], c["K"], c["group"], s["w4"].data_ptr(), s["w4"].numel(), stream=stream)
        block.read_weight(s["w4"].data_ptr(), c["n"], c["K"], c["group"], s["values"].data_ptr(), stream=stream)
        return {"values": s["values"]}
    if c["op"] == "answers":
        dtype = s["binding"].TPQ_OUT_BF16 if c["logits"] == "bf16" else s["binding"].TPQ_OUT_FP32
        first = 0
        for x, r in zip(s["logits"], s["records"]):
            block.token_stats(x.data_ptr(), c["T"], x.shape[1], r.data_ptr(), r.numel(), dtype=dtype, stride=x.stride(0), first=first,
                              tokens_ptr=s["tokens"].data_ptr(), n_top=c["top"], stream=stream)
            first += x.shape[1]
        block.token_logprobs([r.data_ptr() for r in s["records"]], c["T"], s["logprob"].data_ptr(), s["entropy"].data_ptr(), n_top=c["top"],
                             top_ptr=s["top"].data_ptr() if c["top"] else None, top_logprob_ptr=s["top_logprob"].data_ptr() if c["top"] else None, stream=stream)
        return {"logprob": s["logprob"], "entropy": s["entropy"], "top": s["top"], "top_logprob": s["top_logprob"]}
    x, out = s["x"], s["out"]
    if c["op"] == "linear":
        dtype = s["binding"].TPQ_OUT_FP32 if c["out"] == "fp32" else s["binding"].TPQ_OUT_BF16
        block.linear4(s["weights"][0], x.data_ptr(), c["T"], out.data_ptr(), out_dtype=dtype, x_stride=x.stride(0), out_stride=out.stride(0), stream=stream)
    else:
        block.gated(*s["weights"], s["act"], x.data_ptr(), c["T"], out.data_ptr(), x_stride=x.stride(0), out_stride=out.stride(0), stream=stream)
    return {"out": out}


def run(state):
    s, c = state, state["case"]
    if own:
        return _own_run(s)
    if c["op"] == "quantize":
        return {"values": _values(*_quantised(s["w"].float(), c["group"]), c["group"]).to(torch.bfloat16)}
    if c["op"] == "answers":
        x = torch.cat([v.float() for v in s["logits"]], 1)
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        log_total = top + torch.log(e.sum(1, keepdim=True))
        d = x - log_total
        p = torch.exp(d)
        entropy = -(p * d.clamp(min=-1e30)).sum(1)
        best = torch.sort(d, dim=1, descending=True, stable=True) if c["top"] else (d[:, :0], d[:, :0])     # (equal ones: the lowest index first)
        return {"logprob": d.gather(1, s["tokens"].long()[:, None])[:, 0], "entropy": entropy, "top": best[1][:, : c["top"]].to(torch.int32),
                "top_logprob": best[0][:, : c["top"]].contiguous()}
    x = s["x"].float()
    y = [x @ (_values(*w, c["group"]) if c["group"] else w.float()).T for w in s["weights"]]
    return {"out": (y[0] if c["op"] == "linear" else _act(y[0], c["act"]) * y[1]).to(s["out"].dtype)}


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    f64 = torch.float64
    if c["op"] == "answers":
        got = {"logprob": [], "entropy": [], "top": [], "top_logprob": []}
        rows = max(1, (1 << 27) // c["vocab"])
        for a in range(0, c["T"], rows):
            x = torch.cat([v[a:a + rows].to(f64) for v in s["logits"]], 1)
            logp = x.log_softmax(1)
            got["logprob"].append(logp[torch.arange(x.shape[0], device="cuda"), s["tokens"][a:a + rows].long()])
            got["entropy"].append(torch.special.entr(logp.exp()).sum(1))
            order = torch.argsort(x, dim=1, descending=True, stable=True)[:, : c["top"]]
            got["top"].append(order.to(torch.int32))
            got["top_logprob"].append(logp.gather(1, order))
        return {k: torch.cat(v) for k, v in got.items()}

    def held(w, group):
        out = torch.empty(w.shape, dtype=f64, device="cuda")
        w = w.to(f64)
        largest = torch.stack([p.abs().amax(1) for p in w.split(group, 1)], 1)
        cut = (1 << 48) - 1                                                                # the bits behind the 5th significant one
        steps = ((largest * 2 / torch.full_like(largest, 15)).view(torch.int64) + cut & ~cut).view(f64)
        steps = torch.maximum(steps, (steps.amax(1, keepdim=True).view(torch.int64) & 0x7FF << 52).view(f64) * 2.0 ** -15)
        for i, p in enumerate(w.split(group, 1)):
            step = torch.where(steps[:, i:i + 1] > 0, steps[:, i:i + 1], 1.0)
            out[:, i * group: i * group + p.shape[1]] = step * (p / step).round().clamp(-8, 7)
        return out

    if c["op"] == "quantize":
        return {"values": torch.cat([held(part, c["group"]) for part in s["w"].split(4096)])}
    x, y = s["x"].to(f64), []
    for w in s["weights"]:
        if c["group"]:
            codes, steps = w
            y.append(torch.cat([x @ (p.to(f64).T * q.to(f64).repeat_interleave(c["group"], 1)[:, : c["K"]].T) for p, q in zip(codes.split(4096), steps.split(4096))], 1))
        else:
            y.append(x @ w.to(f64).T)
    if c["op"] == "linear":
        return {"out": y[0]}
    if c["act"] == "silu":
        a = y[0] * torch.sigmoid(y[0])
    else:
        a = torch.nn.functional.gelu(y[0], approximate="tanh" if c["act"] == "gelu_tanh" else "none")
    return {"out": a * y[1]}
