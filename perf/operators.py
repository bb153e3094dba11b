"""Operators at the two ends of a weight synchronisation, as cases that can be timed and checked.

On the training side, where the weights that an update carries come from:

  lookup   rows of an embedding (or of the vocabulary shard that a rank holds) for a batch of tokens, scaled
  grad     the gradient of such a lookup: each token's row is summed into the row of the embedding that it named
  clip     the norm of all gradients of a parameter set together, and the gradients scaled down to a largest norm

On the serving side, where the weights that an update has written are used:

  round    a matrix held in microscaled 4-bit floating point (32 values along a row share a power of two): quantised
           and expanded again, the values that a product with it will see
  linear   activations times such a matrix, the activations quantised the same way on the way in

`run` computes a case in plain torch operations in 32 bits, or, where `own` is set, with this library's kernels.
Sizes are those of the workloads (decoders of 7B, 8B and 32B weights and their tensor-parallel shards), or generic.
Tokens follow the usual law of text: the r-th most frequent one comes with a probability of about 1 / r.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 32                               # values that share a scale in the 4-bit format
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_CHUNK = 1 << 28


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decode step of 64 sequences on the rank that holds the first quarter of a 7B-style vocabulary
        dict(name="lookup_decode", op="lookup", tokens=64, vocab=32000, first=0, rows=8000, cols=4096, table="bf16",
             out="bf16", index=64, scale=1.0, pad=0),
        # a training batch, 32B-style, rank 1 of 8: fp32 masters, activations in bf16; ids of other ranks give zeros
        dict(name="lookup_batch", op="lookup", tokens=16384, vocab=152064, first=19008, rows=19008, cols=5120, table="f32",
             out="bf16", index=64, scale=71.554175, pad=0),
        # the gradient of one batch for a whole 7B-style embedding, an odd number of tokens: mostly rows without a token
        dict(name="grad_batch", op="grad", tokens=8191, vocab=32000, first=0, rows=32000, cols=4096, dy="bf16", grad="f32",
             index=64, scale=64.0, accumulate=False, pad=0),
        # a long batch added to the gradient of the micro-batches before it: rank 0 of 8 of a 32B-style vocabulary
        dict(name="grad_accumulate", op="grad", tokens=65536, vocab=152064, first=0, rows=19008, cols=5120, dy="bf16", grad="f32",
             index=64, scale=1.0, accumulate=True, pad=0),
        # a small model of odd sizes, its gradients one right behind the other from an odd element on
        dict(name="clip_small_packed", op="clip", layers=2, hidden=515, heads=5, kv_heads=5, head_dim=103, inter=1409, vocab=4099,
             tp=1, dtype="bf16", packed=True, over=3.0),
        # what one rank of TP 8 holds of half the layers of a 32B-style decoder: fp32 main gradients, 2.2 G of them
        dict(name="clip_32b_rank", op="clip", layers=32, hidden=5120, heads=40, kv_heads=8, head_dim=128, inter=27648, vocab=152064,
             tp=8, dtype="f32", packed=False, over=3.0),
        # a receiver's gate and up projection, 32B-style at TP 8, after an update has been applied to it
        dict(name="round_gate_up", op="round", rows=6912, cols=5120, dtype="bf16", pad=0),
        # the whole head of an 8B-style decoder (TP 1 for rollout)
        dict(name="round_head", op="round", rows=151936, cols=4096, dtype="bf16", pad=0),
        # one token through a fused gate and up projection: the matrix is read once, nothing else counts
        dict(name="linear_token", op="linear", m=1, n=6912, k=5120, out="bf16", pad=0),
        # a decode step of 48 sequences, sizes that fill no tile and no block of 32
        dict(name="linear_decode_odd", op="linear", m=47, n=4099, k=4083, out="bf16", pad=5),
        # logits of 256 sequences from a shard of a 32B-style head
        dict(name="linear_head", op="linear", m=256, n=19008, k=5120, out="f32", pad=0),
        # a chunk of prompts through the same gate and up projection
        dict(name="linear_prompt", op="linear", m=16384, n=6912, k=5120, out="bf16", pad=0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, step):
    """The same, a multiple of `step` half of the time."""
    n = _log(rng, lo, hi)
    return max(lo, n // step * step) if rng.random() < 0.5 else n


def _any(rng):
    op = rng.choice(("lookup", "grad", "clip", "round", "linear"))
    if op in ("lookup", "grad"):
        cols = _size(rng, 96, 8192, 64)
        rows = _size(rng, 500, min(152064, (1 << 29) // cols), 64)
        ranks = rng.choice((1, 1, 2, 4, 8))
        tokens = _log(rng, 1, min(65536, (1 << 29) // cols))
        c = dict(op=op, tokens=tokens, vocab=rows * ranks, first=rows * rng.randrange(ranks), rows=rows, cols=cols,
                 index=rng.choice((32, 64)), scale=rng.choice((1.0, round(math.sqrt(cols), 6))), pad=rng.choice((0, 0, 8, 3)))
        if op == "lookup":
            return dict(c, table=rng.choice(("bf16", "f32")), out=rng.choice(("bf16", "f32")))
        return dict(c, dy=rng.choice(("bf16", "bf16", "f32")), grad=rng.choice(("bf16", "f32", "f32")), accumulate=rng.random() < 0.4)
    if op == "clip":
        heads = rng.choice((4, 8, 16, 32))
        head_dim = rng.choice((64, 80, 128, rng.randrange(61, 131, 2)))
        hidden = heads * head_dim
        return dict(op=op, layers=_log(rng, 1, 16), hidden=hidden, heads=heads, kv_heads=rng.choice((4, heads)), head_dim=head_dim,
                    inter=8 * _log(rng, hidden // 4, hidden // 2), vocab=4 * _log(rng, 500, 16000), tp=rng.choice((1, 2, 4)),
                    dtype=rng.choice(("bf16", "f32")), packed=rng.random() < 0.5, over=rng.choice((0.5, 3.0, 50.0)))
    if op == "round":
        cols = _size(rng, 32, 28000, 32)
        return dict(op=op, rows=_log(rng, 1, (1 << 29) // cols), cols=cols, dtype=rng.choice(("bf16", "bf16", "f32")),
                    pad=rng.choice((0, 0, 8, 3)))
    k = _size(rng, 64, 16384, 32)
    n = _size(rng, 64, 32768, 16)
    return dict(op="linear", m=_log(rng, 1, max(1, min(16384, (1 << 39) // (k * n)))), n=n, k=k,
                out=rng.choice(("bf16", "bf16", "f32")), pad=rng.choice((0, 0, 8, 3)))


def _sizes(c):
    """Every length that a case's tensors have."""
    found = {v for v in c.values() if isinstance(v, int)}
    if c["op"] == "clip":
        q, kv = c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
        found |= {n // t for n in (c["hidden"], q, q + 2 * kv, c["inter"], 2 * c["inter"], c["vocab"]) for t in (1, c["tp"])}
    return found


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    c = _any(rng)
    return c if work(c)["bytes"] <= most and 3072 not in _sizes(c) else draw(rng)


# ---------------------------------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------------------------------
def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + part) & 0x7FFFFFFF)
    return g


def _normal(numel, std, dtype, g):
    out = torch.empty(numel, dtype=dtype, device="cuda")
    for a in range(0, numel, _CHUNK):
        m = min(_CHUNK, numel - a)
        out[a:a + m] = torch.randn(m, generator=g, device="cuda") * std
    return out


def _matrix(rows, cols, pad, std, dtype, g):
    """A matrix whose rows lie `pad` elements further apart than they are long."""
    return _normal(rows * (cols + pad), std, dtype, g).view(rows, cols + pad)[:, :cols]


def _tokens(c, g):
    u = torch.rand(c["tokens"], generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(c["vocab"] + 1)) - 1).to(torch.int64).clamp_(0, c["vocab"] - 1)
    return ids.to(torch.int32 if c["index"] == 32 else torch.int64)


def _row_shares(c):
    """The probability with which one token names each row of the shard."""
    r = np.arange(c["first"], c["first"] + c["rows"], dtype=np.float64)
    return np.log((r + 2) / (r + 1)) / math.log(c["vocab"] + 1)


def _named(c):
    """(tokens that lie in the shard, rows of the shard that some token names), on average."""
    p = _row_shares(c)
    return float(c["tokens"] * p.sum()), float((1 - np.exp(c["tokens"] * np.log1p(-p))).sum())


def _numels(c):
    """Elements of each tensor of the decoder that a rank holds: norms whole, matrices cut."""
    h, tp = c["hidden"], c["tp"]
    q, kv = c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
    layer = [h, (q + 2 * kv) * h // tp, h * q // tp, h, 2 * c["inter"] * h // tp, h * c["inter"] // tp]
    return [c["vocab"] * h // tp] + layer * c["layers"] + [h, c["vocab"] * h // tp]


def _places(c):
    """Where each tensor begins in the one buffer that holds them all, and the buffer's length."""
    at, places = 1 if c["packed"] else 0, []
    for n in _numels(c):
        places.append(at)
        at += n if c["packed"] else -(-n // 256) * 256
    return places, at


def _views(flat, c):
    return [flat[a:a + n] for a, n in zip(_places(c)[0], _numels(c))]


def _pointers(tensors):
    return torch.tensor([t.data_ptr() for t in tensors], dtype=torch.int64, device="cuda")


def _block_parts(x):
    """A matrix in blocks of 32 along its rows, the last one filled up with zeros."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)) if cols % BLOCK else x
    return x.reshape(rows, blocks, BLOCK)


def _exponents(parts):
    """Exponent of each block's scale: that of its largest magnitude, less 2 (6 = 1.5 x 2^2 is the largest value)."""
    top = parts.abs().amax(-1)
    return torch.where(top > 0, torch.frexp(top).exponent - 3, torch.full((), -127, dtype=torch.int32, device=top.device)).clamp_(min=-127)


def _codes(parts, exponents):
    """4-bit codes (sign, two bits of exponent, one of mantissa) of the blocks' values, nearest, ties to even, at most 6."""
    m = torch.ldexp(parts, -exponents.unsqueeze(-1))
    sign = torch.signbit(m).to(torch.uint8) << 3
    m = m.abs_()
    code = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    return code | sign


def _quantised(x):
    """(codes two to a byte, the first in the low half; scales as exponents + 127) of a matrix."""
    parts = _block_parts(x.float())
    e = _exponents(parts)
    code = _codes(parts, e).view(x.shape[0], -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8)


def prepare(case, seed):
    c, g = case, _gen(seed, 1)
    s = {"case": c}
    if c["op"] in ("lookup", "grad"):
        s["tokens"] = _tokens(c, g)
    if c["op"] == "lookup":
        s["table"] = _matrix(c["rows"], c["cols"], c["pad"], 0.02, DTYPES[c["table"]], g)
        s["out"] = torch.empty(c["tokens"], c["cols"], dtype=DTYPES[c["out"]], device="cuda")
    elif c["op"] == "grad":
        s["dy"] = _matrix(c["tokens"], c["cols"], c["pad"], 1e-3, DTYPES[c["dy"]], g)
        s["grad"] = _normal(c["rows"] * c["cols"], 1e-3, DTYPES[c["grad"]], g).view(c["rows"], c["cols"])
    elif c["op"] == "clip":
        numels = _numels(c)
        total = _places(c)[1]
        s["flat"] = _normal(total, 1e-3, DTYPES[c["dtype"]], g)
        s["clipped"] = torch.zeros(total, dtype=DTYPES[c["dtype"]], device="cuda")
        s["grads"], s["outs"] = _views(s["flat"], c), _views(s["clipped"], c)
        s["grad_tab"], s["out_tab"] = _pointers(s["grads"]), _pointers(s["outs"])
        s["offsets"] = torch.tensor([0] + list(np.cumsum(numels)), dtype=torch.int64, device="cuda")
        s["total"] = sum(numels)
        s["norm"] = torch.zeros((), dtype=torch.float32, device="cuda")
        s["max_norm"] = 1e-3 * math.sqrt(s["total"]) / c["over"]     # the norm is about `over` times as much
    elif c["op"] == "round":
        s["x"] = _matrix(c["rows"], c["cols"], c["pad"], 0.02, DTYPES[c["dtype"]], g)
        s["out"] = torch.empty(c["rows"], c["cols"], dtype=DTYPES[c["dtype"]], device="cuda")
        s["lut"] = torch.tensor(MAGNITUDES, device="cuda")
    else:
        s["x"] = _matrix(c["m"], c["k"], c["pad"], 1.0, torch.bfloat16, g)
        s["codes"], s["scales"] = _quantised(_normal(c["n"] * c["k"], 0.02, torch.bfloat16, g).view(c["n"], c["k"]))
        s["out"] = torch.empty(c["m"], c["n"], dtype=DTYPES[c["out"]], device="cuda")
        s["lut"] = torch.tensor(MAGNITUDES, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------
# one pass, in plain operations
# ---------------------------------------------------------------------------------------------------
def _expanded(codes, scales, lut):
    """The values of a quantised matrix, whole blocks."""
    code = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1)
    v = lut[(code & 7).to(torch.int32)]
    v = torch.where(code > 7, -v, v).view(codes.shape[0], -1, BLOCK)
    return torch.ldexp(v, scales.to(torch.int32).unsqueeze(-1) - 127).view(codes.shape[0], -1)


def _plain(s):
    c = s["case"]
    if c["op"] == "lookup":
        at = s["tokens"].long() - c["first"]
        here = (at >= 0) & (at < c["rows"])
        rows = s["table"][torch.where(here, at, 0)].float() * c["scale"]
        s["out"].copy_(torch.where(here.unsqueeze(-1), rows, 0.0))
        return {"out": s["out"]}
    if c["op"] == "grad":
        at = s["tokens"].long() - c["first"]
        here = ((at >= 0) & (at < c["rows"])).nonzero().view(-1)
        grad = s["grad"].float() if c["accumulate"] else torch.zeros(c["rows"], c["cols"], device="cuda")
        total = torch.zeros_like(grad).index_add_(0, at[here], s["dy"][here].float())
        s["grad"].copy_(grad + total * c["scale"])
        return {"grad": s["grad"]}
    if c["op"] == "clip":
        norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
        factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
        [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["outs"])]
        s["norm"].copy_(norm)
        return {"grads": s["clipped"], "norm": s["norm"]}
    if c["op"] == "round":
        codes, scales = _quantised(s["x"])
        s["out"].copy_(_expanded(codes, scales, s["lut"])[:, :c["cols"]])
        return {"values": s["out"]}
    w = _expanded(s["codes"], s["scales"], s["lut"])
    x = _expanded(*_quantised(s["x"]), s["lut"])
    s["out"].copy_(x @ w.t())
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------------
# one pass, with this library
# ---------------------------------------------------------------------------------------------------
def _kernels(s):
    import paper_2605_06534_amd as R

    c = s["case"]
    if c["op"] == "lookup":
        R.embedding_lookup(s["table"], s["tokens"], s["out"], scale=c["scale"], first_row=c["first"])
        return {"out": s["out"]}
    if c["op"] == "grad":
        if "ws" not in s:                # made once and kept, as a program does
            s["ws"] = R.embedding_grad_workspace(c["rows"], c["cols"], c["tokens"])
        R.embedding_grad(s["dy"], s["tokens"], s["grad"], s["ws"], scale=c["scale"], first_row=c["first"], accumulate=c["accumulate"])
        return {"grad": s["grad"]}
    if c["op"] == "clip":
        if "ws" not in s:
            s["ws"] = R.grad_workspace()
        R.grad_clip_norm(s["grad_tab"], s["offsets"], s["total"], DTYPES[c["dtype"]], s["out_tab"], s["max_norm"], s["norm"], s["ws"])
        return {"grads": s["clipped"], "norm": s["norm"]}
    if c["op"] == "round":
        if "quantised" not in s:
            s["quantised"] = R.Mx4(c["rows"], c["cols"])
        R.mx4_quantize(s["x"], s["quantised"])
        R.mx4_dequantize(s["quantised"], s["out"])
        return {"values": s["out"]}
    if "weights" not in s:
        s["weights"] = R.Mx4(c["n"], c["k"], s["codes"], s["scales"])
        s["ws"] = R.mx4_linear_workspace(c["m"], c["n"], c["k"])
    R.mx4_linear(s["x"], s["weights"], s["out"], s["ws"])
    return {"out": s["out"]}


def run(state):
    return _kernels(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------
def work(case):
    c, size = case, {"bf16": 2, "f32": 4}
    if c["op"] == "lookup":
        _, rows = _named(c)
        return {"bytes": c["tokens"] * c["index"] // 8 + rows * c["cols"] * size[c["table"]] + c["tokens"] * c["cols"] * size[c["out"]],
                "flops": c["tokens"] * c["cols"]}
    if c["op"] == "grad":
        tokens, rows = _named(c)
        written = 2 * rows if c["accumulate"] else c["rows"]      # added to: the named rows are read and written, no others
        return {"bytes": c["tokens"] * c["index"] // 8 + tokens * c["cols"] * size[c["dy"]] + written * c["cols"] * size[c["grad"]],
                "flops": (tokens + rows) * c["cols"]}
    if c["op"] == "clip":
        total = sum(_numels(c))
        return {"bytes": 2 * total * size[c["dtype"]], "flops": 3 * total}
    if c["op"] == "round":
        total = c["rows"] * c["cols"]
        return {"bytes": total * (2 * size[c["dtype"]] + 0.5 + 1 / 32), "flops": 2 * total}
    return {"bytes": 2 * c["m"] * c["k"] + c["n"] * c["k"] * (0.5 + 1 / 32) + c["m"] * c["n"] * size[c["out"]],
            "flops": 2 * c["m"] * c["n"] * c["k"]}


# ---------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------
def _nearest(x):
    """Each row's values as the 4-bit format holds them, found by the distance to each value of the format: of two
    that are as near the one with the even code.  In slices of rows, to bound the memory."""
    out = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    for a in range(0, x.shape[0], max(1, (1 << 26) // max(1, x.shape[1]))):
        rows = x[a:a + max(1, (1 << 26) // max(1, x.shape[1]))].double()
        width = -(-rows.shape[1] // BLOCK) * BLOCK
        blocks = torch.zeros(rows.shape[0], width, dtype=torch.float64, device=x.device)
        blocks[:, :rows.shape[1]] = rows
        blocks = blocks.view(rows.shape[0], -1, BLOCK)
        top = blocks.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 2).clamp(min=2.0 ** -127)
        m = blocks.abs() / scale
        below, above = torch.searchsorted(middle, m, right=False), torch.searchsorted(middle, m, right=True)
        value = grid[torch.where(below % 2 == 0, below, above)] * scale * torch.sign(blocks)
        out[a:a + rows.shape[0]] = value.view(rows.shape[0], -1)[:, :rows.shape[1]]
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "lookup":
        out = torch.zeros(c["tokens"], c["cols"], dtype=torch.float64, device="cuda")
        here = [i for i, t in enumerate(s["tokens"].tolist()) if c["first"] <= t < c["first"] + c["rows"]]
        at = torch.tensor(here, dtype=torch.int64, device="cuda")
        out[at] = s["table"][s["tokens"].long()[at] - c["first"]].double() * c["scale"]
        return {"out": out}
    if c["op"] == "grad":
        # the tokens in order of the rows they name, running sums, and differences where the row changes
        ids, order = torch.sort(s["tokens"].long(), stable=True)
        mine = (ids >= c["first"]) & (ids < c["first"] + c["rows"])
        ids, order = ids[mine] - c["first"], order[mine]
        grad = s["grad"].double() if c["accumulate"] else torch.zeros(c["rows"], c["cols"], dtype=torch.float64, device="cuda")
        if len(ids):
            rows, counts = torch.unique_consecutive(ids, return_counts=True)
            ends = torch.cumsum(counts, 0)
            for a in range(0, c["cols"], 1024):
                sums = torch.cumsum(s["dy"][:, a:a + 1024][order].double(), 0)
                sums = torch.cat((torch.zeros_like(sums[:1]), sums))
                grad[rows, a:a + 1024] += (sums[ends] - sums[ends - counts]) * c["scale"]
        return {"grad": grad}
    if c["op"] == "clip":
        total = sum(torch.dot(part, part) for g in s["grads"] for part in (p.double() for p in g.split(_CHUNK)))
        norm = math.sqrt(float(total))
        factor = min(1.0, s["max_norm"] / (norm + 1e-6))
        out = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
        for a, n in zip(_places(c)[0], _numels(c)):
            out[a:a + n] = s["flat"][a:a + n].double().mul_(factor)
        return {"grads": out, "norm": norm}
    if c["op"] == "round":
        return {"values": _nearest(s["x"])}
    grid = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), dtype=torch.float64, device="cuda")
    w = torch.empty(c["n"], 2 * s["codes"].shape[1], dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = grid[(s["codes"] % 16).long()], grid[(s["codes"] // 16).long()]
    w *= torch.exp2(s["scales"].double() - 127).repeat_interleave(BLOCK, dim=1)
    return {"out": torch.mm(_nearest(s["x"]), w[:, :c["k"]].t().contiguous())}
