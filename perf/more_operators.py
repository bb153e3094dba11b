"""Operators between hidden states and tokens, as cases that can be timed and checked.

A receiver of weights answers with tokens that a small model drafts and a large one verifies; the small one learns from the large one's
top logits.

  norm     layer norm (with mean and bias) or root mean square norm of rows, forward; or backward, with the gradients of the
           weight and the bias, which are sums over all rows
  distill  the divergence of a student's distribution from that of a teacher's top logits; or its gradient for all logits; or both
  verify   drafted tokens accepted or refused by the ratio of two models' probabilities and given random numbers, and the next token
           sampled from what the draft left over, or from the target where everything was accepted
  adapter  low-rank adapters, another one for each request, added to the product that all requests share

`run` computes a case in plain torch operations, or, where `own` is set, with this library's kernels.  Sizes are those of the
workloads (decoders of 7B, 8B and 32B weights and their tensor-parallel shards), or generic.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
_CHUNK = 1 << 28


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step of 64 sequences of an 8B-style decoder: the norm in front of a product
        dict(name="norm_decode", op="norm", way="forward", rows=64, cols=4096, center=False, x="bf16", y="bf16", w="bf16", pad=0),
        # a chunk of prompts, or a micro-batch, of a 32B-style decoder
        dict(name="norm_batch", op="norm", way="forward", rows=16384, cols=5120, center=False, x="bf16", y="bf16", w="bf16", pad=0),
        # the backward pass of a layer norm with a bias over such a micro-batch, gradients of the parameters in fp32
        dict(name="norm_backward", op="norm", way="backward", rows=16384, cols=5120, center=True, x="bf16", y="bf16", w="bf16",
             pad=0, accumulate=False),
        # a few tokens of a small vocabulary in fp32, loss and gradient: a short sequence, or a test
        dict(name="distill_few", op="distill", way="both", rows=7, cols=32000, top=20, logits="f32", temperature=2.0, pad=0, index=64),
        # the loss alone over a batch for evaluation, logits of a 7B-style head at odd strides
        dict(name="distill_eval", op="distill", way="loss", rows=8191, cols=32000, top=50, logits="bf16", temperature=1.0, pad=3, index=32),
        # a micro-batch of 4096 tokens with an 8B-style vocabulary: what a training step makes of the logits
        dict(name="distill_train", op="distill", way="both", rows=4096, cols=151936, top=64, logits="bf16", temperature=1.0, pad=0,
             index=32),
        # one sequence, four drafted tokens: latency
        dict(name="verify_one", op="verify", requests=1, most=4, cols=32000, probs="f32", drafts=True, noise=0.5, index=64),
        # 64 sequences with up to eight drafted tokens each, an 8B-style vocabulary
        dict(name="verify_batch", op="verify", requests=64, most=8, cols=151936, probs="f32", drafts=True, noise=0.7, index=64),
        # 200 sequences whose drafts were looked up in their own text: no probabilities, few accepted
        dict(name="verify_lookup", op="verify", requests=200, most=5, cols=152064, probs="bf16", drafts=False, noise=2.0, index=32),
        # one token through an adapter of an attention output projection
        dict(name="adapter_token", op="adapter", m=1, n=4096, k=4096, rank=16, adapters=8, run=1, out="bf16", pad=0),
        # a decode step of 96 sequences, each with one of 40 adapters or none, a shard of a 32B-style gate and up projection
        dict(name="adapter_decode", op="adapter", m=96, n=6912, k=5120, rank=32, adapters=40, run=1, out="bf16", pad=0),
        # prompts of about 300 tokens, each with its adapter
        dict(name="adapter_prompt", op="adapter", m=8192, n=6912, k=5120, rank=64, adapters=16, run=300, out="f32", pad=0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, step):
    """The same, a multiple of `step` half of the time."""
    n = _log(rng, lo, hi)
    return max(lo, n // step * step) if rng.random() < 0.5 else n


def _any(rng):
    op = rng.choice(("norm", "distill", "verify", "adapter"))
    if op == "norm":
        way = rng.choice(("forward", "backward"))
        cols = _size(rng, 48, 8192, 64)
        c = dict(op=op, way=way, rows=_log(rng, 1, min(65536, (1 << 27) // cols)), cols=cols, center=rng.random() < 0.5,
                 x=rng.choice(("bf16", "bf16", "f32")), y=rng.choice(("bf16", "bf16", "f32")), w=rng.choice(("bf16", "f32")),
                 pad=rng.choice((0, 0, 8, 3)))
        return dict(c, accumulate=rng.random() < 0.4) if way == "backward" else c
    if op == "distill":
        cols = _size(rng, 1000, 152064, 64)
        return dict(op=op, way=rng.choice(("loss", "gradient", "both")), rows=_log(rng, 1, min(16384, (1 << 28) // cols)), cols=cols,
                    top=_log(rng, 1, 256), logits=rng.choice(("bf16", "bf16", "f32")), temperature=rng.choice((0.7, 1.0, 2.0)),
                    pad=rng.choice((0, 0, 8, 3)), index=rng.choice((32, 64)))
    if op == "verify":
        cols, most = _size(rng, 1000, 152064, 64), rng.randint(1, 12)
        return dict(op=op, requests=_log(rng, 1, max(1, min(256, (1 << 27) // (cols * (most + 1))))), most=most, cols=cols,
                    probs=rng.choice(("f32", "f32", "bf16")), drafts=rng.random() < 0.6, noise=rng.choice((0.3, 0.7, 2.0)),
                    index=rng.choice((32, 64)))
    k, n = _size(rng, 64, 16384, 32), _size(rng, 64, 16384, 16)
    return dict(op=op, m=_log(rng, 1, min(16384, (1 << 26) // max(n, k))), n=n, k=k, rank=rng.choice((4, 8, 16, 32, 64, 128, rng.randint(3, 100))),
                adapters=_log(rng, 1, 48), run=rng.choice((1, 1, 20, 300)), out=rng.choice(("bf16", "bf16", "f32")),
                pad=rng.choice((0, 0, 8, 3)))


def draw(rng):
    works = [work(c) for c in listed()]
    c = _any(rng)
    w = work(c)
    return c if all(w[k] <= max(v[k] for v in works) for k in w) else draw(rng)


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


def _ids(t, c):
    return t.to(torch.int32 if c["index"] == 32 else torch.int64)


def _uniform(n, g):
    return torch.rand(n, generator=g, device="cuda")


def _norm_inputs(c, s, g):
    rows, cols, dtype = c["rows"], c["cols"], DTYPES[c["w"]]
    s["x"] = _matrix(rows, cols, c["pad"], 1.0, DTYPES[c["x"]], g)
    s["x"] += 0.3
    s["weight"] = (_normal(cols, 0.1, torch.float32, g) + 1).to(dtype)
    s["bias"] = _normal(cols, 0.1, dtype, g) if c["center"] else None
    s["eps"] = 1e-5
    if c["way"] == "forward":
        s["out"] = torch.empty(rows, cols, dtype=DTYPES[c["y"]], device="cuda")
        s["mean"] = torch.empty(rows, device="cuda") if c["center"] else None
        s["rstd"] = torch.empty(rows, device="cuda")
        return
    # what the forward pass left behind
    x = s["x"].double() if rows * cols <= _CHUNK // 8 else s["x"].float()
    mean = x.mean(1) if c["center"] else torch.zeros(rows, dtype=x.dtype, device="cuda")
    s["rstd"] = ((x - mean[:, None]).square_().mean(1) + s["eps"]).rsqrt().float()
    s["mean"] = mean.float() if c["center"] else None
    s["dy"] = _matrix(rows, cols, 0, 1e-2, DTYPES[c["y"]], g)
    s["dx"] = torch.empty(rows, cols, dtype=DTYPES[c["x"]], device="cuda")
    s["dweight"] = _normal(cols, 1e-2, torch.float32, g)
    s["dbias"] = _normal(cols, 1e-2, torch.float32, g) if c["center"] else None


def _distill_inputs(c, s, g):
    rows, cols, top = c["rows"], c["cols"], c["top"]
    s["logits"] = _matrix(rows, cols, c["pad"], 2.0, DTYPES[c["logits"]], g)
    # a teacher's top logits come in descending order; the student has most of them high as well
    start = torch.randint(0, cols, (rows, 1), generator=g, device="cuda")
    step = torch.randint(1, max(2, cols // top), (rows, 1), generator=g, device="cuda")
    ids = (start + step * torch.arange(top, device="cuda")) % cols
    teacher = 9.0 - 1.5 * torch.arange(1, top + 1, device="cuda").float().log() + 0.3 * torch.randn(rows, top, generator=g, device="cuda")
    s["teacher"] = teacher.sort(1, descending=True)[0]
    s["logits"].scatter_(1, ids, (s["teacher"] + torch.randn(rows, top, generator=g, device="cuda")).to(s["logits"].dtype))
    # some rows have fewer entries, and some (a prompt's tokens) none
    kept = torch.where(_uniform(rows, g) < 0.3, (_uniform(rows, g) * (top + 1)).long(), top)
    kept[_uniform(rows, g) < 0.1] = 0
    if rows > 1:
        kept[0] = top
    s["ids"] = _ids(torch.where(torch.arange(top, device="cuda") < kept[:, None], ids, -1), c)
    s["d_loss"] = torch.where(kept > 0, 1.0 / rows, 0.0) * (0.5 + _uniform(rows, g))
    s["loss"], s["lse"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    if c["way"] == "gradient":           # what the forward pass left behind
        for a in range(0, rows, 1024):
            s["lse"][a:a + 1024] = torch.logsumexp(s["logits"][a:a + 1024].double() / c["temperature"], 1).float()
    if c["way"] != "loss":
        s["d_logits"] = torch.empty(rows, cols, dtype=DTYPES[c["logits"]], device="cuda")


def _verify_inputs(c, s, g):
    cols, requests = c["cols"], c["requests"]
    # (all lengths about as often, in some order: as many tokens with every seed)
    lengths = (c["most"] + torch.randperm(requests, generator=g, device="cuda")) % (c["most"] + 1)
    s["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)))
    drafted = int(s["offsets"][-1])
    request = torch.repeat_interleave(torch.arange(requests, device="cuda"), lengths)
    rows = torch.arange(drafted, device="cuda") + request            # the target's row of each drafted token
    dtype = DTYPES[c["probs"]]
    s["target"] = torch.empty(drafted + requests, cols, dtype=dtype, device="cuda")
    s["draft"] = torch.empty(drafted, cols, dtype=dtype, device="cuda") if c["drafts"] else None
    tokens = torch.empty(drafted, dtype=torch.int64, device="cuda")
    for a in range(0, drafted + requests, 256):
        b = min(a + 256, drafted + requests)
        z = torch.randn(b - a, cols, generator=g, device="cuda") * 4.0
        s["target"][a:b] = torch.softmax(z, 1).to(dtype)
        here = ((rows >= a) & (rows < b)).nonzero().view(-1)
        if len(here):
            q = torch.softmax(z[rows[here] - a] + c["noise"] * torch.randn(len(here), cols, generator=g, device="cuda"), 1).to(dtype)
            tokens[here] = torch.multinomial(q.float(), 1, generator=g).view(-1)
            if c["drafts"]:
                s["draft"][here] = q
    s["drafted"] = _ids(tokens, c)
    s["uniforms"] = _uniform(drafted + requests, g)
    s["tokens"] = _ids(torch.zeros(drafted + requests, device="cuda"), c)
    s["accepted"] = torch.zeros(requests, dtype=torch.int32, device="cuda")


def _adapter_inputs(c, s, g):
    m, n, k, rank, adapters = c["m"], c["n"], c["k"], c["rank"], c["adapters"]
    s["x"] = _matrix(m, k, c["pad"], 1.0, torch.bfloat16, g)
    s["down"] = _normal(adapters * rank * k, k ** -0.5, torch.bfloat16, g).view(adapters, rank, k)
    s["up"] = _normal(adapters * n * rank, rank ** -0.5, torch.bfloat16, g).view(adapters, n, rank)
    s["scales"] = 0.5 + _uniform(adapters, g)
    # requests of about `run` rows, the adapter of each; one of ten has none
    starts = _uniform(m, g) < 1.0 / c["run"]
    starts[0] = True
    request = starts.cumsum(0) - 1
    chosen = torch.randint(0, adapters, (m,), generator=g, device="cuda")
    chosen[_uniform(m, g) < 0.1] = -1
    chosen[0] = chosen[0].abs() % adapters
    s["chosen"] = chosen[request].to(torch.int32)
    s["out"] = _matrix(m, n, c["pad"], 1.0, DTYPES[c["out"]], g)


def prepare(case, seed):
    s = {"case": case}
    {"norm": _norm_inputs, "distill": _distill_inputs, "verify": _verify_inputs, "adapter": _adapter_inputs}[case["op"]](case, s, _gen(seed, 1))
    return s


# ---------------------------------------------------------------------------------------------------
# one pass, in plain operations
# ---------------------------------------------------------------------------------------------------
def _outputs(s):
    c = s["case"]
    names = {"forward": ("out", "mean", "rstd"), "backward": ("dx", "dweight", "dbias"), "loss": ("loss", "lse"), "gradient": ("d_logits",),
             "both": ("loss", "lse", "d_logits"), "verify": ("tokens", "accepted"), "adapter": ("out",)}[c.get("way", c["op"])]
    return {name: s[name] for name in names if s[name] is not None}


def _plain_norm(s):
    c, x, w = s["case"], s["x"].float(), s["weight"].float()
    if c["way"] == "forward":
        mean = x.mean(1) if c["center"] else None
        x = x - mean[:, None] if c["center"] else x
        rstd = 1.0 / (x.square().mean(1) + s["eps"]).sqrt()
        y = x * rstd[:, None] * w
        s["out"].copy_(y + s["bias"].float() if c["center"] else y)
        s["rstd"].copy_(rstd)
        if c["center"]:
            s["mean"].copy_(mean)
        return
    rstd, dy = s["rstd"][:, None], s["dy"].float()
    xhat = (x - s["mean"][:, None] if c["center"] else x) * rstd
    g = dy * w
    d = g - xhat * (g * xhat).mean(1, keepdim=True)
    s["dx"].copy_((d - g.mean(1, keepdim=True) if c["center"] else d) * rstd)
    s["dweight"].mul_(c["accumulate"]).add_((dy * xhat).sum(0))
    if c["center"]:
        s["dbias"].mul_(c["accumulate"]).add_(dy.sum(0))


def _plain_distill(s):
    c, t = s["case"], s["case"]["temperature"]
    z, ids = s["logits"].float(), s["ids"].long()
    here = ids >= 0
    at = torch.where(here, ids, 0)
    teacher = torch.where(here, s["teacher"], -math.inf)
    top = torch.where(here.any(1), teacher.amax(1), 0.0)[:, None]
    log_p = (teacher - top) / t
    total = log_p.exp().sum(1, keepdim=True)
    p = torch.where(total > 0, log_p.exp() / total, 0.0)
    if c["way"] == "gradient":
        q = (z / t - s["lse"][:, None]).exp_()
    else:
        most = z.amax(1, keepdim=True)
        q = ((z - most) / t).exp_()
        size = q.sum(1, keepdim=True)
        # (the loss is a small difference: in 64 bits but for the long sum)
        log_q = (z.gather(1, at) - most).double() / t - size.double().log()
        log_p = torch.where(p > 0, log_p.double() - total.double().log(), 0.0)
        s["loss"].copy_((p * (log_p - log_q)).sum(1))
        s["lse"].copy_((most.double() / t + size.double().log()).view(-1))
        q = q.div_(size) if c["way"] == "both" else q
    if c["way"] != "loss":
        d = q.mul_(here.any(1, keepdim=True))
        d.scatter_add_(1, at, -p)
        s["d_logits"].copy_(d.mul_((s["d_loss"] / t)[:, None]))


def _plain_verify(s):
    c, offsets, u = s["case"], s["offsets"], s["uniforms"]
    requests, drafted, ids = c["requests"], s["drafted"].numel(), s["drafted"].long()
    request = torch.arange(requests, device="cuda")
    first, lengths = offsets[:-1], offsets[1:] - offsets[:-1]
    place = torch.arange(c["most"], device="cuda")
    inside = place < lengths[:, None]
    at = torch.where(inside, first[:, None] + place, 0).clamp(max=max(0, drafted - 1))
    rows = at + request[:, None]
    p = s["target"][rows, ids[at]].double()
    q = s["draft"][at, ids[at]].double() if c["drafts"] else 1.0
    kept = ((u[rows].double() * q < p) & inside).long().cumprod(1)
    n = kept.sum(1)
    last, refused = first + request + n, n < lengths
    weights = s["target"][last].double()
    left = torch.where(refused, first + n, 0)
    if c["drafts"]:
        over = (weights - torch.where(refused[:, None], s["draft"][left].double(), 0.0)).clamp_(min=0)
    else:
        over = weights.scatter(1, ids[left][:, None], torch.where(refused, 0.0, weights[request, ids[left]])[:, None])
    weights = torch.where((over.sum(1) > 0)[:, None], over, weights)
    sums = weights.cumsum(1)
    sample = (sums <= (u[first + request + lengths].double() * sums[:, -1])[:, None]).sum(1).clamp(max=c["cols"] - 1)
    s["tokens"].fill_(-1)
    whole = torch.full((drafted + requests,), -1, dtype=torch.int64, device="cuda")
    whole.scatter_reduce_(0, rows.reshape(-1), torch.where(kept > 0, ids[at], -1).reshape(-1), "amax")
    whole[last] = sample
    s["tokens"].copy_(whole)
    s["accepted"].copy_(n)


def _plain_adapter(s):
    c, chosen = s["case"], s["chosen"].long()
    adapters, rank = c["adapters"], c["rank"]
    # the products with all adapters side by side, of which each row keeps its own
    h = (s["x"].float() @ s["down"].float().view(-1, c["k"]).t()).view(c["m"], adapters, rank)
    mine = torch.arange(adapters, device="cuda") == chosen[:, None]
    h = torch.where(mine[:, :, None], h * s["scales"][:, None], 0.0).view(c["m"], -1)
    s["out"].copy_(s["out"].float() + h @ s["up"].float().transpose(1, 2).reshape(-1, c["n"]))


def _plain(s):
    {"norm": _plain_norm, "distill": _plain_distill, "verify": _plain_verify, "adapter": _plain_adapter}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------------------------------
# one pass, with this library
# ---------------------------------------------------------------------------------------------------
def _kernels(s):
    import paper_2605_06534_amd as R

    c = s["case"]
    way = c.get("way")
    if way == "forward":
        R.layer_norm(s["x"], s["weight"], s["out"], bias=s["bias"], mean=s["mean"], rstd=s["rstd"], eps=s["eps"], center=c["center"])
    elif way == "backward":
        if "ws" not in s:                # made once and kept, as a program does
            s["ws"] = R.layer_norm_grad_workspace(c["rows"], c["cols"])
        R.layer_norm_grad(s["dy"], s["x"], s["weight"], s["rstd"], s["dx"], s["dweight"], s["ws"], mean=s["mean"], dbias=s["dbias"],
                          accumulate=c["accumulate"])
    elif way == "gradient":
        R.distill_grad(s["logits"], s["ids"], s["teacher"], s["lse"], s["d_loss"], s["d_logits"], temperature=c["temperature"])
    elif c["op"] == "distill":
        if "ws" not in s:
            s["ws"] = R.distill_workspace(c["rows"], c["cols"])
        if way == "loss":
            R.distill_loss(s["logits"], s["ids"], s["teacher"], s["loss"], s["lse"], s["ws"], temperature=c["temperature"])
        else:
            R.distill_loss_grad(s["logits"], s["ids"], s["teacher"], s["d_loss"], s["loss"], s["lse"], s["d_logits"], s["ws"],
                                temperature=c["temperature"])
    elif c["op"] == "verify":
        if "ws" not in s:
            s["ws"] = R.draft_verify_workspace(c["requests"], c["cols"])
        R.draft_verify(s["target"], s["draft"], s["drafted"], s["offsets"], s["uniforms"], s["tokens"], s["accepted"], s["ws"])
    else:
        if "weights" not in s:
            s["weights"] = R.Adapters(s["down"], s["up"], s["scales"])
            s["ws"] = R.adapter_linear_workspace(c["m"], s["weights"])
        R.adapter_linear(s["x"], s["weights"], s["chosen"], s["out"], s["ws"])


def run(state):
    if own:
        _kernels(state)
    else:
        _plain(state)
    return _outputs(state)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "norm":
        cells = c["rows"] * c["cols"]
        if c["way"] == "forward":
            return {"bytes": cells * (SIZE[c["x"]] + SIZE[c["y"]]) + c["cols"] * SIZE[c["w"]] * (1 + c["center"]) + c["rows"] * 4 * (1 + c["center"]),
                    "flops": cells * (7 if c["center"] else 4)}
        return {"bytes": cells * (2 * SIZE[c["x"]] + SIZE[c["y"]]) + c["cols"] * (SIZE[c["w"]] + 4 * (1 + c["center"]) * (1 + c["accumulate"])) +
                c["rows"] * 4 * (1 + c["center"]), "flops": cells * (14 if c["center"] else 11)}
    if c["op"] == "distill":
        cells, passes = c["rows"] * c["cols"], 1 if c["way"] == "loss" else 2
        return {"bytes": passes * cells * SIZE[c["logits"]] + c["rows"] * c["top"] * (c["index"] // 8 + 4) + c["rows"] * 8,
                "flops": cells * {"loss": 4, "gradient": 4, "both": 8}[c["way"]]}
    if c["op"] == "verify":
        # a row of the target for each request, and one of the draft where something is refused: nearly always where drafts are many
        rows = c["requests"] * (1 + c["drafts"] * c["most"] / (c["most"] + 1))
        return {"bytes": rows * c["cols"] * SIZE[c["probs"]], "flops": rows * c["cols"] * 2}
    used = c["adapters"] * (1 - (1 - 1 / c["adapters"]) ** (c["m"] / c["run"]))
    rows = max(1.0, 0.9 * c["m"])
    return {"bytes": rows * (2 * c["k"] + 2 * SIZE[c["out"]] * c["n"]) + max(1.0, used) * c["rank"] * 2 * (c["k"] + c["n"]) + 4 * c["m"],
            "flops": 2 * rows * c["rank"] * (c["k"] + c["n"])}


# ---------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------
def _exact_norm(s, c):
    parts, weight = [], s["weight"].double()
    dweight, dbias = torch.zeros_like(weight), torch.zeros_like(weight)
    for a in range(0, c["rows"], 2048):
        x = s["x"][a:a + 2048].double()
        if c["way"] == "forward":
            mean = x.sum(1) / c["cols"] if c["center"] else torch.zeros(len(x), dtype=torch.float64, device="cuda")
            x -= mean[:, None]
            rstd = ((x * x).sum(1) / c["cols"] + s["eps"]) ** -0.5
            parts.append((x * rstd[:, None] * weight + (s["bias"].double() if c["center"] else 0.0), mean, rstd))
            continue
        rstd, dy = s["rstd"][a:a + 2048, None].double(), s["dy"][a:a + 2048].double()
        if c["center"]:
            x -= s["mean"][a:a + 2048, None].double()
        x *= rstd
        dweight += torch.einsum("ij,ij->j", dy, x)
        dbias += dy.sum(0)
        dy *= weight
        along = torch.einsum("ij,ij->i", dy, x) / c["cols"]
        middle = dy.sum(1) / c["cols"] if c["center"] else torch.zeros_like(along)
        parts.append(((dy - middle[:, None] - along[:, None] * x) * rstd,))
    whole = [torch.cat(p) for p in zip(*parts)]
    if c["way"] == "forward":
        return {"out": whole[0], **({"mean": whole[1]} if c["center"] else {}), "rstd": whole[2]}
    if c["accumulate"]:
        dweight += s["dweight"].double()
        dbias += s["dbias"].double() if c["center"] else 0.0
    return {"dx": whole[0], "dweight": dweight, **({"dbias": dbias} if c["center"] else {})}


def _exact_distill(s, c):
    t, out = c["temperature"], {name: [] for name in ("loss", "lse", "d_logits")}
    for a in range(0, c["rows"], 512):
        z = s["logits"][a:a + 512].double() / t
        ids, teacher = s["ids"][a:a + 512].long(), s["teacher"][a:a + 512].double() / t
        teacher[ids < 0] = -math.inf
        empty = (ids < 0).all(1)
        p = torch.softmax(teacher, 1).masked_fill(empty[:, None], 0.0)
        lse = torch.logsumexp(z, 1)
        log_ratio = torch.log(p.clamp(min=1e-300)) - z.gather(1, ids.clamp(min=0)) + lse[:, None]
        out["loss"].append((p * log_ratio).sum(1))
        out["lse"].append(lse)
        if c["way"] != "loss":
            used = s["lse"][a:a + 512].double() if c["way"] == "gradient" else lse
            q = torch.exp(z - used[:, None]).masked_fill_(empty[:, None], 0.0)
            spare = torch.cat((q, torch.zeros_like(q[:, :1])), 1)                 # a column for the entries that are not there
            spare.scatter_add_(1, torch.where(ids < 0, c["cols"], ids), -p)
            d = spare[:, :-1] * (s["d_loss"][a:a + 512].double() / t)[:, None]
            out["d_logits"].append(d if c["rows"] * c["cols"] <= _CHUNK else d.float())
    wanted = {"loss": ("loss", "lse"), "gradient": ("d_logits",), "both": ("loss", "lse", "d_logits")}[c["way"]]
    return {name: torch.cat(out[name]) for name in wanted}


def _exact_verify(s, c):
    offsets, ids, u = s["offsets"].tolist(), s["drafted"].tolist(), s["uniforms"].double().tolist()
    tokens, accepted = [], []
    for r in range(c["requests"]):
        a, b = offsets[r], offsets[r + 1]
        n, row = 0, a + r
        while a + n < b:
            d = ids[a + n]
            q = float(s["draft"][a + n, d]) if c["drafts"] else 1.0
            if not u[row + n] * q < float(s["target"][row + n, d]):
                break
            n += 1
        w = s["target"][row + n].double().cpu().numpy()
        if a + n < b:
            q = np.zeros_like(w)
            if c["drafts"]:
                q = s["draft"][a + n].double().cpu().numpy()
            else:
                q[ids[a + n]] = w[ids[a + n]]
            over = np.maximum(w - q, 0.0)
            w = over if over.any() else w
        sums = np.cumsum(w)
        token = int(np.searchsorted(sums, u[row + b - a] * sums[-1], side="right"))
        tokens += ids[a:a + n] + [min(token, c["cols"] - 1)] + [-1] * (b - a - n)
        accepted.append(n)
    return {"tokens": torch.tensor(tokens), "accepted": torch.tensor(accepted)}


def _exact_adapter(s, c):
    out = s["out"].double()
    for a in range(c["adapters"]):
        rows = (s["chosen"] == a).nonzero().view(-1)
        if len(rows):
            h = torch.mm(s["x"][rows].double(), s["down"][a].double().t().contiguous())
            out[rows] += torch.mm(h * s["scales"][a].double(), s["up"][a].double().t().contiguous())
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "distill": _exact_distill, "verify": _exact_verify, "adapter": _exact_adapter}[case["op"]](s, case)
