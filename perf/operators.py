"""Cases of the operators of a model's output head: products of 8-bit floats with a scale for each block of 128 and the
quantizer in front of them, log probabilities of given tokens, and distillation from a teacher's top log probabilities.

`own = False` computes each in elementary torch operations, `own = True` through the library's entry points.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 128


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one token's activations in front of a product, and a layer's in both forms for a training step's three products
        dict(name="quantize one token", op="quantize", nodes=1, rows=1, cols=4096, dtype="bf16", both=False),
        dict(name="quantize 8192x8192 both", op="quantize", nodes=1, rows=8192, cols=8192, dtype="bf16", both=True),
        # a served token, a batch of nodes with ragged sizes, the weight gradient of a large layer added to what is there
        dict(name="matmul one token", op="matmul", nodes=1, M=1, N=4096, K=4096, dtype="bf16", bias=False, addend=False),
        dict(name="matmul 4 nodes ragged", op="matmul", nodes=4, M=1500, N=1000, K=1000, dtype="fp32", bias=True, addend=False),
        dict(name="matmul 8192 gradient", op="matmul", nodes=1, M=8192, N=8192, K=8192, dtype="fp32", bias=False, addend=True),
        # a served token with its alternatives, an evaluation, a policy's log probabilities with their gradient on odd rows
        dict(name="logprobs one token", op="logprobs", rows=1, V=131072, dtype="bf16", k=20, temperature=0.7, train=False),
        dict(name="logprobs 2048 rows", op="logprobs", rows=2048, V=131072, dtype="bf16", k=8, temperature=1.0, train=False),
        dict(name="logprobs training odd", op="logprobs", rows=1999, V=50021, dtype="fp32", k=0, temperature=1.0, train=True),
        # the ten classes of this repository's networks on 40 nodes, a teacher's list renormalised, a language model's head
        dict(name="distill 40 nodes 10 classes", op="distill", nodes=40, B=32, V=10, dtype="fp32", k=3, temperature=2.0, tail=True),
        dict(name="distill 8 nodes 32003", op="distill", nodes=8, B=64, V=32003, dtype="fp32", k=32, temperature=1.0, tail=False),
        dict(name="distill 4 nodes 131072", op="distill", nodes=4, B=1024, V=131072, dtype="bf16", k=64, temperature=1.0, tail=True),
    ]


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("quantize", "matmul", "logprobs", "distill"))
    if op == "quantize":
        dtype = rng.choice(("fp32", "bf16", "fp16"))
        nodes, rows = rng.choice((1, 1, 2, 5)), _log_between(rng, 1, 8192)
        cols = min(_log_between(rng, 16, 16384), (1 << 25) // (nodes * rows))
        return dict(op=op, nodes=nodes, rows=rows, cols=max(cols, 1), dtype=dtype, both=rng.random() < 0.5)
    if op == "matmul":
        nodes, M = rng.choice((1, 1, 2, 6)), _log_between(rng, 1, 8192)
        N, K = _log_between(rng, 16, 8192), _log_between(rng, 16, 8192)
        while nodes * M * N * K > 1 << 39:
            K = (K + 1) // 2
        return dict(op=op, nodes=nodes, M=M, N=N, K=K, dtype=rng.choice(("fp32", "bf16")), bias=rng.random() < 0.5,
                    addend=rng.random() < 0.3)
    V = _log_between(rng, 10, 200000)
    dtype = rng.choice(("fp32", "bf16", "fp16"))
    temperature = rng.choice((1.0, 0.7, 2.0))
    if op == "logprobs":
        rows = min(_log_between(rng, 1, 8192), (1 << 28) // V)
        return dict(op=op, rows=rows, V=V, dtype=dtype, k=min(V, rng.choice((0, 1, 5, 20, 64))), temperature=temperature,
                    train=rng.random() < 0.4)
    nodes = rng.choice((1, 4, 16))
    B = max(1, min(_log_between(rng, 1, 1024), (1 << 28) // (nodes * V)))
    return dict(op=op, nodes=nodes, B=B, V=V, dtype=dtype, k=min(V, rng.choice((1, 3, 16, 64, 100))), temperature=temperature,
                tail=rng.random() < 0.6)


# ------------------------------------------------------------------ plain forms
def _blocks(x):
    pad = -x.shape[-1] % BLOCK
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, BLOCK))


def _quantize(x):
    """Codes (e4m3, shape of x) and exponents (int32) of the blocks of 128 along the last dimension of x."""
    xb = _blocks(x.float())
    mantissa, exponent = torch.frexp(xb.abs().amax(-1))               # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).int()                       # least e with amax <= 448 * 2^e = 0.875 * 2^(9 + e)
    e = torch.where(mantissa == 0, 0, e).clamp(-127, 127)
    codes = (xb * torch.exp2(-e.float()).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return codes.flatten(-2)[..., :x.shape[-1]], e


def _scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _dequantized(q, s, cols, dtype):
    """Values of codes [.., rows, pitch] with scale bytes [.., rows, pitch of scales]."""
    nb = -(-cols // BLOCK)
    v = _blocks(q[..., :cols].view(torch.float8_e4m3fn).to(dtype))
    return (v * torch.exp2(s[..., :nb].to(dtype) - 127).unsqueeze(-1)).flatten(-2)[..., :cols]


def _matmul(st, dtype):
    a, b = (_dequantized(st[q], st[s], st["K"], dtype) for q, s in (("A", "sA"), ("B", "sB")))
    c = torch.matmul(a, b.transpose(1, 2))
    if st["bias"] is not None:
        c = c + st["bias"].to(dtype).unsqueeze(1)
    if st["addend"] is not None:
        c = c + st["addend"].to(dtype)
    return c


def _top(z, k):
    """The k largest values' positions, the lower position first among equals."""
    bits = (z + 0.0).view(torch.int32).long()
    ordered = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    key = (ordered << 32) - torch.arange(z.shape[-1], device=z.device)
    return torch.topk(key, k, dim=-1, sorted=True).indices


def _logprobs(st):
    z = st["logits"].float() / st["temperature"]
    m = z.amax(-1, keepdim=True)
    shifted = z - m
    e = torch.exp(shifted)
    total = e.sum(-1, keepdim=True)
    log_total = torch.log(total)
    logp = shifted - log_total
    p = e / total
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    at = st["tokens"].long().unsqueeze(1)
    out = {"logprob": logp.gather(1, at).squeeze(1), "entropy": entropy, "lse": (m + log_total).squeeze(1)}
    if st["k"]:
        index = _top(st["logits"].float(), st["k"])
        out["top_logprob"], out["top_index"] = logp.gather(1, index), index.int()
    if st["train"]:
        g, h = st["d_logprob"].unsqueeze(1), st["d_entropy"].unsqueeze(1)
        d = -torch.where(p > 0, p * (g + h * (logp + entropy.unsqueeze(1))), 0.0)
        d.scatter_add_(1, at, g)
        out["dlogits"] = (d / st["temperature"]).to(st["logits"].dtype)
    return out


def _distill(st):
    rows, V = st["logits"].shape
    z = st["logits"].float() / st["temperature"]
    given = st["teacher_index"] >= 0
    at = torch.where(given, st["teacher_index"], 0).long()
    listed_ = torch.zeros(rows, V + 1, dtype=torch.bool, device=z.device)
    listed_.scatter_(1, torch.where(given, at, V), True)
    listed_ = listed_[:, :V]
    m = z.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))
    logt = torch.where(given, st["teacher_logprob"], -math.inf).double()
    if st["tail"]:
        t = torch.exp(logt)
        rest = (1 - t.sum(-1, keepdim=True)).clamp(min=0)
    else:
        t = torch.nan_to_num(torch.softmax(logt, -1), nan=0.0)
        rest = torch.zeros_like(t[:, :1])
        logt = torch.log(t)
    loss = torch.where(t > 0, t * (logt - (z.gather(1, at) - lse).double()), 0.0).sum(-1, keepdim=True)
    total, outside = t.sum(-1, keepdim=True), 0.0
    if st["tail"]:                                                    # one more class, where any token is outside the list
        zr = torch.where(listed_, -math.inf, z)
        mr = zr.amax(-1, keepdim=True).clamp(min=-3e38)
        sr = torch.exp(zr - mr).sum(-1, keepdim=True)
        lse_r = mr + torch.log(sr)
        some = (rest > 0) & (sr > 0)
        loss += torch.where(some, rest * (torch.log(rest) - (lse_r - lse).double()), 0.0)
        total = total + torch.where(some, rest, 0.0)
        outside = torch.where(some & ~listed_, rest.float() * torch.exp(z - lse_r), 0.0)
    d = torch.exp(z - lse) * total.float()
    d.scatter_add_(1, at, -t.float())
    d -= outside
    w = st["row_weight"].unsqueeze(1)
    loss = torch.where(w != 0, loss, 0.0)
    d = torch.where(w != 0, d * (w / (st["B"] * st["temperature"])), 0.0)
    per_node = (loss * w).view(st["nodes"], st["B"]).mean(1)
    return {"loss": per_node.float(), "row_loss": loss.squeeze(1).float(), "dlogits": d.to(st["logits"].dtype)}


def _plain(st):
    if st["op"] == "quantize":
        q, e = _quantize(st["x"])
        out = {"q": q, "scale": _scales(e)}
        if st["both"]:
            q, e = _quantize(st["x"].transpose(1, 2))
            out |= {"qt": q, "scale_t": _scales(e)}
        return out
    if st["op"] == "matmul":
        return {"C": _matmul(st, torch.float32).to(st["dtype"])}
    return _logprobs(st) if st["op"] == "logprobs" else _distill(st)


# ------------------------------------------------------------------ the library's calls
def _buffers(st):
    """What a user's program allocates once."""
    from paper_2111_09389_b200 import api
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    b = {"api": api}
    if st["op"] == "quantize":
        n, r, c = st["x"].shape
        b["q"] = new(n, r, api.lpdt_e4m3_pitch(c), dtype=torch.uint8)
        b["scale"] = new(n, r, api.lpdt_e4m3_scale_pitch(c), dtype=torch.uint8)
        if st["both"]:
            b["qt"] = new(n, c, api.lpdt_e4m3_pitch(r), dtype=torch.uint8)
            b["scale_t"] = new(n, c, api.lpdt_e4m3_scale_pitch(r), dtype=torch.uint8)
    elif st["op"] == "matmul":
        b["C"] = new(st["nodes"], st["M"], st["N"], dtype=st["dtype"])
    elif st["op"] == "logprobs":
        rows = st["logits"].shape[0]
        b |= {n: new(rows) for n in ("logprob", "entropy", "lse")}
        if st["k"]:
            b |= {"top_logprob": new(rows, st["k"]), "top_index": new(rows, st["k"], dtype=torch.int32)}
        if st["train"]:
            b["dlogits"] = torch.empty_like(st["logits"])
    else:
        b |= {"loss": new(st["nodes"]), "row_loss": new(st["nodes"] * st["B"]), "dlogits": torch.empty_like(st["logits"])}
    return b


def _own(st):
    if "buffers" not in st:
        st["buffers"] = _buffers(st)
    b = st["buffers"]
    api = b["api"]
    if st["op"] == "quantize":
        n, r, c = st["x"].shape
        api.lpdt_quantize_e4m3(st["x"], n, r, c, b["q"], b["scale"], b.get("qt"), b.get("scale_t"))
        blocks = lambda v: -(-v // BLOCK)  # noqa: E731
        out = {"q": b["q"].view(torch.float8_e4m3fn)[..., :c], "scale": b["scale"].view(torch.float8_e8m0fnu)[..., :blocks(c)]}
        if st["both"]:
            out |= {"qt": b["qt"].view(torch.float8_e4m3fn)[..., :r],
                    "scale_t": b["scale_t"].view(torch.float8_e8m0fnu)[..., :blocks(r)]}
        return out
    if st["op"] == "matmul":
        api.lpdt_matmul_e4m3(st["nodes"], st["M"], st["N"], st["K"], st["A"], st["sA"], st["B"], st["sB"], b["C"],
                             bias=st["bias"], bias_node_stride=st["N"], addend=st["addend"])
        return {"C": b["C"]}
    if st["op"] == "logprobs":
        rows, V = st["logits"].shape
        api.lpdt_token_logprobs(rows, V, st["logits"], st["tokens"], b["logprob"], b["entropy"], b["lse"],
                                b.get("top_logprob"), b.get("top_index"), top_k=st["k"], temperature=st["temperature"])
        if st["train"]:
            api.lpdt_token_logprobs_bwd(rows, V, st["logits"], st["tokens"], b["lse"], b["entropy"], b["dlogits"],
                                        d_logprob=st["d_logprob"], d_entropy=st["d_entropy"], temperature=st["temperature"])
        return {n: b[n] for n in ("logprob", "entropy", "lse", "top_logprob", "top_index", "dlogits") if n in b}
    api.lpdt_distill_topk(st["nodes"], st["B"], st["logits"].shape[1], st["logits"], st["k"], st["teacher_logprob"],
                          st["teacher_index"], b["loss"], b["row_loss"], dlogits=b["dlogits"], row_weight=st["row_weight"],
                          tail=st["tail"], temperature=st["temperature"])
    return {n: b[n] for n in ("loss", "row_loss", "dlogits")}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ inputs
def _gaussian(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _uniform(g, low, high, *shape):
    return torch.empty(*shape, device="cuda").uniform_(low, high, generator=g)


def _operand(g, nodes, rows, cols):
    """Codes and scale bytes of a matrix whose rows differ in size, laid out as the library has them: rows of a multiple
    of 16 bytes, scales of a multiple of 4."""
    x = _gaussian(g, nodes, rows, cols) * torch.exp(_gaussian(g, nodes, rows, 1))
    codes, e = _quantize(x)
    q = torch.zeros(nodes, rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda")
    s = torch.zeros(nodes, rows, -(-e.shape[-1] // 4) * 4, dtype=torch.uint8, device="cuda")
    q[..., :cols] = codes.view(torch.uint8)
    s[..., :e.shape[-1]] = (e + 127).to(torch.uint8)
    return q, s


def _logits(g, rows, V, dtype):
    """Logits of a head: a broad bulk, a few tokens ahead of it in each row."""
    z = _gaussian(g, rows, V, dtype=dtype) * 2.0
    ahead = torch.randint(0, V, (rows, 8), generator=g, device="cuda")
    z.scatter_(1, ahead, _uniform(g, 5, 14, rows, 8).to(dtype))
    return z


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    st = {"op": case["op"]}
    if case["op"] == "quantize":
        n, r, c = case["nodes"], case["rows"], case["cols"]
        x = _gaussian(g, n, r, c) * torch.exp(2 * _gaussian(g, n, r, 1))
        return st | {"x": x.to(dtype), "both": case["both"]}
    if case["op"] == "matmul":
        n, M, N, K = (case[d] for d in ("nodes", "M", "N", "K"))
        A, sA = _operand(g, n, M, K)
        B, sB = _operand(g, n, N, K)
        bias = _gaussian(g, n, N) if case["bias"] else None
        addend = (_gaussian(g, n, M, N) * math.sqrt(K)).to(dtype) if case["addend"] else None
        return st | dict(nodes=n, M=M, N=N, K=K, A=A, sA=sA, B=B, sB=sB, bias=bias, addend=addend, dtype=dtype)
    V, k = case["V"], case["k"]
    rows = case["rows"] if case["op"] == "logprobs" else case["nodes"] * case["B"]
    logits = _logits(g, rows, V, dtype)
    st |= {"logits": logits, "k": k, "temperature": case["temperature"]}
    if case["op"] == "logprobs":
        tokens = torch.randint(0, V, (rows,), generator=g, device="cuda")
        if V >= 256:                                                  # a vocabulary of which some rows may use a part
            logits[::4, 3:V // 8] = -math.inf
            tokens = torch.where((tokens >= 3) & (tokens < V // 8), 0, tokens)
        st |= {"tokens": tokens.int(), "train": case["train"]}
        if case["train"]:
            st |= {"d_logprob": _gaussian(g, rows), "d_entropy": 0.01 * _gaussian(g, rows)}
        return st
    first = torch.randint(0, V, (rows, 1), generator=g, device="cuda")
    step = torch.randint(1, V // k + 1, (rows, 1), generator=g, device="cuda")
    index = (first + step * torch.arange(k, device="cuda")) % V
    logits.scatter_(1, index, (logits.gather(1, index).float() + _uniform(g, 1, 8, rows, k)).to(dtype))
    mass = _uniform(g, 0.5, 0.98, rows, 1)
    value = torch.log_softmax(2 * _gaussian(g, rows, k).sort(-1, descending=True).values, -1) + torch.log(mass)
    if k > 1:
        index[1::8, k // 2:] = -1                                     # shorter lists
    weight = _uniform(g, 0.5, 1.5, rows)
    weight[5::16] = 0                                                 # padding of the batch
    return st | dict(nodes=case["nodes"], B=case["B"], tail=case["tail"], teacher_logprob=value.contiguous(),
                     teacher_index=index.int().contiguous(), row_weight=weight)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "quantize":
        n = case["nodes"] * case["rows"] * case["cols"]
        return {"bytes": n * size + n * (1 + 1 / BLOCK) * (2 if case["both"] else 1), "flops": 2 * n}
    if case["op"] == "matmul":
        n, M, N, K = (case[d] for d in ("nodes", "M", "N", "K"))
        out = n * M * N * size * (2 if case["addend"] else 1) + (4 * n * N if case["bias"] else 0)
        return {"bytes": n * (M + N) * K * (1 + 1 / BLOCK) + out, "flops": 2 * n * M * N * K}
    rows = case["rows"] if case["op"] == "logprobs" else case["nodes"] * case["B"]
    n = rows * case["V"]
    if case["op"] == "logprobs":
        return {"bytes": n * size * (2 if case["train"] else 1) + rows * (16 + 8 * case["k"] + (8 if case["train"] else 0)),
                "flops": n * (12 if case["train"] else 6)}
    return {"bytes": 2 * n * size + rows * (8 + 8 * case["k"]), "flops": 10 * n}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_quantize(x):
    n, r, c = x.shape
    values, scales = torch.empty(n, r, c, dtype=torch.float64, device=x.device), []
    for at in range(0, c, BLOCK):
        part = x[..., at:at + BLOCK].double()
        amax = part.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(amax / 448)).clamp(-127, 127)
        e = torch.where(amax > 448 * torch.exp2(e), e + 1, torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e)).clamp(min=-127)
        e = torch.where(amax == 0, 0.0, e)
        v = part / torch.exp2(e)
        unit = torch.exp2(torch.floor(torch.log2(v.abs())).clamp(min=-6) - 3)        # spacing of the type at v
        values[..., at:at + BLOCK] = torch.round(v / unit) * unit                    # halves go to the even neighbour
        scales.append(torch.exp2(e))
    return values, torch.cat(scales, -1)


def _exact_rows(case, st, rows):
    """Outputs of the rows in the slice `rows`."""
    x = st["logits"][rows].double() / case["temperature"]
    logp = torch.log_softmax(x, -1)
    p = logp.exp()
    if case["op"] == "logprobs":
        token = st["tokens"][rows].long()
        at = torch.arange(len(token), device=x.device)
        plogp = torch.nan_to_num(p * logp, nan=0.0)
        entropy = -plogp.sum(-1)
        out = {"logprob": logp[at, token], "entropy": entropy, "lse": torch.logsumexp(x, -1)}
        if case["k"]:
            order = torch.sort(st["logits"][rows].double(), dim=-1, descending=True, stable=True).indices[:, :case["k"]]
            out["top_logprob"], out["top_index"] = logp.gather(1, order), order.int()
        if case["train"]:
            g, h = st["d_logprob"][rows].double(), st["d_entropy"][rows].double()
            onehot = torch.zeros_like(p)
            onehot[at, token] = 1
            out["dlogits"] = ((onehot - p) * g[:, None] - (plogp + p * entropy[:, None]) * h[:, None]) / case["temperature"]
        return out
    index, value = st["teacher_index"][rows].long(), st["teacher_logprob"][rows].double()
    target, inside = torch.zeros_like(p), torch.zeros_like(p)
    loss = torch.zeros(len(p), dtype=torch.float64, device=p.device)
    t = torch.where(index >= 0, value.exp(), 0.0)
    if not case["tail"]:
        t = t / t.sum(-1, keepdim=True)
    for j in range(case["k"]):
        some = index[:, j] >= 0
        at = index[:, j].clamp(min=0)[:, None]
        target.scatter_add_(1, at, t[:, j:j + 1])
        inside.scatter_add_(1, at, some[:, None].double())
        loss += torch.where(some, t[:, j] * (torch.log(t[:, j]) - logp.gather(1, at)[:, 0]), 0.0)
    grad = p * target.sum(-1, keepdim=True) - target
    if case["tail"]:
        remains = (1 - target.sum(-1)).clamp(min=0)
        outside = torch.where(inside > 0, 0.0, p)
        mass = outside.sum(-1)
        some = (remains > 0) & (mass > 0)
        loss += torch.where(some, remains * torch.log(remains / mass), 0.0)
        share = outside / mass[:, None]
        grad += torch.where(some[:, None], remains[:, None] * (p - share), 0.0)
    weight = st["row_weight"][rows].double()
    loss = torch.where(weight == 0, 0.0, loss)
    return {"row_loss": loss, "dlogits": grad * weight[:, None] / (case["B"] * case["temperature"]), "weighted": loss * weight}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "quantize":
        values, scale = _exact_quantize(st["x"])
        out = {"q": values, "scale": scale}
        if case["both"]:
            out["qt"], out["scale_t"] = _exact_quantize(st["x"].transpose(1, 2))
        return out
    if case["op"] == "matmul":
        nb = -(-case["K"] // BLOCK)
        value = lambda q, s: (q.view(torch.float8_e4m3fn)[..., :case["K"]].double()  # noqa: E731
                              * torch.exp2(s[..., :nb].double() - 127).repeat_interleave(BLOCK, -1)[..., :case["K"]])
        c = torch.einsum("nmk,njk->nmj", value(st["A"], st["sA"]), value(st["B"], st["sB"]))
        c += 0 if st["bias"] is None else st["bias"].double()[:, None]
        c += 0 if st["addend"] is None else st["addend"].double()
        return {"C": c}
    total, V = st["logits"].shape
    step = max(1, (1 << 26) // V)
    parts = [_exact_rows(case, st, slice(r, r + step)) for r in range(0, total, step)]
    out = {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
    if case["op"] == "distill":
        out["loss"] = out.pop("weighted").view(case["nodes"], case["B"]).mean(1)
    return out
