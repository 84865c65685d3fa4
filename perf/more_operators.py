"""The ends of a token policy's learner step, operator by operator, as they are timed
and compared: with ``own`` false in plain torch operations, with ``own`` true through
this library's calls.

  embed           the network's inputs: rows of the vocabulary's table [V, H], scaled
  embed_grad      the table's gradient, summed over the steps of each token, alone or
                  on top of the gradient that the tied output layer left
  orthogonalize   updates made nearly orthogonal by Newton-Schulz products

A token of -1 marks a step that takes no part (a prompt, or the padding behind a
sequence).
"""

import math

import torch

own = False

MOST_EMBED = 65536 * 2048  # steps times H of a drawn lookup
MOST_EMBED_GRAD = 65536 * 2048
MOST_TABLE = 131072 * 4096  # V times H of either
MOST_PRODUCTS = 6e12  # operations of a drawn set of updates, bfloat16
MOST_WIDE_PRODUCTS = 6e11  # and float32
STEPS, COEFFICIENTS = 5, (3.4445, -4.7750, 2.0315)
EPSILON = 1e-7
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _embed(name, op, T, B, H, V, **options):
    c = dict(op=op, T=T, B=B, H=H, V=V, scale=1.0, ragged=False, text=True, table="bf16", steps="bf16", tied=False)
    c.update(options)
    return dict(c, name=name) if name else c


def _updates(name, shapes, dtype):
    """shapes: "rows x columns * how many" of each kind of matrix."""
    c = dict(op="orthogonalize", shapes=shapes, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One step of 48 actors: their last tokens' rows, a vocabulary of odd size.
        _embed("embed_actors", "embed", 1, 48, 2048, 100003),
        # The DeepMind Lab learner batch (unroll 100, 32 trajectories), float32 master
        # rows scaled by sqrt(H) and rounded for the network, ragged.
        _embed("embed_learner", "embed", 100, 32, 1024, 32768, scale=32.0, ragged=True, table="f32"),
        # A long batch of answers: the largest lookup.
        _embed("embed_long", "embed", 4096, 16, 2048, 131072),
        # The Atari learner batch (unroll 20, 32 trajectories), added to the tied layer's gradient.
        _embed("embed_grad_small", "embed_grad", 20, 32, 256, 32768, table="f32", steps="f32", tied=True),
        # The DeepMind Lab learner batch, mixed precision, a table of its own.
        _embed("embed_grad_learner", "embed_grad", 100, 32, 1024, 32768, scale=32.0),
        # Odd everything: ragged lanes, a hidden size that is no power of two, a vocabulary
        # of odd size, tokens without the few very frequent ones of text.
        _embed("embed_grad_ragged", "embed_grad", 83, 13, 1000, 50021, ragged=True, text=False, table="f32"),
        # A long batch of answers on top of the tied layer's gradient: frequent tokens have
        # thousands of steps.
        _embed("embed_grad_long", "embed_grad", 4096, 16, 2048, 131072, tied=True),
        # The recurrent core of a small agent, 256 units: nothing but latency.
        _updates("update_core", "256x1024*1", "f32"),
        # All matrices of a small convolutional agent with that core, filters as rows.
        _updates("update_agent", "16x192*1,32x256*1,256x2592*1,1024x513*1,18x256*1", "f32"),
        # Odd sizes, down to a single row and a single column.
        _updates("update_odd", "1000x1000*1,999x83*2,83x1001*2,50x1*1,1x257*1", "bf16"),
        # The matrices of a policy of hidden size 1024, four layers, mixed precision.
        _updates("update_policy", "1024x1024*16,4096x1024*4,1024x4096*4", "bf16"),
        # Those of one layer of hidden size 4096: the largest.
        _updates("update_large", "4096x4096*4,16384x4096*1,4096x16384*1", "bf16"),
    ]


def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "orthogonalize", "orthogonalize"])
    if op == "orthogonalize":
        dtype = rng.choice(["f32", "bf16"])
        left = MOST_WIDE_PRODUCTS if dtype == "f32" else MOST_PRODUCTS
        parts = []
        for _ in range(rng.randint(1, 4)):
            m, n = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
            count = min(_log_int(rng, 1, 16), int(left / max(1.0, _products(m, n))))
            if count > 0:
                parts.append(f"{m}x{n}*{count}")
                left -= count * _products(m, n)
        return _updates(None, ",".join(parts or ["64x64*1"]), dtype)
    H = 8 * _log_int(rng, 8, 512)
    V = _log_int(rng, 2000, min(131072, MOST_TABLE // H))
    N = _log_int(rng, 1, min(65536, (MOST_EMBED if op == "embed" else MOST_EMBED_GRAD) // H))
    B = _log_int(rng, 1, min(64, N))
    return _embed(None, op, max(1, N // B), B, H, V, scale=rng.choice([1.0, round(math.sqrt(H), 3)]), ragged=rng.random() < 0.4,
                  text=rng.random() < 0.6, table=rng.choice(["f32", "bf16"]), steps=rng.choice(["f32", "bf16"]),
                  tied=op == "embed_grad" and rng.random() < 0.5)


def _products(m, n):
    """Operations of one matrix: the symmetric products by their halves."""
    r, c = min(m, n), max(m, n)
    return STEPS * (3.0 * r * r * c + 1.0 * r * r * r)


def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        size, count = part.split("*")
        m, n = size.split("x")
        out += [(int(m), int(n))] * int(count)
    return out


def _lengths(case):
    """The lanes' lengths: from about half of T to T, the same for each seed but for their order."""
    T, B = case["T"], case["B"]
    if not case["ragged"]:
        return [T] * B
    return [T - (b * 7919 + 3) % (T // 2 + 1) for b in range(B)]


def _kw(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(generator=g, device="cuda", dtype=torch.float32)


def _random(shape, dtype, deviation, kw):
    """A large normal tensor, made in pieces."""
    out = torch.empty(shape, device="cuda", dtype=dtype)
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        m = min(1 << 26, flat.numel() - at)
        flat[at:at + m] = (torch.randn(m, **kw) * deviation).to(dtype)
    return out


def _tokens(case, kw):
    """Tokens of text: the k-th most frequent about 1/k as frequent as the first."""
    T, B, V = case["T"], case["B"], case["V"]
    u = torch.rand((T, B), **kw).double()
    t = torch.exp(u * math.log(V + 1.0)) - 1.0 if case["text"] else u * V
    t = t.long().clamp(max=V - 1)
    lengths = torch.tensor(_lengths(case), device="cuda")[torch.randperm(B, generator=kw["generator"], device="cuda")]
    behind = torch.arange(T, device="cuda").unsqueeze(1) >= lengths.unsqueeze(0)
    return torch.where(behind, -1, t).to(torch.int32)


def _inputs(case, seed):
    kw = _kw(seed)
    if case["op"] == "orthogonalize":
        # Gradients of layers: a few strong directions above a floor of noise.
        x = []
        for m, n in _shapes(case):
            r = max(1, min(m, n) // 16)
            g = torch.randn((m, r), **kw) @ torch.randn((r, n), **kw) / math.sqrt(r)
            x.append((1e-3 * (g + 0.3 * torch.randn((m, n), **kw))).to(DTYPE[case["dtype"]]))
        return dict(matrices=x)
    T, B, H, V = case["T"], case["B"], case["H"], case["V"]
    tokens = _tokens(case, kw)
    if case["op"] == "embed":
        return dict(vocab_weight=_random((V, H), DTYPE[case["table"]], 1.0 / math.sqrt(H), kw), tokens=tokens)
    x = dict(d_embedded=_random((T, B, H), DTYPE[case["steps"]], 1e-3, kw), tokens=tokens)
    if case["tied"]:
        x["d_weight"] = _random((V, H), DTYPE[case["table"]], 1e-3, kw)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    kept = {}
    if own:  # what a program keeps beside its inputs
        import paper_1802_01561_amd as vt

        if case["op"] == "orthogonalize":
            kept["workspace"] = vt.OrthogonalWorkspace(x["matrices"])
        elif case["op"] == "embed_grad":
            kept["workspace"] = vt.EmbedWorkspace(case["T"], case["B"], case["V"], case["H"])
    return case, x, kept


def run(state):
    case, x, kept = state
    if not own:
        return _PLAIN[case["op"]](case, x)
    import paper_1802_01561_amd as vt

    if case["op"] == "embed":
        return vt.vtrace_vocab_embed(x["vocab_weight"], x["tokens"], case["scale"], out_dtype=DTYPE[case["steps"]])
    if case["op"] == "embed_grad":
        return vt.vtrace_vocab_embed_grad(x["d_embedded"], x["tokens"], case["V"], case["scale"],
                                          grad_dtype=DTYPE[case["table"]], accumulate_into=x.get("d_weight"), **kept)
    return vt.vtrace_orthogonalize(x["matrices"], **kept)


def _plain_embed(case, x):
    rows = x["vocab_weight"][x["tokens"].clamp(min=0).long()].float() * case["scale"]
    return torch.where(x["tokens"].unsqueeze(-1) >= 0, rows, 0.0).to(DTYPE[case["steps"]])


def _plain_embed_grad(case, x):
    V, H = case["V"], case["H"]
    tokens = x["tokens"].reshape(-1).long()
    keep = tokens >= 0
    rows = torch.where(keep.unsqueeze(-1), x["d_embedded"].reshape(-1, H).float() * case["scale"], 0.0)
    total = torch.zeros((V, H), device="cuda").index_add_(0, tokens.clamp(min=0), rows)
    if not case["tied"]:
        return total.to(DTYPE[case["table"]])
    return x["d_weight"].copy_(x["d_weight"].float() + total)


def _plain_orthogonalize(case, x):
    """The products of float32 updates in 64 bits: small singular values grow by 3.44 a step, and
    what 32 bits lose beside the largest ones with them."""
    a, b, c = COEFFICIENTS
    wide = torch.float64 if case["dtype"] == "f32" else torch.float32
    out = []
    for g in x["matrices"]:
        u = g.to(wide)
        u = u / torch.linalg.vector_norm(u).clamp(min=EPSILON)
        tall = u.shape[0] > u.shape[1]
        u = u.t().contiguous() if tall else u
        for _ in range(STEPS):
            gram = u @ u.t()
            u = a * u + (b * gram + c * (gram @ gram)) @ u
        out.append((u.t() if tall else u).to(g.dtype).contiguous())
    return out


_PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "orthogonalize": _plain_orthogonalize}


def _distinct(case, n):
    """How many different tokens n steps have, on average."""
    V = case["V"]
    k = torch.arange(V, dtype=torch.float64)
    p = (torch.log(k + 2.0) - torch.log(k + 1.0)) / math.log(V + 1.0) if case["text"] else torch.full((V,), 1.0 / V, dtype=torch.float64)
    return float((1.0 - torch.exp(n * torch.log1p(-p))).sum())


def work(case):
    """Each input read once and each output written once: of the table the rows that the steps
    have, of its gradient those too where it is added to, else all of them.  Updates: the
    products, half of each symmetric one."""
    if case["op"] == "orthogonalize":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": sum(2 * size * m * n for m, n in _shapes(case)), "flops": sum(_products(m, n) for m, n in _shapes(case))}
    T, B, H, V = case["T"], case["B"], case["H"], case["V"]
    n = sum(_lengths(case))
    rows = _distinct(case, n) * H
    table, steps = (4 if case[k] == "f32" else 2 for k in ("table", "steps"))
    if case["op"] == "embed":
        return {"bytes": table * rows + steps * T * B * H + 4 * T * B, "flops": n * H if case["scale"] != 1.0 else 0}
    return {"bytes": table * (2 * rows if case["tied"] else V * H) + steps * n * H + 4 * T * B, "flops": 2 * n * H}


def _exact_embed(case, x):
    T, B, H = case["T"], case["B"], case["H"]
    out = torch.zeros((T * B, H), dtype=torch.float64, device="cuda")
    at = torch.nonzero(x["tokens"].reshape(-1) >= 0).squeeze(-1)
    out[at] = torch.index_select(x["vocab_weight"], 0, x["tokens"].reshape(-1)[at]).double() * float(torch.tensor(case["scale"]))
    return out.view(T, B, H)


def _exact_embed_grad(case, x):
    """Steps in the order of their tokens: a token's sum is a difference of running sums."""
    V, H = case["V"], case["H"]
    tokens = x["tokens"].reshape(-1).long()
    order = torch.argsort(tokens, stable=True)
    order = order[int((tokens < 0).sum()):]
    total = torch.zeros((V, H), dtype=torch.float64, device="cuda")
    if len(order):
        present, count = torch.unique_consecutive(tokens[order], return_counts=True)
        end = torch.cumsum(count, 0)
        for h in range(0, H, 512):
            running = torch.cumsum(x["d_embedded"].view(-1, H)[:, h:h + 512][order].double(), 0)
            running = torch.cat([torch.zeros_like(running[:1]), running])
            total[present, h:h + 512] = running[end] - running[end - count]
            del running
    total *= float(torch.tensor(case["scale"]))
    return total + x["d_weight"].double() if case["tied"] else total


def _exact_orthogonalize(case, x):
    """The polynomial s -> a s + b s^3 + c s^5 of the singular values, in the smaller of the two
    products' terms: X p(X'X) where X is tall, p(XX') X where it is wide."""
    a, b, c = COEFFICIENTS
    out = []
    for g in x["matrices"]:
        y = g.double()
        y = y / torch.sqrt((y * y).sum()).clamp(min=EPSILON)
        eye = torch.eye(min(y.shape), dtype=torch.float64, device="cuda")
        for _ in range(STEPS):
            if y.shape[0] > y.shape[1]:
                s = y.t().contiguous() @ y
                y = y @ (a * eye + s @ (b * eye + c * s))
            else:
                s = y @ y.t().contiguous()
                y = (a * eye + s @ (b * eye + c * s)) @ y
        out.append(y)
    return out


def exact(case, seed):
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "orthogonalize": _exact_orthogonalize}[case["op"]](case, _inputs(case, seed))
