"""The operators of a pipeline's two ends and of its residual stream, as they are measured.

The first stage looks token embeddings up and returns their gradient; the last one
turns the stream into log probabilities of the tokens that follow, and its gradient
starts there; every stage may drop elements of a branch before it joins the stream.
Kinds of case:

  "embed"       rows of the embedding by token id, times a scale; ids outside the
                vocabulary are padding and give rows of zeros
  "embed-back"  the embedding's gradient: the sum of the rows of dy of each token,
                written over the whole buffer or added to it (``accumulate``)
  "dropout"     residual + dropout(x), the mask drawn from a counter-based generator
                and not stored; or, with ``back``, the branch's gradient
  "logprobs"    from logits: log probability of given ids, the distribution's
                entropy, its ``top`` most likely ids; with ``train`` the gradient of
                the logits for gradients of the first two
  "head"        the same from the stream and the head's weights; with ``train`` the
                gradients of both

Widths and vocabularies are those of the repository's parameter sets (768 x 50257,
2048 x 128256, 4096 x 32000) and of its odd-sized tests, token counts generic.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LARGEST = 8192 * 4096 * 32000   # tokens x dim x vocabulary of the largest head
ELEMENTS = 8192 * 32000         # logits
STREAM = 8192 * 8192            # elements of a stream
TABLE = 32000 * 4096            # elements of an embedding
M32 = 0xFFFFFFFF


def listed():
    return [
        # one token of a 7B set: latency of a single launch
        dict(name="embed-1-token", kind="embed", tokens=1, vocab=32000, dim=4096, dtype="bf16",
             scale=1.0),
        # a microbatch of the 7B set
        dict(name="embed-7b", kind="embed", tokens=8192, vocab=32000, dim=4096, dtype="bf16",
             scale=64.0),
        # its gradient, written over the whole buffer
        dict(name="embed-7b-back", kind="embed-back", tokens=8192, vocab=32000, dim=4096,
             dtype="bf16", scale=64.0, accumulate=False),
        # odd sizes, added to what a tied head has left in an fp32 buffer
        dict(name="embed-odd-back-add", kind="embed-back", tokens=5003, vocab=50257, dim=777,
             dtype="f32", scale=1.0, accumulate=True),
        # a small fp32 branch with rows that end inside a draw
        dict(name="dropout-odd-f32", kind="dropout", rows=517, cols=777, dtype="f32", p=0.3,
             back=False),
        # a microbatch's branch joining the stream of a 7B layer
        dict(name="dropout-7b", kind="dropout", rows=8192, cols=4096, dtype="bf16", p=0.1,
             back=False),
        # one sequence's next token among the 1B set's vocabulary, with alternatives
        dict(name="logprobs-1-row-top", kind="logprobs", rows=1, vocab=128256, dtype="f32",
             scale=1.25, top=8, train=False),
        # GPT-2's odd vocabulary in bf16, loss and gradient
        dict(name="logprobs-gpt2-step", kind="logprobs", rows=4096, vocab=50257, dtype="bf16",
             scale=1.0, top=0, train=True),
        # scoring a batch with alternatives from fp32 logits
        dict(name="logprobs-score", kind="logprobs", rows=1000, vocab=32000, dtype="f32", scale=1.0,
             top=5, train=False),
        # one token through the 1B set's head: the weights' bytes count
        dict(name="head-1b-1-token", kind="head", tokens=1, dim=2048, vocab=128256, scale=1.0,
             top=8, train=False),
        # a short ragged batch through GPT-2's tied head
        dict(name="head-gpt2-step", kind="head", tokens=1001, dim=768, vocab=50257, scale=1.0,
             top=0, train=True),
        # the largest: a microbatch through the 7B set's head
        dict(name="head-7b-step", kind="head", tokens=8192, dim=4096, vocab=32000, scale=1.0,
             top=0, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed-back", "embed-back", "dropout", "logprobs", "logprobs",
                       "head", "head", "head"])
    if kind in ("embed", "embed-back"):
        while True:
            tokens, vocab, dim = _log(rng, 1, 65536), _log(rng, 50, 128256), _log(rng, 8, 8192)
            if rng.random() < 0.5:
                dim = -(-dim // 8) * 8
            if tokens * dim <= STREAM and vocab * dim <= TABLE:
                break
        c = dict(kind=kind, tokens=tokens, vocab=vocab, dim=dim, dtype=rng.choice(["bf16", "f32"]),
                 scale=rng.choice([1.0, math.sqrt(dim)]))
        return c if kind == "embed" else dict(c, accumulate=rng.random() < 0.5)
    if kind == "dropout":
        while True:
            rows, cols = _log(rng, 1, 16384), _log(rng, 8, 16384)
            if rows * cols <= STREAM:
                break
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["bf16", "f32"]),
                    p=rng.choice([0.05, 0.1, 0.2, 0.5]), back=rng.random() < 0.5)
    scale = rng.choice([1.0, 1.0, 0.7])
    if kind == "logprobs":
        while True:
            rows, vocab = _log(rng, 1, 8192), _log(rng, 40, 128256)
            if rows * vocab <= ELEMENTS:
                break
        train = rng.random() < 0.5
        return dict(kind=kind, rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "f32"]),
                    scale=scale, top=0 if train else rng.choice([0, 1, 5, 20]), train=train)
    while True:
        tokens, dim, vocab = _log(rng, 1, 8192), 8 * _log(rng, 8, 512), _log(rng, 300, 128256)
        if tokens * dim * vocab <= LARGEST and vocab * dim <= 2048 * 128256:
            break
    train = tokens > 8 and rng.random() < 0.7
    return dict(kind=kind, tokens=tokens, dim=dim, vocab=vocab, scale=scale,
                top=8 if tokens <= 16 and not train else 0, train=train)


# ---------------------------------------------------------------- inputs ----

def _randn(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def _ids(gen, n, vocab):
    """Token ids whose frequencies fall as their rank's reciprocal, a few of many padding."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp(max=vocab - 1)
    ids = ids * 7919 % vocab if math.gcd(7919, vocab) == 1 else ids   # common ones anywhere
    padding = torch.rand(n, generator=gen, device="cuda") < (0.03 if n > 1 else 0.0)
    return torch.where(padding, -1, ids)


def _loss_gradients(gen, s, n):
    """Of the log probabilities (advantages) and of the entropy (a bonus)."""
    s["dlogp"] = torch.randn(n, generator=gen, device="cuda") / n
    s["dentropy"] = torch.rand(n, generator=gen, device="cuda") * (0.01 / n)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    kind = case["kind"]
    if kind in ("embed", "embed-back"):
        t, v, d, dt = case["tokens"], case["vocab"], case["dim"], DT[case["dtype"]]
        s["ids"] = _ids(gen, t, v)
        if kind == "embed":
            s["table"] = _randn(gen, v, d, scale=0.02, dtype=dt)
        else:
            s["dy"] = _randn(gen, t, d, scale=1e-3, dtype=dt)
            s["dtable"] = _randn(gen, v, d, scale=1e-3, dtype=dt)   # the gradient buffer
        return s
    if kind == "dropout":
        n, d, dt = case["rows"], case["cols"], DT[case["dtype"]]
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=torch.Generator().manual_seed(seed)))
        s["site"] = seed % 97
        s["x"] = _randn(gen, n, d, dtype=dt)
        s["residual"] = None if case["back"] else _randn(gen, n, d, scale=3.0, dtype=dt)
        return s
    if kind == "logprobs":
        n, v, dt = case["rows"], case["vocab"], DT[case["dtype"]]
        z = torch.randn(n, v, generator=gen, device="cuda").mul_(2.0)
        real = v - v // 200 if v >= 1000 else v                       # a padded vocabulary
        s["ids"] = _ids(gen, n, real)
        hit = torch.rand(n, generator=gen, device="cuda") < 0.6   # tokens the model expects
        z[torch.arange(n, device="cuda"), s["ids"].clamp(min=0)] += torch.where(hit, 9.0, 0.0)
        z[:, real:] = -math.inf
        s["logits"] = z.to(dt)
        if case["train"]:
            _loss_gradients(gen, s, n)
        return s
    t, d, v = case["tokens"], case["dim"], case["vocab"]
    s["x"] = _randn(gen, t, d)
    s["w"] = _randn(gen, v, d, scale=2.0 * d ** -0.5)
    s["ids"] = _ids(gen, t, v)
    if case["train"]:
        _loss_gradients(gen, s, t)
        s["dw"] = torch.zeros_like(s["w"])   # the gradient buffer
    return s


# ------------------------------------------------------------ plain forms ----

def _mulhi(a, b):
    """High and low words of 32-bit products, as 64-bit integers."""
    low = a * (b & 0xFFFF)
    high = a * (b >> 16) + (low >> 16)
    return high >> 16, (high << 16 | low & 0xFFFF) & M32


def _halves(rows, cols, seed, site):
    """16 random bits for each element: Philox4x32 in ten rounds on the counter (block of
    eight columns, row, 0, site) under the seed; element 2 j + h of a block has half h of
    word j."""
    blocks = -(-cols // 8)
    c0 = torch.arange(blocks, device="cuda").expand(rows, blocks)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)
    c2, c3 = torch.zeros_like(c0), torch.full_like(c0, site)
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        h0, l0 = _mulhi(c0, 0xD2511F53)
        h1, l1 = _mulhi(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    w = torch.stack((c0, c1, c2, c3), -1)
    return torch.stack((w & 0xFFFF, w >> 16), -1).view(rows, -1)[:, :cols]


def _plain_embed(s):
    t, ids = s["table"], s["ids"]
    known = (ids >= 0) & (ids < t.shape[0])
    rows = t[ids.clamp(0, t.shape[0] - 1)].float() * s["case"]["scale"]
    return dict(out=torch.where(known[:, None], rows, 0.0).to(t.dtype))


def _plain_embed_back(s):
    d, ids = s["dtable"], s["ids"]
    known = (ids >= 0) & (ids < d.shape[0])
    rows = torch.where(known[:, None], s["dy"].float(), 0.0)
    total = torch.zeros(d.shape, device="cuda").index_add_(0, ids.clamp(0, d.shape[0] - 1), rows)
    total = total * s["case"]["scale"]
    d.copy_(total + d.float() if s["case"]["accumulate"] else total)
    return dict(dtable=d)


def _plain_dropout(s):
    x = s["x"]
    cut = math.floor(s["case"]["p"] * 65536 + 0.5)
    kept = _halves(*x.shape, s["seed"], s["site"]) >= cut
    y = torch.where(kept, x.float() * (65536 / (65536 - cut)), 0.0)
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return dict(y=y.to(x.dtype))


def _distribution(z, ids):
    """What the operators give of rows of scaled logits, and what their gradients need."""
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    logs = d - torch.log(total)
    p = e / total
    known = (ids >= 0) & (ids < z.shape[1])
    at = ids.clamp(0, z.shape[1] - 1)[:, None]
    logp = torch.where(known, logs.gather(1, at)[:, 0], 0.0)
    entropy = -torch.where(p > 0, p * logs, 0.0).sum(1)
    return logs, p, known, at, logp, entropy


def _top(z, logs, k):
    """The k largest, ties to the lowest id."""
    ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    return dict(top_logp=logs.gather(1, ids), top_ids=ids)


def _gradient(s, logs, p, known, at, entropy):
    """Of the scaled logits."""
    a = torch.where(known, s["dlogp"], 0.0)[:, None]
    b = s["dentropy"][:, None]
    g = -p * (a + b * torch.where(p > 0, logs + entropy[:, None], 0.0))
    return g.scatter_add_(1, at, a)


def _plain_logprobs(s):
    case = s["case"]
    z = s["logits"].float() * case["scale"]
    logs, p, known, at, logp, entropy = _distribution(z, s["ids"])
    out = dict(logp=logp, entropy=entropy)
    if case["top"]:
        out.update(_top(z, logs, case["top"]))
    if case["train"]:
        g = _gradient(s, logs, p, known, at, entropy) * case["scale"]
        out["dlogits"] = g.to(s["logits"].dtype)
    return out


def _plain_head(s):
    case = s["case"]
    x, w = s["x"].float(), s["w"].float()
    z = (x @ w.t()) * case["scale"]
    logs, p, known, at, logp, entropy = _distribution(z, s["ids"])
    out = dict(logp=logp, entropy=entropy)
    if case["top"]:
        out.update(_top(z, logs, case["top"]))
    if case["train"]:
        g = _gradient(s, logs, p, known, at, entropy) * case["scale"]
        s["dw"].copy_(g.t() @ x)
        out.update(dx=(g @ w).bfloat16(), dw=s["dw"])
    return out


# ------------------------------------------------------- the framework's ----

def _own_embed(s):
    from paper_2606_30634_gb300 import ends
    return dict(out=ends.embed(s["ids"], s["table"], scale=s["case"]["scale"]))


def _own_embed_back(s):
    from paper_2606_30634_gb300 import ends
    c = s["case"]
    return dict(dtable=ends.embed_backward(s["dy"], s["ids"], s["dtable"], scale=c["scale"],
                                           accumulate=c["accumulate"]))


def _own_dropout(s):
    from paper_2606_30634_gb300 import ends
    if s["case"]["back"]:
        return dict(y=ends.dropout_backward(s["x"], s["case"]["p"], s["seed"], site=s["site"]))
    return dict(y=ends.dropout_add(s["x"], s["residual"], s["case"]["p"], s["seed"], site=s["site"]))


def _own_out(o, case):
    out = dict(logp=o.logp, entropy=o.entropy)
    if case["top"]:
        out.update(top_logp=o.top_logp, top_ids=o.top_ids)
    return out


def _own_logprobs(s):
    from paper_2606_30634_gb300 import ends
    case = s["case"]
    o = ends.token_logprobs(s["logits"], s["ids"], scale=case["scale"], top=case["top"])
    out = _own_out(o, case)
    if case["train"]:
        out["dlogits"] = ends.token_logprobs_backward(s["dlogp"], s["logits"], s["ids"], o,
                                                      dentropy=s["dentropy"])
    return out


def _own_head(s):
    from paper_2606_30634_gb300 import ends
    case = s["case"]
    o, kept = ends.head_logprobs(s["x"], s["w"], s["ids"], scale=case["scale"], top=case["top"],
                                 keep=case["train"])
    out = _own_out(o, case)
    if case["train"]:
        dx = ends.head_logprobs_backward(s["dlogp"], kept, s["x"], s["w"], s["ids"], o, s["dw"],
                                         dentropy=s["dentropy"])
        out.update(dx=dx, dw=s["dw"])
    return out


PLAIN = {"embed": _plain_embed, "embed-back": _plain_embed_back, "dropout": _plain_dropout,
         "logprobs": _plain_logprobs, "head": _plain_head}
OWN = {"embed": _own_embed, "embed-back": _own_embed_back, "dropout": _own_dropout,
       "logprobs": _own_logprobs, "head": _own_head}


def run(s):
    return (OWN if own else PLAIN)[s["case"]["kind"]](s)


# ------------------------------------------------------------------ work ----

def work(case):
    kind = case["kind"]
    if kind == "head":
        t, d, v = case["tokens"], case["dim"], case["vocab"]
        flops, size = 2 * t * d * v, 2 * (t * d + v * d) + 16 * t + 12 * t * case["top"]
        if case["train"]:
            flops, size = 3 * flops, size + 2 * (t * d + v * d) + 8 * t
        return dict(bytes=size, flops=flops)
    b = 4 if case["dtype"] == "f32" else 2
    if kind in ("embed", "embed-back"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        # rows of the table that are met: each id x with probability log((x + 2) / (x + 1)) / log(v + 1)
        x = np.arange(v)
        p = 0.97 * np.log((x + 2) / (x + 1)) / np.log(v + 1)
        met = float((1 - (1 - p) ** t).sum()) if t > 1 else 1.0
        if kind == "embed":
            return dict(bytes=int(met * d * b) + t * d * b + 8 * t, flops=t * d)
        size = 2 * met if case["accumulate"] else v
        return dict(bytes=t * d * b + 8 * t + int(size * d * b), flops=t * d)
    if kind == "dropout":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * b * (2 if case["back"] else 3), flops=2 * n)
    n = case["rows"] * case["vocab"]
    passes = 3 if case["train"] else 1   # logits read twice: the gradient needs the whole row's sum
    size = n * b * (2 if case["train"] else 1)
    return dict(bytes=size + case["rows"] * (16 + 12 * case["top"]), flops=4 * n * passes)


# ----------------------------------------------------------- in 64 bits ----

def _drawn_bits(rows, cols, seed, site):
    """The halves of _halves(), from the generator's definition in numpy's 64-bit integers."""
    groups = -(-cols // 8)
    u = np.uint64
    ctr = np.zeros((4, rows * groups), u)
    ctr[0], ctr[1], ctr[3] = np.tile(np.arange(groups), rows), np.repeat(np.arange(rows), groups), site
    for i in range(10):
        keys = [u(((seed >> (32 * j)) + i * w) % 2 ** 32) for j, w in enumerate((0x9E3779B9, 0xBB67AE85))]
        first, second = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = np.stack([(second >> u(32)) ^ ctr[1] ^ keys[0], second & u(M32),
                        (first >> u(32)) ^ ctr[3] ^ keys[1], first & u(M32)])
    words = np.ascontiguousarray(ctr.T.astype("<u4"))
    return torch.from_numpy(words.view("<u2").astype(np.int32).reshape(rows, -1)[:, :cols].copy()).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        ids = s["ids"]
        out = s["table"].double().index_select(0, ids.clamp(min=0)).mul_(case["scale"])
        out[ids < 0] = 0
        return dict(out=out)
    if kind == "embed-back":
        real = s["ids"] >= 0
        dt = s["dtable"].double() if case["accumulate"] else torch.zeros(s["dtable"].shape, device="cuda",
                                                                         dtype=torch.float64)
        dt.index_put_((s["ids"][real],), s["dy"][real].double() * case["scale"], accumulate=True)
        return dict(dtable=dt)
    if kind == "dropout":
        cut = round(case["p"] * 65536)
        drop = _drawn_bits(case["rows"], case["cols"], s["seed"], s["site"]) < cut
        y = (s["x"].double() / (1 - cut / 65536)).masked_fill(drop, 0.0)
        return dict(y=y if case["back"] else y + s["residual"].double())
    ids = s["ids"]
    if kind == "head":
        if 6.0 * case["tokens"] * case["dim"] * case["vocab"] > 1e13:
            return None
        x, w = s["x"].double(), s["w"].double()
        z = torch.mm(x, w.T).mul_(case["scale"])
    else:
        z = s["logits"].double() * case["scale"]
    logs = z - torch.logsumexp(z, 1)[:, None]
    p = logs.exp()
    own_logs = torch.where(p == 0, 0.0, logs)
    entropy = -torch.einsum("ij,ij->i", p, own_logs)
    r = torch.arange(len(ids), device="cuda")
    real = ids >= 0
    out = dict(logp=torch.where(real, logs[r, ids.clamp(min=0)], 0.0), entropy=entropy)
    if case["top"]:
        out["top_logp"], out["top_ids"] = torch.topk(logs, case["top"]).values, None
    if case["train"]:
        a, b = s["dlogp"].double() * real, s["dentropy"].double()
        g = p * (own_logs + entropy[:, None]) * -b[:, None] - p * a[:, None]
        g[r[real], ids[real]] += a[real]
        g *= case["scale"]
        if kind == "logprobs":
            out["dlogits"] = g
        else:
            out["dx"], out["dw"] = torch.mm(g, w), torch.mm(g.T, x)
    return out
