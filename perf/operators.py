"""The operators around the optimizer step whose time is measured, on work that a
training run has them do:

  ortho   a list of matrices made orthogonal by Newton-Schulz products
  muon    the Muon step of a model's matrices: momentum, orthogonalized update,
          decoupled weight decay
  xent    softmax cross entropy of hidden states against a vocabulary table, with
          the gradients of both, without keeping the logits
  embed   rows of a token table, scaled
  grad    the token table's gradient from the rows' gradients

A case names the operator, its sizes and its types. ``run`` computes it in plain
torch operations in fp32, or, where ``own`` is true, with the package's kernels.
Matrices of one shape lie in one stack, as trainers lay out equal layers, and
their updates come back as these stacks.
"""

import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)
NS_STEPS = 5
NS_EPS = 1e-7
MUON = dict(lr=1e-3, momentum=0.95, weight_decay=0.1)
IGNORE = -100


def _case(name, op, **fields):
    case = dict(name=name, op=op)
    case.update(fields)
    return case


def listed():
    return [
        # The smallest lists: a probe's or an adapter's four matrices, where launches count.
        _case("ortho-tiny", "ortho", model="tiny", src="bf16", dst="bf16"),
        # Matrices of odd sizes from 1 to 2048 (probes, heads, a 1000-class classifier), in
        # and out in fp32.
        _case("ortho-ragged", "ortho", model="ragged", matrices=6, largest=2048, src="f32",
              dst="f32"),
        # One eighth of the 1.5-billion-parameter decoder's layers, as one rank of eight has them.
        _case("ortho-gpt", "ortho", model="gpt", hidden=1600, layers=6, src="bf16", dst="bf16"),
        # The Muon step of the tiny set, where launches count.
        _case("muon-tiny", "muon", model="tiny", grad="f32", scale="rms", nesterov=True),
        # The convolutions of ResNet-50 as matrices: many small ones, of 20 shapes, some odd.
        _case("muon-resnet50", "muon", model="resnet50", grad="f32", scale="spectral",
              nesterov=True),
        # Every matrix of the encoder layers of BERT-Large, bf16 gradients.
        _case("muon-bert-large", "muon", model="bert", hidden=1024, layers=24, grad="bf16",
              scale="rms", nesterov=True),
        # A few tokens against a small vocabulary: latency.
        _case("xent-small", "xent", tokens=7, dim=256, vocab=2003, ignored=0.0),
        # Masked-token pre-training of BERT-Large: the masked positions of 16 sequences of 512.
        _case("xent-bert-large", "xent", tokens=1229, dim=1024, vocab=30522, ignored=0.03),
        # The 1.5-billion-parameter decoder's loss over eight sequences of 1024.
        _case("xent-gpt", "xent", tokens=8192, dim=1600, vocab=50257, ignored=0.0),
        # One decoding step of 64 sequences: single tokens.
        _case("embed-decode", "embed", tokens=64, dim=1600, vocab=50257, table="bf16",
              out="bf16"),
        # BERT-Large's token table from 16 sequences of 512, a fresh fp32 gradient.
        _case("grad-bert-large", "grad", tokens=8192, dim=1024, vocab=30522, rows="bf16",
              out="f32", add=False),
        # The decoder's tied table: added to the gradient that the loss left there.
        _case("grad-gpt-tied", "grad", tokens=8191, dim=1600, vocab=50257, rows="bf16",
              out="bf16", add=True),
    ]


def _log(rng, low, high):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return n + (n == 3072)  # BERT-Base's feed-forward width, which no case here has


def draw(rng):
    op = rng.choice(["ortho", "muon", "xent", "xent", "embed", "grad"])
    if op in ("ortho", "muon"):
        model = rng.choice(["ragged", "ragged", "bert", "gpt"])
        case = dict(op=op, model=model)
        if model == "ragged":
            case.update(matrices=_log(rng, 1, 12), largest=_log(rng, 40, 2500))
        else:
            hidden = 8 * _log(rng, 8, 160)  # but BERT-Base's 768 (see _log)
            case.update(hidden=hidden + 8 if hidden == 768 else hidden, layers=_log(rng, 1, 8))
        if op == "ortho":
            case.update(src=rng.choice(["f32", "bf16"]), dst=rng.choice(["bf16", "bf16", "f32"]))
        else:
            case.update(grad=rng.choice(["f32", "bf16"]), scale=rng.choice(["rms", "spectral"]),
                        nesterov=rng.random() < 0.7)
        return case
    case = dict(op=op, tokens=_log(rng, 1, 8192), dim=8 * _log(rng, 8, 200),
                vocab=_log(rng, 500, 50257))
    if op == "xent":
        case.update(ignored=rng.choice([0.0, 0.1, 0.85]))
    elif op == "embed":
        case.update(table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]))
    else:
        case.update(rows=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]),
                    add=rng.random() < 0.5)
    return case


def _shapes(case):
    """[(rows, cols, how many)]: the case's matrices, stacked by shape."""
    model = case["model"]
    if model == "tiny":
        return [(256, 256, 1), (256, 1024, 1), (1024, 256, 1), (64, 256, 1)]
    if model == "ragged":
        n, top = case["matrices"], case["largest"]
        found = []
        for i in range(n):
            long = max(1, int(top ** ((i + 1) / n)))
            short = max(1, int(long * (0.37, 0.91, 1.0)[i % 3]))
            found.append((long, short, 1) if i % 2 else (short, long, 1))
        return found
    if model == "resnet50":
        count = {(64, 147): 1, (1000, 2048): 1}
        c_in = 64
        for w, n in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(n):
                made = [(w, c_in), (w, 9 * w), (4 * w, w)] + ([(4 * w, c_in)] if b == 0 else [])
                for s in made:
                    count[s] = count.get(s, 0) + 1
                c_in = 4 * w
        return [(r, c, k) for (r, c), k in count.items()]
    h, layers = case["hidden"], case["layers"]
    return [(h, h, 4 * layers), (h, 4 * h, layers), (4 * h, h, layers)]


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(6151 * int(seed) + 3)


def _tokens(case, gen):
    """Token ids with the frequencies of text: the k-th most frequent id is 1/k as
    frequent as the first, and ids are not in the order of their frequency."""
    n, v = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(v + 1.0)) - 1.0).long().clamp_(0, v - 1)
    return torch.randperm(v, generator=gen, device="cuda")[rank]


def prepare(case, seed):
    gen = _gen(seed)

    def normal(*shape, sigma=1.0, dtype="f32"):
        t = torch.randn(*shape, generator=gen, device="cuda").mul_(sigma)
        return t.to(_dtype(dtype))

    s = dict(case=case)
    op = case["op"]
    if op == "ortho":
        s["g"] = [normal(k, r, c, sigma=1e-3, dtype=case["src"]) for r, c, k in _shapes(case)]
        s["out"] = [torch.empty(g.shape, dtype=_dtype(case["dst"]), device="cuda")
                    for g in s["g"]]
    elif op == "muon":
        shapes = _shapes(case)
        s["x"] = [normal(k, r, c, sigma=0.02) for r, c, k in shapes]
        s["g"] = [normal(k, r, c, sigma=1e-3, dtype=case["grad"]) for r, c, k in shapes]
        s["m"] = [normal(k, r, c, sigma=1.6e-4) for r, c, k in shapes]
    else:
        n, d, v = case["tokens"], case["dim"], case["vocab"]
        s["tokens"] = _tokens(case, gen)
        if op == "xent":
            # hidden states after a layer norm, a table as it is initialised: logits of
            # standard deviation 0.02 sqrt(d), and some positions that carry no target
            s["hidden"] = normal(n, d, dtype="bf16")
            s["table"] = normal(v, d, sigma=0.02, dtype="bf16")
            none = torch.rand(n, generator=gen, device="cuda") < case["ignored"]
            s["tokens"].masked_fill_(none, IGNORE)
            s["grad_hidden"] = torch.empty_like(s["hidden"])
            s["grad_table"] = torch.empty_like(s["table"])
        elif op == "embed":
            s["table"] = normal(v, d, sigma=0.02, dtype=case["table"])
            s["scale"] = math.sqrt(d)
        else:
            s["rows"] = normal(n, d, sigma=1e-3, dtype=case["rows"])
            s["grad"] = normal(v, d, sigma=1e-3, dtype=case["out"])
            s["scale"] = math.sqrt(d)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_1904_00962_amd import ops, optim
    s["ops"] = ops
    case = s["case"]
    flat = lambda stacks: [a for stack in stacks for a in stack.unbind(0)]  # noqa: E731
    if case["op"] == "ortho":
        s["plan"] = ops.Orthogonalizer(flat(s["g"]), flat(s["out"]), steps=NS_STEPS,
                                       coefficients=COEF, eps=NS_EPS)
    elif case["op"] == "muon":
        s["opt"] = optim.Muon(flat(s["x"]), flat(s["g"]), m=flat(s["m"]),
                              nesterov=case["nesterov"], scale=case["scale"], steps=NS_STEPS,
                              coefficients=COEF, eps=NS_EPS, **MUON)


def _newton_schulz(g):
    """A stack of matrices, [k, rows, cols] in fp32, made orthogonal."""
    tall = g.shape[1] > g.shape[2]
    x = g.mT if tall else g
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + NS_EPS)
    a, b, c = COEF
    for _ in range(NS_STEPS):
        gram = torch.bmm(x, x.mT)
        poly = b * gram + c * torch.bmm(gram, gram)
        x = a * x + torch.bmm(poly, x)
    return x.mT if tall else x


def _update_scale(case, rows, cols):
    if case["scale"] == "rms":
        return 0.2 * math.sqrt(max(rows, cols))
    return math.sqrt(max(1.0, rows / cols))


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "ortho":
        return dict(out=[_newton_schulz(g.float()).to(_dtype(case["dst"])) for g in s["g"]])
    if op == "muon":
        mu, lr = MUON["momentum"], MUON["lr"]
        for x, g, m in zip(s["x"], s["g"], s["m"]):
            gf = g.float()
            m.mul_(mu).add_(gf, alpha=1.0 - mu)
            u = m * mu + gf * (1.0 - mu) if case["nesterov"] else m
            o = _newton_schulz(u)
            x.mul_(1.0 - lr * MUON["weight_decay"])
            x.sub_(o, alpha=lr * _update_scale(case, x.shape[1], x.shape[2]))
        return dict(x=s["x"], m=s["m"])
    if op == "xent":
        h, w, t = s["hidden"].float(), s["table"].float(), s["tokens"]
        keep = t != IGNORE
        at = t.clamp(min=0)[:, None]
        logits = h @ w.T
        top = logits.max(dim=1, keepdim=True).values
        p = torch.exp(logits - top)
        total = p.sum(dim=1, keepdim=True)
        loss = (torch.log(total) + top - logits.gather(1, at))[:, 0] * keep
        count = keep.sum().clamp(min=1)
        p.div_(total)
        p.scatter_add_(1, at, torch.full_like(total, -1.0))
        p.mul_((keep / count)[:, None])
        return dict(mean=loss.sum() / count, loss=loss, grad_hidden=(p @ w).to(torch.bfloat16),
                    grad_table=(p.T @ h).to(torch.bfloat16))
    if op == "embed":
        return (s["table"][s["tokens"]].float() * s["scale"]).to(_dtype(case["out"]))
    sums = torch.zeros(s["grad"].shape, device="cuda")
    sums.index_add_(0, s["tokens"], s["rows"].float()).mul_(s["scale"])
    if case["add"]:
        sums.add_(s["grad"])
    s["grad"].copy_(sums)
    return s["grad"]


def run(s):
    if not own:
        return _run_plain(s)
    case, ops = s["case"], s["ops"]
    op = case["op"]
    if op == "ortho":
        s["plan"].run()
        return dict(out=s["out"])
    if op == "muon":
        s["opt"].step()
        return dict(x=s["x"], m=s["m"])
    if op == "xent":
        mean, loss, lse = ops.linear_cross_entropy(s["hidden"], s["table"], s["tokens"],
                                                   ignore_index=IGNORE)
        ops.linear_cross_entropy_grad(s["hidden"], s["table"], s["tokens"], lse,
                                      s["grad_hidden"], s["grad_table"], ignore_index=IGNORE)
        return dict(mean=mean, loss=loss, grad_hidden=s["grad_hidden"],
                    grad_table=s["grad_table"])
    if op == "embed":
        return ops.embedding(s["tokens"], s["table"], scale=s["scale"],
                             out_dtype=_dtype(case["out"]))
    ops.embedding_grad(s["tokens"], s["rows"], s["grad"], scale=s["scale"],
                       accumulate=case["add"])
    return s["grad"]


def work(case):
    """Flops of a Newton-Schulz step on a matrix of long side L and short side S: S x S
    products of the symmetric kind cost half, so L S^2 for the Gram matrix, S^3 for its
    square and 2 L S^2 for the product with the matrix. Cross entropy: 2 N D V for the
    logits and 4 N D V for the two gradients. Bytes: inputs once, outputs once; of a
    table, the rows that tokens can touch."""
    size = {"f32": 4, "bf16": 2}
    op = case["op"]
    if op in ("ortho", "muon"):
        flops = numel = 0
        for r, c, k in _shapes(case):
            long, short = max(r, c), min(r, c)
            flops += k * NS_STEPS * (3 * long * short ** 2 + short ** 3)
            numel += k * r * c
        per = size[case["src"]] + size[case["dst"]] if op == "ortho" else 16 + size[case["grad"]]
        return {"bytes": float(numel * per), "flops": float(flops)}
    n, d, v = case["tokens"], case["dim"], case["vocab"]
    if op == "xent":
        return {"bytes": float(2 * 2 * (n + v) * d + 12 * n), "flops": 6.0 * n * d * v}
    if op == "embed":
        touched = min(n, v)
        return {"bytes": float(touched * d * size[case["table"]] + n * d * size[case["out"]]
                               + 8 * n), "flops": float(n * d)}
    # distinct ids among n draws whose frequencies fall as 1 / rank
    total = math.log(v + 1.0)
    edges = [math.exp(total * i / 64) for i in range(65)]
    distinct = sum((b - a) * -math.expm1(-n * (total / 64) / total / (b - a))
                   for a, b in zip(edges, edges[1:]))
    written = distinct * d * 2 * size[case["out"]] if case["add"] else v * d * size[case["out"]]
    return {"bytes": float(n * d * size[case["rows"]] + written + 8 * n), "flops": float(n * d)}


def _exact_ns(g):
    """The definition in 64 bits: y <- (a I + b q + c q q) y with q = y y^T."""
    long_rows = g.shape[0] > g.shape[1]
    y = g.t().contiguous() if long_rows else g.clone()
    y /= torch.linalg.vector_norm(y) + NS_EPS
    for _ in range(NS_STEPS):
        q = y @ y.t()
        r = COEF[2] * (q @ q)
        r += COEF[1] * q
        r.diagonal().add_(COEF[0])
        y = r @ y
    return y.t() if long_rows else y


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "ortho":
        return dict(out=[torch.stack([_exact_ns(a.double()) for a in g]) for g in s["g"]])
    if op == "muon":
        mu, lr = MUON["momentum"], MUON["lr"]
        xs, ms = [], []
        for x, g, m in zip(s["x"], s["g"], s["m"]):
            m2 = torch.lerp(g.double(), m.double(), mu)
            x2 = torch.empty_like(m2)
            for i in range(len(x)):
                u = torch.lerp(g[i].double(), m2[i], mu) if case["nesterov"] else m2[i]
                x2[i] = (x[i].double() * (1.0 - lr * MUON["weight_decay"])
                         - lr * _update_scale(case, *u.shape) * _exact_ns(u))
            xs.append(x2)
            ms.append(m2)
        return dict(x=xs, m=ms)
    t = s["tokens"]
    if op == "xent":
        n = case["tokens"]
        w = s["table"].double()
        kept = max(1, int((t != IGNORE).sum()))
        loss = torch.zeros(n, dtype=torch.float64, device="cuda")
        gh = torch.zeros(n, case["dim"], dtype=torch.float64, device="cuda")
        gw = torch.zeros_like(w)
        for at in range(0, n, 1024):
            rows = (t[at:at + 1024] != IGNORE).nonzero()[:, 0] + at
            if len(rows) == 0:
                continue
            h = s["hidden"][rows].double()
            z = h @ w.T
            lse = torch.logsumexp(z, dim=1)
            loss[rows] = lse - z[torch.arange(len(rows), device="cuda"), t[rows]]
            z = torch.exp(z - lse[:, None])
            z[torch.arange(len(rows), device="cuda"), t[rows]] -= 1.0
            z /= kept
            gh[rows] = z @ w
            gw += z.T @ h
        return dict(mean=loss.sum() / kept, loss=loss, grad_hidden=gh, grad_table=gw)
    if op == "embed":
        return s["table"].double()[t] * s["scale"]
    order = torch.argsort(t)
    ids, counts = torch.unique_consecutive(t[order], return_counts=True)
    sums = torch.segment_reduce(s["rows"].double()[order].cpu(), "sum", lengths=counts.cpu(),
                                axis=0).cuda()
    out = s["grad"].double() if case["add"] else torch.zeros(s["grad"].shape,
                                                             dtype=torch.float64, device="cuda")
    out[ids] += sums * s["scale"]
    return out
