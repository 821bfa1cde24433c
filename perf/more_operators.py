"""The operators between a model's products and its optimizer step whose time is
measured, on work that a training or a serving run has them do:

  norm    a branch's output added to the residual stream, and the root-mean-square norm
          of the sum
  norm8   the same with the norm's result in 8 bits (e4m3), a scale for each row or for
          each group of its columns
  grad    the norm's gradients: of its input, joined by the gradient that reaches the
          stream from further up, and of its weight
  gnorm   the norms of all gradient tensors and of all of them together
  clip    the gradients scaled so that their common norm keeps a limit

A case names the operator, its sizes and its types. ``run`` computes it in plain torch
operations in fp32 (norms of gradients in fp64), or, where ``own`` is true, with the
package's kernels. The gradients of a model lie one after another in one buffer of each
type, as trainers lay out what they reduce between workers.
"""

import math

import torch

own = False

EPS = 1e-6
LARGEST_E4M3 = 448.0
LEAST_SCALE = 2.0 ** -126  # of a row or group whose values are all zero, or nearly
LIMIT = 1.0  # of the gradients' norm


def _case(name, op, **fields):
    case = dict(name=name, op=op)
    case.update(fields)
    return case


def listed():
    return [
        # One decoding step of 64 sequences: single tokens, where a launch counts.
        _case("norm-decode", "norm", tokens=64, dim=1600, x="bf16", stream="bf16", weight="bf16",
              out="bf16"),
        # The masked positions of 16 sequences before a head of odd width, all in fp32.
        _case("norm-odd", "norm", tokens=1229, dim=1001, x="f32", stream="none", weight="f32",
              out="f32"),
        # The 1.5-billion-parameter decoder over 32 sequences of 1024: bf16 branches on a
        # stream that is kept in fp32.
        _case("norm-gpt", "norm", tokens=32768, dim=1600, x="bf16", stream="f32", weight="f32",
              out="bf16"),
        # One token of one sequence, a scale for its row.
        _case("norm8-single", "norm8", tokens=1, dim=1600, stream="bf16", x="bf16", weight="bf16",
              group=0),
        # The decoder's products in 8 bits, scales for 128 columns, of which 1600 has 12.5.
        _case("norm8-gpt", "norm8", tokens=32768, dim=1600, x="bf16", stream="bf16",
              weight="bf16", group=128),
        # A few tokens of a probe of odd width.
        _case("grad-small", "grad", tokens=7, dim=250, x="f32", dy="f32", stream=False,
              weight="f32"),
        # BERT-Large's width over 16 sequences of 512.
        _case("grad-bert-large", "grad", tokens=8192, dim=1024, x="bf16", dy="bf16", stream=True,
              weight="f32"),
        # The decoder's stream in fp32 over 32 sequences of 1024.
        _case("grad-gpt", "grad", tokens=32768, dim=1600, x="f32", dy="bf16", stream=True,
              weight="f32"),
        # Tensors of 1 to 300,000 elements and both types, that begin anywhere.
        _case("gnorm-ragged", "gnorm", model="ragged", tensors=23, largest=300000, grad="mixed",
              norm="l2"),
        # The 391 tensors of BERT-Large, 335 million elements.
        _case("gnorm-bert-large", "gnorm", model="bert", hidden=1024, layers=24, grad="bf16",
              norm="l2"),
        # A step of the tiny set that stays below the limit: nothing is written.
        _case("clip-tiny", "clip", model="tiny", grad="f32", norm="l2", out="same", above=False),
        # The decoder's 1.5 billion fp32 sums of micro-batches, clipped to the bf16 gradients
        # that the step reads.
        _case("clip-gpt", "clip", model="gpt", hidden=1600, layers=48, grad="f32", norm="l2",
              out="bf16", above=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm8", "grad", "grad", "gnorm", "clip"])
    if op in ("norm", "norm8", "grad"):
        dim = _log(rng, 33, 8192)
        if rng.random() < 0.6:
            dim = max(8, dim // 8 * 8)
        case = dict(op=op, dim=dim, tokens=_log(rng, 1, min(32768, 52_000_000 // dim)),
                    weight=rng.choice(["f32", "bf16", "none"]))
        if op == "grad":
            case.update(x=rng.choice(["f32", "bf16"]), dy=rng.choice(["f32", "bf16"]),
                        stream=rng.random() < 0.7)
            return case
        case.update(rng.choice([dict(x="bf16", stream="bf16"), dict(x="bf16", stream="f32"),
                                dict(x="f32", stream="f32"), dict(x="bf16", stream="none"),
                                dict(x="f32", stream="none")]))
        if op == "norm":
            case.update(out=rng.choice(["f32", "bf16"]))
        else:
            case.update(group=rng.choice([0, 0, 32, 64, 128]))
        return case
    model = rng.choice(["ragged", "ragged", "bert", "gpt"])
    case = dict(op=op, model=model, norm=rng.choice(["l2", "l2", "l1", "linf"]))
    if model == "ragged":
        case.update(tensors=_log(rng, 1, 300), largest=_log(rng, 40, 2_000_000),
                    grad=rng.choice(["mixed", "f32", "bf16"]))
    else:
        case.update(hidden=8 * _log(rng, 8, 160), layers=_log(rng, 1, 12),
                    grad=rng.choice(["f32", "bf16"]))
    if op == "clip":
        # what is clipped in place is clipped once: a second pass finds it within the limit
        above = rng.random() < 0.7
        case.update(above=above, out=rng.choice(["f32", "bf16"] if above else ["same", "bf16"]))
        if case["out"] == "same":
            case.update(norm="l2")
    return case


def _shapes(case):
    """The tensors of a model, as numbers of elements, in their order."""
    model = case["model"]
    if model == "tiny":
        return [65536, 256, 262144, 1024, 262144, 256, 16384, 256]
    if model == "ragged":
        n, top = case["tensors"], case["largest"]
        return [max(1, int(top ** (((7 * i) % n + 1) / n)) - i % 2) for i in range(n)]
    h, layers = case["hidden"], case["layers"]
    if model == "bert":
        sizes = [30522 * h, 512 * h, 2 * h, h, h]
        for _ in range(layers):
            sizes += 4 * [h * h, h] + [h, h, 4 * h * h, 4 * h, 4 * h * h, h, h, h]
        return sizes + [h * h, h]
    sizes = [50257 * h, 1024 * h]
    for _ in range(layers):
        sizes += [h, h, 3 * h * h, 3 * h, h * h, h, h, h, 4 * h * h, 4 * h, 4 * h * h, h]
    return sizes + [h, h]


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _types(case):
    """The type of each gradient tensor."""
    if case["grad"] == "mixed":
        return [("f32", "bf16")[i % 2] for i in range(len(_shapes(case)))]
    return [case["grad"]] * len(_shapes(case))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(9176 * int(seed) + 5)


def _normal(gen, *shape, sigma=1.0, dtype="f32"):
    return torch.randn(*shape, generator=gen, device="cuda").mul_(sigma).to(_dtype(dtype))


def _views(flat, case):
    """The tensors of the buffers ``flat``, one after another in that of their type."""
    at, views = dict.fromkeys(flat, 0), []
    for n, t in zip(_shapes(case), _types(case)):
        views.append(flat[t][at[t]:at[t] + n])
        at[t] += n
    return views


def _gradients(case, gen):
    """Gradients whose standard deviation differs from tensor to tensor, over two
    decades, scaled so that their norm is about twice the limit, or half of it."""
    sizes, types = _shapes(case), _types(case)
    spread = (torch.rand(len(sizes), generator=gen, device="cuda") * 4.6).exp_().tolist()
    power = sum(n * s * s for n, s in zip(sizes, spread))
    common = {"l2": math.sqrt(power), "linf": 4.0 * max(spread),
              "l1": 0.8 * sum(n * s for n, s in zip(sizes, spread))}[case["norm"]]
    target = (2.0 if case.get("above", True) else 0.5) * LIMIT
    flat = {t: torch.randn(sum(n for n, u in zip(sizes, types) if u == t), generator=gen,
                           device="cuda") for t in sorted(set(types))}
    for v, s in zip(_views(flat, case), spread):
        v.mul_(s * target / common)
    return {t: v.to(_dtype(t)) for t, v in flat.items()}


def prepare(case, seed):
    gen = _gen(seed)
    s = dict(case=case)
    op = case["op"]
    if op in ("gnorm", "clip"):
        s["flat"] = _gradients(case, gen)
        s["grads"] = _views(s["flat"], case)
        s["to"] = None
        if op == "clip" and case["out"] != "same":
            s["to"] = {t: torch.empty(v.shape, dtype=_dtype(case["out"]), device="cuda")
                       for t, v in s["flat"].items()}
        if own:
            _prepare_own(s)
        return s
    n, d = case["tokens"], case["dim"]
    # a residual stream has a few columns that are far larger than the others, and tokens
    # of different size
    columns = torch.ones(d, device="cuda")
    columns[torch.randint(0, d, (max(1, d // 200),), generator=gen, device="cuda")] = 15.0
    rows = torch.rand(n, 1, generator=gen, device="cuda").mul_(2.0).exp_()
    wide = torch.randn(n, d, generator=gen, device="cuda").mul_(columns).mul_(rows)
    s["weight"] = (None if case["weight"] == "none" else
                   (_normal(gen, d, sigma=0.2) + 1.0).to(_dtype(case["weight"])))
    if op == "grad":
        s["x"] = wide.to(_dtype(case["x"]))
        s["dy"] = _normal(gen, n, d, sigma=1e-3, dtype=case["dy"])
        s["ds"] = _normal(gen, n, d, sigma=1e-3, dtype=case["x"]) if case["stream"] else None
        s["grad_x"] = torch.empty_like(s["x"])
        s["grad_weight"] = (None if s["weight"] is None else
                            torch.empty(d, dtype=torch.float32, device="cuda"))
    elif case["stream"] == "none":
        s["x"], s["stream"] = wide.to(_dtype(case["x"])), None
    else:
        s["x"] = _normal(gen, n, d, dtype=case["x"])
        s["stream"] = wide.to(_dtype(case["stream"]))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_1904_00962_amd import ops
    s["ops"] = ops
    if "grads" in s:
        outputs = None if s["to"] is None else _views(s["to"], s["case"])
        s["plan"] = ops.GradNorm(s["grads"], outputs, norm=s["case"]["norm"])


def _inverse(x):
    """1 / root mean square of each row of an fp32 tensor."""
    return torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS)


def _run_norm(s):
    """(the sum of x and the stream, or None; the norm's result in fp32)."""
    x = s["x"].float()
    summed = None
    if s["stream"] is not None:
        # what is normed is the sum as the stream keeps it
        summed = (x + s["stream"].float()).to(s["stream"].dtype)
        x = summed.float()
    y = x * _inverse(x)
    return summed, y if s["weight"] is None else y * s["weight"].float()


def _tensor_norms(grads, kind):
    if kind == "l2":
        return torch.stack([g.double().square().sum() for g in grads]).sqrt()
    if kind == "l1":
        return torch.stack([g.double().abs().sum() for g in grads])
    return torch.stack([g.abs().max().double() for g in grads])


def _common_norm(norms, kind):
    if kind == "l2":
        return norms.square().sum().sqrt()
    return norms.sum() if kind == "l1" else norms.max()


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        summed, y = _run_norm(s)
        y = y.to(_dtype(case["out"]))
        return dict(out=y) if summed is None else dict(out=y, summed=summed)
    if op == "norm8":
        summed, y = _run_norm(s)
        n, d = y.shape
        group = case["group"] or d
        y = torch.nn.functional.pad(y, (0, -d % group)).view(n, -1, group)
        scales = (y.abs().amax(dim=2) / LARGEST_E4M3).clamp_(min=LEAST_SCALE)
        q = (y / scales[:, :, None]).view(n, -1)[:, :d].to(torch.float8_e4m3fn)
        return dict(out=q, scales=scales) | ({} if summed is None else dict(summed=summed))
    if op == "grad":
        x, dy = s["x"].float(), s["dy"].float()
        inverse = _inverse(x)
        x = x * inverse
        g = dy if s["weight"] is None else dy * s["weight"].float()
        g = (g - x * (g * x).mean(dim=1, keepdim=True)) * inverse
        s["grad_x"].copy_(g if s["ds"] is None else g + s["ds"].float())
        if s["weight"] is None:
            return dict(grad_x=s["grad_x"])
        s["grad_weight"].copy_((dy * x).sum(dim=0))
        return dict(grad_x=s["grad_x"], grad_weight=s["grad_weight"])
    norms = _tensor_norms(s["grads"], case["norm"])
    total = _common_norm(norms, case["norm"])
    if op == "gnorm":
        return dict(total=total, norms=norms)
    factor = (LIMIT / total).clamp(max=1.0).float()
    to = s["flat"] if s["to"] is None else s["to"]
    for t, v in s["flat"].items():
        to[t].copy_(v.float() * factor)
    return dict(total=total, grads=to)


def run(s):
    if not own:
        return _run_plain(s)
    case, ops = s["case"], s["ops"]
    op = case["op"]
    if op == "norm":
        got = ops.rms_norm(s["x"], s["weight"], residual=s["stream"], eps=EPS,
                           out_dtype=_dtype(case["out"]))
        return dict(out=got) if s["stream"] is None else dict(out=got[0], summed=got[1])
    if op == "norm8":
        q, scales, *summed = ops.rms_norm_fp8(s["x"], s["weight"], residual=s["stream"], eps=EPS,
                                              group=case["group"])
        return dict(out=q, scales=scales) | (dict(summed=summed[0]) if summed else {})
    if op == "grad":
        ops.rms_norm_grad(s["x"], s["weight"], s["dy"], s["grad_x"], s["grad_weight"], eps=EPS,
                          grad_sum=s["ds"])
        if s["weight"] is None:
            return dict(grad_x=s["grad_x"])
        return dict(grad_x=s["grad_x"], grad_weight=s["grad_weight"])
    if op == "gnorm":
        return dict(total=s["plan"].run(), norms=s["plan"].norms)
    return dict(total=s["plan"].clip(LIMIT), grads=s["flat"] if s["to"] is None else s["to"])


def work(case):
    """Bytes: inputs once, outputs once (gradients that keep the limit in place are only
    read). Flops: an addition or a product each, for an element."""
    size = {"f32": 4, "bf16": 2, "none": 0}
    op = case["op"]
    if op in ("gnorm", "clip"):
        numel = sum(_shapes(case))
        read = sum(n * size[t] for n, t in zip(_shapes(case), _types(case)))
        written = 0
        if op == "clip" and case["out"] != "same":
            written = numel * size[case["out"]]
        return {"bytes": float(read + written),
                "flops": float(numel * (3 if written else 2))}
    n, d = case["tokens"], case["dim"]
    if op == "grad":
        each = size[case["x"]] * (3 if case["stream"] else 2) + size[case["dy"]]
        weight = d * (size[case["weight"]] + 4) if case["weight"] != "none" else 0
        return {"bytes": float(n * d * each + weight), "flops": 12.0 * n * d}
    each = size[case["x"]] + 2 * size[case["stream"]]
    extra = d * size[case["weight"]]
    if op == "norm":
        each += size[case["out"]]
    else:
        each += 1
        extra += 4 * n * (-(-d // case["group"]) if case["group"] else 1)
    return {"bytes": float(n * d * each + extra), "flops": (8.0 if op == "norm8" else 5.0) * n * d}


def _exact_norm(s):
    h = s["x"].double()
    if s["stream"] is not None:
        h = h + s["stream"].double()
    kept = h
    if s["stream"] is not None and s["stream"].dtype == torch.bfloat16:
        # the norm is that of the rounded stream: a sum of two bf16 numbers is exact in 64 bits
        kept = h.to(torch.bfloat16).double()
    elif s["stream"] is not None:
        kept = h.to(torch.float32).double()
    power = torch.linalg.vector_norm(kept, dim=1, keepdim=True).square() / h.shape[1] + EPS
    y = kept / torch.sqrt(power)
    return h, y if s["weight"] is None else y * s["weight"].double()


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op in ("norm", "norm8"):
        h, y = _exact_norm(s)
        got = dict(out=y)
        if s["stream"] is not None:
            got["summed"] = h
        if op == "norm8":
            n, d = y.shape
            step = case["group"] or d
            parts = torch.split(y, step, dim=1)
            scales = torch.stack([torch.linalg.vector_norm(p, ord=math.inf, dim=1)
                                  for p in parts], dim=1) / LARGEST_E4M3
            scales = torch.clamp(scales, min=LEAST_SCALE)
            got["out"] = torch.cat([p / scales[:, i:i + 1] for i, p in enumerate(parts)], dim=1)
            got["scales"] = scales
        return got
    if op == "grad":
        x, dy = s["x"].double(), s["dy"].double()
        d = case["dim"]
        power = torch.linalg.vector_norm(x, dim=1, keepdim=True).square() / d + EPS
        w = torch.ones(d, dtype=torch.float64, device="cuda")
        if s["weight"] is not None:
            w = s["weight"].double()
        # d/dx_j of sum_i dy_i w_i x_i p^-1/2 with p = mean x^2 + eps
        along = torch.linalg.vecdot(dy * w, x, dim=1)[:, None]
        gx = dy * w / power.sqrt() - x * along / (d * power ** 1.5)
        if s["ds"] is not None:
            gx += s["ds"].double()
        if s["weight"] is None:
            return dict(grad_x=gx)
        return dict(grad_x=gx, grad_weight=(dy * (x / power.sqrt())).sum(dim=0))
    order = {"l2": 2.0, "l1": 1.0, "linf": math.inf}[case["norm"]]
    norms = torch.stack([torch.linalg.vector_norm(g.double(), ord=order) for g in s["grads"]])
    total = torch.linalg.vector_norm(norms, ord=order)
    if op == "gnorm":
        return dict(total=total, norms=norms)
    factor = min(1.0, LIMIT / float(total))
    return dict(total=total, grads={t: v.double() * factor for t, v in s["flat"].items()})
