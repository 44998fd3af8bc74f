"""The language-model operators whose speed is measured: one dict of plain values per case.

A training step of a language model around the compressed gradient: tokens are looked up in the embedding, the gradient of
the embedding is summed by token into the flat gradient that is compressed, and once the workers' messages have been
decompressed the weight matrices take a step whose direction is the orthogonalised momentum.  Serving needs the first of
them alone, down to a single token.

``listed()`` names the cases, ``draw(rng)`` gives others of the same ranges, ``prepare`` makes what a program has in hand
before the call, ``run`` is one pass: with ``own`` set through the package's entry points, otherwise in elementary torch
operations.  ``exact`` is the definition in 64 bits, written apart from both.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)   # the odd quintic of a Newton-Schulz step
EPS = 1e-7                                 # added to the Frobenius norm
BETA, KEEP, ALPHA = 0.95, 0.998, -0.02     # momentum, 1 - rate * decay, -rate


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one new token of one sequence: latency alone
        {"name": "lookup_one_token", "kind": "lookup", "tokens": 1, "vocab": 32_000, "dim": 4096, "type": "bfloat16",
         "index": 8, "scale": 1.0, "padded": 0.0},
        # a batch of the LSTM language model: 20 sequences of 35 tokens, rows of an odd length
        {"name": "lookup_lstm", "kind": "lookup", "tokens": 700, "vocab": 33_278, "dim": 650, "type": "float32",
         "index": 8, "scale": 1.0, "padded": 0.0},
        # a padded batch of long prompts, scaled by the square root of the width
        {"name": "lookup_long", "kind": "lookup", "tokens": 65_539, "vocab": 131_072, "dim": 4096, "type": "bfloat16",
         "index": 8, "scale": 64.0, "padded": 0.1},
        # the rows of eight tokens added to a gradient that holds the tied output layer's part already
        {"name": "gradient_few", "kind": "gradient", "tokens": 8, "vocab": 32_000, "dim": 1024, "type": "float32",
         "index": 4, "scale": 1.0, "padded": 0.0, "accumulate": True},
        # the LSTM language model's batch: the whole table's gradient, most of its rows zero
        {"name": "gradient_lstm", "kind": "gradient", "tokens": 700, "vocab": 33_278, "dim": 650, "type": "float32",
         "index": 8, "scale": 1.0, "padded": 0.0, "accumulate": False},
        # an ordinary batch, padded, added to the tied output layer's part
        {"name": "gradient_batch", "kind": "gradient", "tokens": 16_381, "vocab": 50_001, "dim": 1600, "type": "bfloat16",
         "index": 8, "scale": 1.0, "padded": 0.2, "accumulate": True},
        # the largest batch on a large table
        {"name": "gradient_long", "kind": "gradient", "tokens": 131_072, "vocab": 131_072, "dim": 4096, "type": "bfloat16",
         "index": 8, "scale": 64.0, "padded": 0.0, "accumulate": False},
        # one small projection: a chain of small products
        {"name": "orthogonalize_small", "kind": "orthogonalize", "matrices": "512x128", "type": "bfloat16", "steps": 5},
        # the gate matrices of the two-layer LSTM
        {"name": "orthogonalize_lstm", "kind": "orthogonalize", "matrices": "2600x650 2600x650 2600x650 2600x650",
         "type": "float32", "steps": 5},
        # a square projection of a wide model, kept in 16 bits
        {"name": "orthogonalize_square", "kind": "orthogonalize", "matrices": "4096x4096", "type": "bfloat16", "steps": 5},
        # the step on all convolutions and the classifier of ResNet101 (105 matrices and what lies between them)
        {"name": "update_resnet101", "kind": "update", "matrices": "resnet101", "type": "float32", "steps": 5, "nesterov": True},
        # ... and of VGG16, whose first fully connected layer has three quarters of the parameters
        {"name": "update_vgg16", "kind": "update", "matrices": "vgg16", "type": "float32", "steps": 5, "nesterov": True},
    ]


def _size(rng, lo, hi):
    """A size spread over its logarithm, odd ones and round ones among them."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(1, min(hi, rng.choice([n, n | 1, (n + 63) // 64 * 64])))


def draw(rng):
    kind = rng.choice(["lookup", "gradient", "orthogonalize", "update"])
    if kind in ("lookup", "gradient"):
        case = {"kind": kind, "tokens": _size(rng, 1, 65_536), "vocab": _size(rng, 1000, 131_072), "dim": _size(rng, 64, 4096),
                "type": rng.choice(["float32", "bfloat16", "float16"]), "index": rng.choice([4, 8]),
                "scale": rng.choice([1.0, 0.3, 32.0]), "padded": rng.choice([0.0, 0.1, 0.5])}
        if kind == "gradient":
            case["accumulate"] = rng.random() < 0.5
        return case
    shapes = []
    for _ in range(rng.choice([1, 1, 2, 4, 12])):
        a, b = _size(rng, 16, 2560), _size(rng, 16, 5120)
        shapes.append("%dx%d" % ((a, b) if rng.random() < 0.5 else (b, a)))
    case = {"kind": kind, "matrices": " ".join(shapes), "type": rng.choice(["float32", "float32", "bfloat16", "float16"]),
            "steps": rng.choice([3, 5, 5, 6])}
    if kind == "update":
        case["type"] = rng.choice(["float32", "float32", "bfloat16"])
        case["nesterov"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------------------------------------------------
# the flat vectors of the matrices' operators
# ---------------------------------------------------------------------------------------------------------------------

def _layout(case):
    """The tensors of a flat parameter vector, in order: (rows, cols), rows 0 for one that is no matrix."""
    name = case["matrices"]
    if name == "resnet101":
        # a convolution is its output channels by all that one of them reads
        out = [(64, 147), (0, 64), (0, 64)]
        cin = 64
        for blocks, w in ((3, 64), (4, 128), (23, 256), (3, 512)):
            for b in range(blocks):
                for r, c in ((w, cin), (w, 9 * w), (4 * w, w)):
                    out += [(r, c), (0, r), (0, r)]
                if b == 0:
                    out += [(4 * w, cin), (0, 4 * w), (0, 4 * w)]
                cin = 4 * w
        return out + [(1000, 2048), (0, 1000)]
    if name == "vgg16":
        out, cin = [], 3
        for c in (64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512):
            out += [(c, 9 * cin), (0, c)]
            cin = c
        for r, c in ((4096, 25088), (4096, 4096), (1000, 4096)):
            out += [(r, c), (0, r)]
        return out
    return [tuple(int(v) for v in s.split("x")) for s in name.split()]


def _matrices(case):
    """(length of the flat vector, [(offset, rows, cols)])."""
    at, found = 0, []
    for rows, cols in _layout(case):
        if rows:
            found.append((at, rows, cols))
        at += max(rows, 1) * cols
    return at, found


def _scale(rows, cols):
    """The step of a matrix, so that its entries change as much as with a normalised element-wise step."""
    return 0.2 * math.sqrt(max(rows, cols))


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------

def _shares(vocab):
    """How often the tokens of a text occur, the most frequent first."""
    p = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7)
    return p / p.sum()


def _tokens(case, gen):
    """Tokens of a text over a shuffled vocabulary; padded places hold -1, which is no token."""
    T, V = case["tokens"], case["vocab"]
    edges = torch.from_numpy(np.cumsum(_shares(V))).cuda()
    rank = torch.searchsorted(edges, torch.rand(T, dtype=torch.float64, device="cuda", generator=gen)).clamp_(max=V - 1)
    t = torch.randperm(V, device="cuda", generator=gen)[rank]
    if case["padded"]:
        t = torch.where(torch.rand(T, device="cuda", generator=gen) < case["padded"], -1, t)
    return t.to(torch.int64 if case["index"] == 8 else torch.int32)


def _gradient_like(rows, cols, gen):
    """A matrix as momentum is: few directions that many steps share, and the noise of the last ones."""
    r = min(8, rows, cols)
    u = torch.randn(rows, r, device="cuda", generator=gen)
    v = torch.randn(r, cols, device="cuda", generator=gen)
    g = torch.randn(rows, cols, device="cuda", generator=gen)
    return g.addmm_(u, v, alpha=0.5 / math.sqrt(r)).mul_(1e-4)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], {"case": case}
    if kind in ("lookup", "gradient"):
        T, V, D, t = case["tokens"], case["vocab"], case["dim"], TYPES[case["type"]]
        s["tokens"] = _tokens(case, gen)
        if kind == "lookup":
            s["table"] = torch.randn(V, D, device="cuda", generator=gen).mul_(0.02).to(t)
            s["out"] = torch.empty(T, D, dtype=t, device="cuda")
        else:
            s["grad_out"] = torch.randn(T, D, device="cuda", generator=gen).mul_(1e-3).to(t)
            s["table_grad"] = torch.randn(V, D, device="cuda", generator=gen).mul_(1e-3)
        return s
    n, s["matrices"] = _matrices(case)
    x = torch.randn(n, device="cuda", generator=gen).mul_(1e-4)
    for at, rows, cols in s["matrices"]:
        x[at:at + rows * cols] = _gradient_like(rows, cols, gen).view(-1)
    if kind == "orthogonalize":
        s["x"] = x.to(TYPES[case["type"]])
        s["out"] = torch.zeros_like(s["x"])
        return s
    s["momentum"] = x.mul_(10.0)
    s["grad"] = torch.randn(n, device="cuda", generator=gen).mul_(1e-4)
    s["params"] = torch.randn(n, device="cuda", generator=gen).mul_(0.02).to(TYPES[case["type"]])
    s["scales"] = [_scale(rows, cols) for _, rows, cols in s["matrices"]]
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------

def _lookup(s):
    t, V = s["tokens"].long(), s["case"]["vocab"]
    rows = s["table"][t.clamp(0, V - 1)].float() * s["case"]["scale"]
    s["out"].copy_(torch.where(((t >= 0) & (t < V))[:, None], rows, 0.0))
    return s["out"]


def _gradient(s):
    t, V, g = s["tokens"].long(), s["case"]["vocab"], s["table_grad"]
    real = (t >= 0) & (t < V)
    rows = torch.where(real[:, None], s["grad_out"].float(), 0.0)
    # places that hold no token add zeros, each to a row of its own: all to one would be a queue at that row
    t = torch.where(real, t, torch.arange(t.numel(), device=t.device) % V)
    if not s["case"]["accumulate"]:
        g.zero_()
    return g.index_add_(0, t, rows, alpha=s["case"]["scale"])


def _orthogonal(x, steps):
    """The Newton-Schulz products on a batch of matrices of one shape, float32."""
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt().float() + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        g = x @ x.transpose(1, 2)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.transpose(1, 2) if tall else x


def _by_shape(matrices):
    found = {}
    for i, (_, rows, cols) in enumerate(matrices):
        found.setdefault((rows, cols), []).append(i)
    return found.items()


def _orthogonal_all(flat, matrices, steps):
    """The orthogonalised matrices of a flat vector, matrices of one shape together, in their order."""
    got = [None] * len(matrices)
    for (rows, cols), at in _by_shape(matrices):
        x = torch.stack([flat[matrices[i][0]:matrices[i][0] + rows * cols].view(rows, cols) for i in at]).float()
        for i, y in zip(at, _orthogonal(x, steps)):
            got[i] = y
    return got


def _orthogonalize(s):
    for (at, rows, cols), y in zip(s["matrices"], _orthogonal_all(s["x"], s["matrices"], s["case"]["steps"])):
        s["out"][at:at + rows * cols].view(rows, cols).copy_(y)
    return s["out"]


def _update(s):
    mom, grad, params, matrices = s["momentum"], s["grad"], s["params"], s["matrices"]
    new = BETA * mom + grad
    along = grad + BETA * new if s["case"]["nesterov"] else new
    ys = _orthogonal_all(along, matrices, s["case"]["steps"])
    for (at, rows, cols), scale, y in zip(matrices, s["scales"], ys):
        part = slice(at, at + rows * cols)
        mom[part] = new[part]
        params[part].view(rows, cols).copy_(KEEP * params[part].view(rows, cols).float() + (ALPHA * scale) * y)
    return {"momentum": mom, "params": params}


def _own(s):
    """The same through the package.  Workspaces are made on a state's first pass and kept with it."""
    from paper_2305_12201_amd import binding
    case, kind = s["case"], s["case"]["kind"]
    if kind == "lookup":
        binding.gravac_embedding_lookup(s["table"], s["tokens"], s["out"], scale=case["scale"])
        return s["out"]
    if kind == "gradient":
        if "workspace" not in s:
            size = binding.gravac_embedding_gradient_workspace_bytes(case["tokens"], case["vocab"], case["dim"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        binding.gravac_embedding_gradient(s["grad_out"], s["tokens"], s["table_grad"], scale=case["scale"],
                                          accumulate=case["accumulate"], workspace=s["workspace"])
        return s["table_grad"]
    if "orthogonalizer" not in s:
        n = s["x" if kind == "orthogonalize" else "params"].numel()
        s["orthogonalizer"] = binding.Orthogonalizer(n, s["matrices"], dtype=TYPES[case["type"]], steps=case["steps"],
                                                     coefficients=COEFFICIENTS, eps=EPS)
    if kind == "orthogonalize":
        s["orthogonalizer"](s["x"], s["out"])
        return s["out"]
    s["orthogonalizer"].update(s["grad"], s["momentum"], s["params"], beta=BETA, nesterov=case["nesterov"], keep=KEEP,
                               alpha=ALPHA, scales=s["scales"])
    return {"momentum": s["momentum"], "params": s["params"]}


def run(s):
    if own:
        return _own(s)
    return {"lookup": _lookup, "gradient": _gradient, "orthogonalize": _orthogonalize, "update": _update}[s["case"]["kind"]](s)


def work(case):
    """Bytes read and written once, and the products that cannot be left out.

    A lookup reads its tokens and the distinct rows that they name and writes its output; a gradient reads the tokens and the
    rows of the output's gradient and writes the table's (read too, and only the named rows, if it is added to).  A
    Newton-Schulz step of an m by n matrix (m <= n) is X X^T and its square, of which half is needed (both are symmetric),
    and one product with X: m m n + m m m + 2 m m n operations counted in pairs."""
    kind = case["kind"]
    if kind in ("lookup", "gradient"):
        T, V, D, size = case["tokens"], case["vocab"], case["dim"], BYTES[case["type"]]
        real = T * (1.0 - case["padded"])
        named = float(np.sum(-np.expm1(real * np.log1p(-_shares(V)))))
        if kind == "lookup":
            return {"bytes": case["index"] * T + named * D * size + T * D * size, "flops": T * D}
        table = 8 * named * D if case["accumulate"] else 4 * V * D
        return {"bytes": case["index"] * T + real * D * size + table, "flops": real * D}
    n, matrices = _matrices(case)
    inside = sum(r * c for _, r, c in matrices)
    flops = 0
    for _, r, c in matrices:
        m, k = min(r, c), max(r, c)
        flops += case["steps"] * (3 * m * m * k + m * m * m)
    size = BYTES[case["type"]]
    return {"bytes": inside * (2 * size if kind == "orthogonalize" else 12 + 2 * size), "flops": flops}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------

def _exact_direction(x, steps):
    """sum over the singular directions of p(p(...p(s / (|x| + eps)))) u v^T, p(s) = a s + b s^3 + c s^5, by products in
    64 bits from the left or from the right, whichever is smaller."""
    a, b, c = COEFFICIENTS
    x = x.double()
    y = x / (torch.linalg.vector_norm(x) + EPS)
    one = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
    for _ in range(steps):
        q = y.t().mm(y) if x.shape[0] > x.shape[1] else y.mm(y.t())
        poly = a * one + q.mm(b * one + c * q)
        y = y.mm(poly) if x.shape[0] > x.shape[1] else poly.mm(y)
    return y


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("lookup", "gradient"):
        t, V = s["tokens"].cpu().numpy().astype(np.int64), case["vocab"]
        at = torch.from_numpy(np.flatnonzero((t >= 0) & (t < V))).cuda()
        ids = s["tokens"][at].long()
        if kind == "lookup":
            out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
            out[at] = s["table"].double()[ids] * case["scale"]
            return out
        sums = torch.zeros(V, case["dim"], dtype=torch.float64, device="cuda")
        sums.index_put_((ids,), s["grad_out"].double()[at], accumulate=True)
        sums *= case["scale"]
        return sums + s["table_grad"].double() if case["accumulate"] else sums
    if kind == "orthogonalize":
        out = torch.zeros(s["x"].numel(), dtype=torch.float64, device="cuda")
        for at, rows, cols in s["matrices"]:
            out[at:at + rows * cols] = _exact_direction(s["x"][at:at + rows * cols].view(rows, cols), case["steps"]).reshape(-1)
        return out
    beta, keep, grad = BETA, KEEP, s["grad"].double()
    mom, params = s["momentum"].double(), s["params"].double()
    for (at, rows, cols), scale in zip(s["matrices"], s["scales"]):
        part = slice(at, at + rows * cols)
        mom[part] = beta * mom[part] + grad[part]
        along = grad[part] + beta * mom[part] if case["nesterov"] else mom[part]
        params[part] = keep * params[part] + ALPHA * scale * _exact_direction(along.view(rows, cols), case["steps"]).reshape(-1)
    return {"momentum": mom, "params": params}
