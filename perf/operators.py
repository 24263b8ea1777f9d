"""The operators of a layer with sparse weights, as cases that can be timed: forward, backward, and the clipping of its gradients.

Y = act(A x X + bias) + residual, A sparse (the weights of a pruned layer, m outputs x k inputs), X dense with a column
per token.  A case names the operator and its sizes:

  forward   the product with its epilogue: bias, activation, residual; in training also the values in front of the activation
  epilogue  the gradient through the epilogue: the activation's, and the bias's as sums over the tokens
  values    the gradient of the stored weights: one scalar product of two rows, N long, for each entry of A
  clip      the norm over all gradients of a step, and the gradients scaled to a given norm

The gradient of X is a forward case as well: the same product with the transpose of A and no epilogue.
Without `own` the operators are computed in their plain form: the weights as a dense matrix in 32 bits that the
program keeps, products, sums and comparisons.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTIVATIONS = ("none", "relu", "silu", "gelu", "gelu_tanh")
MOST_PRODUCTS = 5.2e10                       # stored entries x N of the largest forward case
MOST_DENSE = 5.2e11                          # m x k x N of the largest case whose plain form multiplies dense matrices


def listed():
    return [
        # one token through a layer as serving has it: what counts is reading the weights once
        dict(name="forward_token", op="forward", m=8000, k=8000, N=1, density=0.1, type="bf16", act="gelu", bias=True, residual=True, keep=False),
        # the smallest training step, where launches and the host path are all there is
        dict(name="forward_256", op="forward", m=256, k=256, N=256, density=0.1, type="f32", act="relu", bias=True, residual=False, keep=True),
        # nothing square, nothing a multiple of anything
        dict(name="forward_ragged", op="forward", m=1777, k=2301, N=1117, density=0.03, type="f16", act="silu", bias=True, residual=True, keep=True),
        # the headline matrix of bench.py as a layer: very sparse weights over many tokens
        dict(name="forward_sparse", op="forward", m=8000, k=8000, N=8000, density=0.005, type="bf16", act="gelu_tanh", bias=True, residual=True, keep=False),
        # the densest of the large ones
        dict(name="forward_8000", op="forward", m=8000, k=8000, N=8000, density=0.1, type="f32", act="gelu", bias=True, residual=True, keep=True),
        # a small batch through the epilogue's gradient
        dict(name="epilogue_1000", op="epilogue", m=1000, N=333, type="f32", act="gelu"),
        # a wide layer over a long batch
        dict(name="epilogue_14000", op="epilogue", m=14000, N=8000, type="bf16", act="silu"),
        # the smallest training step again
        dict(name="values_256", op="values", m=256, k=256, N=256, density=0.1, type="f32"),
        # very sparse weights over many tokens
        dict(name="values_sparse", op="values", m=8000, k=8000, N=8000, density=0.005, type="bf16"),
        # weights of which every twentieth is left, odd sizes
        dict(name="values_4001", op="values", m=4001, k=3999, N=4003, density=0.05, type="bf16"),
        # the gradients of one small layer
        dict(name="clip_layer", op="clip", entries=80000, tensors=3, type="f32"),
        # the gradients of a whole network: many tensors of very different sizes
        dict(name="clip_network", op="clip", entries=150000000, tensors=60, type="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _around(rng, n, most):
    return n if rng.random() < 0.3 else max(1, min(most, int(n * rng.uniform(0.5, 1.9))))


def draw(rng):
    op = rng.choice(["forward", "forward", "forward", "epilogue", "values", "values", "clip"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op == "clip":
        return dict(op=op, entries=_spread(rng, 5000, 150000000), tensors=_spread(rng, 1, 60), type=rng.choice(["f32", "f32", "bf16", "f16"]))
    if op == "epilogue":
        m = _spread(rng, 100, 14000)
        return dict(op=op, m=m, N=_spread(rng, 1, 8000), type=kind, act=rng.choice(ACTIVATIONS[1:]))
    m = _spread(rng, 256, 14000)
    k, N = _around(rng, m, 14000), _spread(rng, 1, 8000)
    if rng.random() < 0.15:
        N = rng.randint(1, 16)
    density = min(math.exp(rng.uniform(math.log(0.0005), math.log(0.25))), MOST_PRODUCTS / (m * k * N))
    N = max(1, min(N, int(MOST_DENSE / (m * k))))
    case = dict(op=op, m=m, k=k, N=N, density=round(max(density, 2e-5), 6), type=kind)
    if op == "forward":
        case.update(act=rng.choice(ACTIVATIONS), bias=rng.random() < 0.8, residual=rng.random() < 0.6, keep=rng.random() < 0.4)
    return case


def _entries(case):
    return max(1, int(round(case["density"] * case["m"] * case["k"])))


def _csr(case, g):
    """Cells drawn without replacement, columns of a row ascending; weights of a layer whose outputs are of order one."""
    m, k, want = case["m"], case["k"], _entries(case)
    cells = torch.empty(0, dtype=torch.int64, device=DEV)
    while cells.numel() < want:
        more = torch.randint(m * k, (int(1.2 * (want - cells.numel())) + 64,), generator=g, device=DEV)
        cells = torch.unique(torch.cat([cells, more]))
    keep = torch.randperm(cells.numel(), generator=g, device=DEV)[:want]
    cells = torch.sort(cells[keep]).values
    rows = torch.div(cells, k, rounding_mode="floor")
    row_ptr = torch.zeros(m + 1, dtype=torch.int64, device=DEV)
    row_ptr[1:] = torch.cumsum(torch.bincount(rows, minlength=m), 0)
    vals = torch.randn(want, generator=g, device=DEV, dtype=torch.float32) * (m / want) ** 0.5
    return row_ptr.to(torch.int32), (cells - rows * k).to(torch.int32), vals, rows


def _sizes(case):
    """Elements of each gradient: as uneven as a network's are, matrices beside vectors."""
    n, total = case["tensors"], case["entries"]
    shares = [1.0 / (1 + (i * 7919) % 23) ** 1.5 for i in range(n)]
    return [max(1, int(total * s / sum(shares))) for s in shares]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, kind = case["op"], TYPES[case["type"]]

    def normal(*shape, scale=1.0, type=kind):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(type)

    state = dict(case=case, op=op, kind=kind, act=case.get("act", "none"))
    if op == "clip":
        state["grads"] = [normal(n, scale=2e-3) for n in _sizes(case)]
        state["out"] = [torch.empty_like(x) for x in state["grads"]]
        state["max_norm"] = 1.0
        return state
    m, N = case["m"], case["N"]
    if op == "epilogue":
        state["dY"], state["Z"] = normal(m, N, scale=0.1), normal(m, N)
        return state
    k = case["k"]
    row_ptr, cols, vals, rows = _csr(case, g)
    state["X"] = normal(k, N)
    if op == "forward":
        state["bias"] = normal(m, scale=0.1, type=torch.float32) if case["bias"] else None
        state["residual"] = normal(m, N) if case["residual"] else None
    else:
        state["dZ"] = normal(m, N, scale=0.1)
    if own:
        from paper_2005_14469_amd import binding
        p = binding.gcoo_default_p(m, k, vals.numel(), N)
        state["A"] = binding.gcoo_from_csr(m, k, row_ptr, cols, vals, p, known_nnz=True)
    elif op == "forward":
        state["W"] = torch.zeros((m, k), dtype=torch.float32, device=DEV)
        state["W"][rows, cols.long()] = vals
    else:
        state["cells"] = (rows, cols.long())
    return state


# ---- plain form ----

def _activate(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 2 ** -0.5))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 2 ** -0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if name == "gelu_tanh":
        a = (2 / math.pi) ** 0.5
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain(state):
    op, kind = state["op"], state["kind"]
    if op == "forward":
        z = state["W"] @ state["X"].float()
        if state["bias"] is not None:
            z = z + state["bias"][:, None]
        y = _activate(state["act"], z)
        if state["residual"] is not None:
            y = y + state["residual"].float()
        return (y.to(kind), z.to(kind)) if state["case"]["keep"] else (y.to(kind),)
    if op == "epilogue":
        dz = state["dY"].float() * _slope(state["act"], state["Z"].float())
        return dz.to(kind), dz.sum(1)
    if op == "values":
        return ((state["dZ"].float() @ state["X"].float().t().contiguous())[state["cells"]],)
    squares = torch.stack([x.float().square().sum(dtype=torch.float64) for x in state["grads"]])
    norm = squares.sum().sqrt().float()
    scale = torch.clamp(state["max_norm"] / (norm + 1e-6), max=1.0)
    return (norm, *[(x.float() * scale).to(kind) for x in state["grads"]])


# ---- the framework's operators ----

def _own(state):
    from paper_2005_14469_amd import binding
    op, act = state["op"], state["act"]
    if op == "forward":
        m, N = state["case"]["m"], state["case"]["N"]
        z = torch.empty((m, N), dtype=state["kind"], device=DEV) if state["case"]["keep"] else None
        y = binding.gcoo_spdm_epilogue(state["A"], state["X"], bias=state["bias"], activation=act, residual=state["residual"], Z_out=z)
        return (y,) if z is None else (y, z)
    if op == "epilogue":
        return binding.gcoo_epilogue_grad(state["dY"], Z=state["Z"], activation=act)
    if op == "values":
        return (binding.gcoo_spdm_grad_values(state["A"], state["dZ"], state["X"]),)
    norm = binding.gcoo_clip_grad_norm(state["grads"], state["max_norm"], out=state["out"])
    return (norm, *state["out"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    op = case["op"]
    if op == "clip":
        n, size = sum(_sizes(case)), TYPES[case["type"]].itemsize
        return dict(bytes=2.0 * n * size, flops=3.0 * n)
    size, m, N = TYPES[case["type"]].itemsize, case["m"], case["N"]
    if op == "epilogue":
        return dict(bytes=3.0 * m * N * size + 4.0 * m, flops=10.0 * m * N)
    k, nnz = case["k"], _entries(case)
    touched = k * -math.expm1(-nnz / k)          # rows of X that a stored entry touches
    if op == "forward":
        moved = 8.0 * nnz + 4.0 * (m + 1) + touched * N * size
        moved += m * N * size * (1 + case["residual"] + case["keep"]) + 4.0 * m * case["bias"]
        return dict(bytes=moved, flops=2.0 * nnz * N)
    rows = m * -math.expm1(-nnz / m)
    return dict(bytes=8.0 * nnz + 4.0 * (m + 1) + (touched + rows) * N * size, flops=2.0 * nnz * N)


# ---- the definition in 64 bits, entry by entry ----

def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "clip":
        total = math.fsum(float((x.double() * x.double()).sum()) for x in state["grads"])
        norm = math.sqrt(total)
        factor = min(1.0, state["max_norm"] / (norm + 1e-6))
        return (torch.tensor(norm, dtype=torch.float64, device=DEV), *[x.double() * factor for x in state["grads"]])
    if op == "epilogue":
        z = state["Z"].double().requires_grad_()
        dz, = torch.autograd.grad(_activate_64(case["act"], z), z, state["dY"].double())
        return dz, dz.sum(1)
    m, N = case["m"], case["N"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    _, cols, vals, rows = _csr(case, g)
    X = state["X"].double()
    step = max(1, 400000000 // N)
    if op == "values":
        dZ = state["dZ"].double()
        out = torch.empty(cols.numel(), dtype=torch.float64, device=DEV)
        for i in range(0, cols.numel(), step):
            c, r = cols[i:i + step].long(), rows[i:i + step]
            out[i:i + step] = (dZ[r] * X[c]).sum(1)
        return (out,)
    z = torch.zeros((m, N), dtype=torch.float64, device=DEV)
    for i in range(0, cols.numel(), step):
        c = cols[i:i + step].long()
        z.index_add_(0, rows[i:i + step], vals[i:i + step].double()[:, None] * X[c])
    if state["bias"] is not None:
        z += state["bias"].double()[:, None]
    y = _activate_64(case["act"], z)
    if state["residual"] is not None:
        y = y + state["residual"].double()
    return (y, z) if case["keep"] else (y,)


def _activate_64(name, z):
    """Each activation from its definition, for numbers in 64 bits."""
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z * torch.special.expit(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * torch.special.expit(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z
