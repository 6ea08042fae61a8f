"""The operators that train a routed feed-forward block, as timed cases.

A router sends each token to a few experts.  The experts' products on weights
in 16 or 32 bits, which training needs and which serve a block that is not
quantised, run on the pairs (token, slot) that each expert has, few or many;
their gradients go to the inputs, the weights and the routing weights; and the
weights' gradients are orthogonalised before they are applied.

Kinds of case:
  linear      isc_expert_linear: each pair's row times its expert's matrix,
              rectified (a block's first product), or summed over a token's
              slots under the routing weights (its second)
  linear_bwd  isc_expert_linear_bwd: the gradients of the inputs, of the
              experts' weights and, of a sum, of the routing weights
  orth        isc_orthogonalize: odd polynomials of each matrix of a stack,
              which bring its singular values towards one
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def _linear(name, T, E, k, K, N, dtype, relu=False, combine=False, shared=True, skew=0.3, empty=0.0, kind="linear"):
    return {"name": name, "kind": kind, "T": T, "E": E, "k": k, "K": K, "N": N, "dtype": dtype, "relu": relu,
            "combine": combine, "shared": shared, "skew": skew, "empty": empty}


def _orth(name, B, M, N, dtype, out="bf16", steps=5):
    return {"name": name, "kind": "orth", "B": B, "M": M, "N": N, "dtype": dtype, "out": out, "steps": steps}


def listed():
    return [
        # one token of a decoding step through the first products of its experts: the smallest call
        _linear("up_token", 1, 64, 8, 2048, 1408, "bf16", relu=True),
        # a decoding batch's second products, added up under the routing weights
        _linear("down_decode", 16, 64, 8, 1408, 2048, "bf16", combine=True, shared=False),
        # a prompt, or a training step's forward pass, through the first products
        _linear("up_prompt", 4096, 64, 8, 2048, 1408, "bf16", relu=True),
        # a batch's second products in the other 16-bit type, on experts that are loaded unevenly
        _linear("down_uneven", 2048, 64, 8, 1408, 2048, "f16", combine=True, shared=False, skew=1.0),
        # a small block in 32 bits, of odd widths, with tokens that were dropped from full experts
        _linear("up_odd", 777, 7, 2, 1155, 515, "f32", relu=True, empty=0.1),
        # the first products' gradients in a training step
        _linear("up_bwd_batch", 4096, 64, 8, 2048, 1408, "bf16", relu=True, kind="linear_bwd"),
        # the second products', with the routing weights' own
        _linear("down_bwd_batch", 2048, 64, 8, 1408, 2048, "bf16", combine=True, shared=False, kind="linear_bwd"),
        # the small block's gradients
        _linear("down_bwd_odd", 777, 7, 2, 515, 1155, "f32", combine=True, shared=False, empty=0.1, kind="linear_bwd"),
        # a router's own weights: a narrow matrix
        _orth("orth_router", 1, 2048, 64, "bf16"),
        # three matrices of odd sizes at once, gradients kept in 32 bits
        _orth("orth_odd", 3, 777, 1155, "f32"),
        # a fully connected layer behind 256 maps of 6 x 6
        _orth("orth_fc", 1, 4096, 9216, "bf16"),
        # every expert's first matrix in one call: the largest
        _orth("orth_experts", 64, 1408, 2048, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _multiple(rng, lo, hi, of):
    """An odd multiple of `of` in [lo, hi], spread over the logarithm."""
    return max(1, _log(rng, lo, hi) // of | 1) * of


def draw(rng):
    """One more case of a kind above: from one token and narrow matrices up,
    widths odd or odd multiples of 2 to 128, over the listed cases' range."""
    kind = rng.choice(("linear", "linear", "linear_bwd", "orth"))
    if kind == "orth":
        while True:
            of = rng.choice((1, 8, 32, 128))
            B, M, N = rng.choice((1, 1, 2, 5, 8)), _multiple(rng, 16, 9216, of), _multiple(rng, 16, 9216, of)
            if B * min(M, N) ** 2 * max(M, N) <= 6e10:
                break
        c = _orth("", B, M, N, rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice(("bf16", "bf16", "f16")),
                  rng.choice((1, 3, 5, 5, 6)))
    else:
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        most = 9e10 / (6 if dtype == "f32" else 1)
        while True:
            E = _log(rng, 2, 128)
            k = min(E, rng.choice((1, 2, 4, 6, 8)))
            T = _log(rng, 1, 8192)
            of = rng.choice((1, 2, 8, 32, 128))
            K, N = _multiple(rng, 33, 4096, of), _multiple(rng, 33, 4096, of)
            if T * k * K * N <= most and E * K * N <= 1.8e8:
                break
        combine = rng.random() < 0.5
        c = _linear("", T, E, k, K, N, dtype, not combine and rng.random() < 0.7, combine, rng.random() < (0.2 if combine else 0.8),
                    rng.choice((0.0, 0.3, 1.0)), rng.choice((0.0, 0.0, 0.15)), kind)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _route(case, gen):
    """(ids, weights, offsets, order) as the router gives them: each token's experts, some asked for more than
    others, their weights, and the pairs t * k + j by expert; an empty slot has id -1, weight 0 and no place."""
    T, E, k = case["T"], case["E"], case["k"]
    liked = _randn(gen, 1, E) * case["skew"]
    top = (_randn(gen, T, E) + liked).topk(k, -1)
    there = torch.rand((T, k), generator=gen, device="cuda") >= case["empty"]
    ids = top.indices.where(there, -1).int()
    weights = torch.softmax(top.values, -1).where(there, 0.0)
    key = ids.flatten().long().where(ids.flatten() >= 0, E)
    by = torch.sort(key, stable=True)
    offsets = torch.searchsorted(by.values.contiguous(), torch.arange(E + 1, device="cuda")).int()
    return ids, weights, offsets, by.indices.where(by.values < E, -1).int()


def _linear_inputs(case, seed):
    g, t = _gen(seed), DTYPES[case["dtype"]]
    T, E, k, K, N = (case[c] for c in ("T", "E", "k", "K", "N"))
    route = _route(case, g)
    x = _randn(g, T, K) if case["shared"] else _randn(g, T, k, K)
    x = torch.relu(x) if case["combine"] else x  # a second product's input is the first one's, rectified
    w = torch.empty((E, N, K), dtype=t, device="cuda")
    w.copy_(_randn(g, E, N, K) * K ** -0.5)
    return x.to(t), w, route


def _bwd_inputs(case, seed):
    """The same with the output's gradient, and the rectified output that the forward pass kept."""
    x, w, route = _linear_inputs(case, seed)
    dy = _randn(_gen(seed + 7919), *((case["T"], case["N"]) if case["combine"] else (case["T"], case["k"], case["N"])))
    y = _plain_linear(x, w, route, True, False) if case["relu"] else None
    return dy.to(x.dtype), x, w, route, y


def _gradient(case, seed):
    """Gradients as weights have them: a few strong directions, over noise in all."""
    g = _gen(seed)
    B, M, N = case["B"], case["M"], case["N"]
    r = min(32, M, N)
    strong = _randn(g, B, M, r) * torch.logspace(0, -2, r, device="cuda")
    return (1e-3 * (torch.bmm(strong, _randn(g, B, r, N)) + 0.1 * _randn(g, B, M, N))).to(DTYPES[case["dtype"]])


def prepare(case, seed):
    st = {"case": case, "own": own}
    if own:
        import paper_1704_07724_amd as isc
        st["isc"] = isc
    if case["kind"] == "orth":
        st["g"] = _gradient(case, seed)
    elif case["kind"] == "linear":
        st["x"], st["w"], st["route"] = _linear_inputs(case, seed)
    else:
        st["dy"], st["x"], st["w"], st["route"], st["y"] = _bwd_inputs(case, seed)
    return st


# --------------------------------------------------------------------- run --

def run(st):
    return _own(st) if st["own"] else _plain(st)


def _own(st):
    isc, case = st["isc"], st["case"]
    if case["kind"] == "orth":
        return isc.isc_orthogonalize(st["g"], steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS,
                                     dtype=DTYPES[case["out"]])
    if case["kind"] == "linear":
        return isc.isc_expert_linear(st["x"], st["w"], st["route"], relu=case["relu"], combine=case["combine"])
    g = isc.isc_expert_linear_bwd(st["dy"], st["x"], st["w"], st["route"], y=st["y"], combine=case["combine"])
    return _gradients(g.dx, g.dw, g.dweights)


def _gradients(dx, dw, dweights):
    out = {"dx": dx, "dw": dw, "dweights": dweights}
    return {k: v for k, v in out.items() if v is not None}


def _plain(st):
    case = st["case"]
    if case["kind"] == "orth":
        return _plain_orth(st["g"], case)
    if case["kind"] == "linear":
        return _plain_linear(st["x"], st["w"], st["route"], case["relu"], case["combine"])
    return _plain_bwd(st["dy"], st["x"], st["w"], st["route"], st["y"], case["combine"])


def _by_expert(route):
    """[E, C] of each expert's pairs, C the most that one has; T * k where there is none."""
    ids, _, offsets, order = route
    offsets, P = offsets.long(), ids.numel()
    counts = offsets[1:] - offsets[:-1]
    at = torch.arange(max(1, int(counts.max())), device=ids.device)[None]
    pairs = order.long()[(offsets[:-1, None] + at).clamp(max=P - 1)]
    return pairs.where(at < counts[:, None], P)


def _rows(x, k):
    """x's row of every pair in 32 bits, and a row of zeros behind the last."""
    x = x.float()
    x = x[:, None, :].expand(-1, k, -1) if x.dim() == 2 else x
    x = x.reshape(-1, x.shape[-1])
    return torch.cat((x, x.new_zeros(1, x.shape[1])))


def _scatter(v, pairs, P):
    """[P, .] of [E, C, .] by expert; a pair without an expert has zeros."""
    out = v.new_zeros(P + 1, v.shape[-1])
    out[pairs] = v
    out[P] = 0.0
    return out[:P]


def _products(x, w, pairs, few):
    """Every pair's row of x times its expert's matrix [E, N, K], for rows x [P + 1, K]: [P, N]."""
    P = len(x) - 1
    if few is not None:
        y = torch.bmm(w[few.clamp_min(0)].float(), x[:P, :, None].contiguous())[..., 0]
        return y.where((few >= 0)[:, None], 0.0)
    return _scatter(torch.bmm(x[pairs], w.float().transpose(1, 2).contiguous()), pairs, P)


def _plain_linear(x, w, route, relu, combine):
    ids, weights = route[:2]
    T, k = ids.shape
    few = ids.flatten().long() if T * k <= 16 else None  # so few pairs that not every expert's weights are read
    y = _products(_rows(x, k), w, None if few is not None else _by_expert(route), few).view(T, k, -1)
    y = torch.relu(y) if relu else y
    y = (y * weights[..., None]).sum(1) if combine else y
    return y.to(x.dtype)


def _plain_bwd(dy, x, w, route, y, combine):
    ids, weights = route[:2]
    T, k = ids.shape
    P = T * k
    pairs = _by_expert(route)
    xs = _rows(x, k)[pairs]
    d = dy.float()
    d = d.where(y > 0, 0.0) if y is not None else d
    ds = _rows(d, k)[pairs]
    back = torch.bmm(ds, w.float())  # the gradient of a pair's row before the routing weight
    scale = None
    dweights = None
    if combine:
        dweights = _scatter((back * xs).sum(-1, keepdim=True), pairs, P).view(T, k)
        scale = torch.cat((weights.flatten(), weights.new_zeros(1)))[pairs][..., None]
        back, ds = back * scale, ds * scale
    dw = torch.bmm(ds.transpose(1, 2).contiguous(), xs)
    dx = _scatter(back, pairs, P).view(T, k, -1)
    dx = dx.sum(1) if x.dim() == 2 else dx
    return _gradients(dx.to(x.dtype), dw.to(w.dtype), dweights)


def _plain_orth(g, case):
    a, b, c = COEFFICIENTS
    x = g.float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(case["steps"]):
        s = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * s + c * torch.bmm(s, s), x)
    x = x.transpose(1, 2) if tall else x
    return x.to(DTYPES[case["out"]]).contiguous()


# -------------------------------------------------------------- work, exact --

def work(case):
    """Each input read once and each output written once; of the weights those
    of experts that a batch meets (expected: a token's experts are drawn alike);
    multiplications and additions of the products, a symmetric one's half."""
    if case["kind"] == "orth":
        B, M, N = case["B"], case["M"], case["N"]
        m, n = float(min(M, N)), float(max(M, N))
        return {"bytes": B * m * n * (BYTES[case["dtype"]] + BYTES[case["out"]]),
                "flops": B * case["steps"] * (m * m * n + m * m * m + 2.0 * m * m * n)}
    T, E, k, K, N = (case[c] for c in ("T", "E", "k", "K", "N"))
    b = BYTES[case["dtype"]]
    pairs = T * k * (1.0 - case["empty"])
    met = E * (1.0 - (1.0 - k / E * (1.0 - case["empty"])) ** T)
    x = (T if case["shared"] else T * k) * K * b
    y = (T if case["combine"] else T * k) * N * b
    lists = 4.0 * (T * k * (3 if case["combine"] else 2) + E)
    if case["kind"] == "linear":
        return {"bytes": x + y + met * N * K * b + lists, "flops": 2.0 * pairs * N * K}
    # dy, x and the weights read, the rectified output too; dx, every weight's gradient, the routing weights' written
    return {"bytes": 2.0 * x + y * (2 if case["relu"] else 1) + (met + E) * N * K * b + lists,
            "flops": 4.0 * pairs * N * K}


def _exact_linear(x, w, route, relu, combine):
    ids, weights = route[0].long(), route[1].double()
    out = torch.zeros((*ids.shape, w.shape[1]), dtype=torch.float64, device=x.device)
    for e in range(w.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if len(t):
            out[t, j] = (x[t] if x.dim() == 2 else x[t, j]).double() @ w[e].double().t().contiguous()
    out = out.clamp_min(0.0) if relu else out
    return (out * weights[..., None]).sum(1) if combine else out


def _exact_bwd(dy, x, w, route, y, combine):
    ids, weights = route[0].long(), route[1].double()
    T, k = ids.shape
    dx = torch.zeros((T, k, w.shape[2]), dtype=torch.float64, device=x.device)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=x.device)
    dweights = torch.zeros((T, k), dtype=torch.float64, device=x.device)
    for e in range(w.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not len(t):
            continue
        xe, we = (x[t] if x.dim() == 2 else x[t, j]).double(), w[e].double()
        if combine:
            de = dy[t].double()
            dweights[t, j] = (de * (xe @ we.t().contiguous())).sum(-1)
            de = de * weights[t, j][:, None]
        else:
            de = dy[t, j].double()
            de = de * (y[t, j] > 0) if y is not None else de
        dx[t, j] = de @ we
        dw[e] = de.t().contiguous() @ xe
    return _gradients(dx.sum(1) if x.dim() == 2 else dx, dw, dweights if combine else None)


def _exact_orth(g, steps):
    """Each matrix by itself, in its own orientation: x (a + b s + c s^2) with s = x^T x, or from the left."""
    a, b, c = COEFFICIENTS
    out = []
    for x in g.double():
        x = x / (torch.sqrt((x * x).sum()) + EPS)
        wide = x.shape[0] <= x.shape[1]
        for _ in range(steps):
            xt = x.t().contiguous()
            s = x @ xt if wide else xt @ x
            p = c * (s @ s) + b * s
            p.diagonal().add_(a)
            x = p @ x if wide else x @ p
        out.append(x)
    return torch.stack(out)


def exact(case, seed):
    if case["kind"] == "orth":
        return _exact_orth(_gradient(case, seed), case["steps"])
    if case["kind"] == "linear":
        x, w, route = _linear_inputs(case, seed)
        return _exact_linear(x, w, route, case["relu"], case["combine"])
    return _exact_bwd(*_bwd_inputs(case, seed), case["combine"])
