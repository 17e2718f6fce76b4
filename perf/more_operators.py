"""Performance cases of the operators of a gated residual branch: the gated unit and the gated recurrence along a line.

A case is a dict of plain values.  Four kinds of work, each one call of ``binding``:

  gated_fwd    y = fn(u) v with u = W x + b and v = V x + c, W and V stacked as the 2 f' rows of one matrix; ``kept`` says
               whether u and v are kept for the backward pass (training) or not (prediction)
  gated_bwd    its Jacobian with the gradients of weights and biases, from the kept u and v
  lines_fwd    h_t = f_t h_(t-1) + (1 - f_t) x_t with f = logistic(z), along one dimension of an array
  lines_bwd    its Jacobian: the gradients of z, of x and of the state before the first step

Operands are dense arrays in 32 bits.  The gated unit takes images [map][z][y][x] (``maps`` layout: every voxel's maps are
its features, axis 0) or rows of features (``rows`` layout, axis 1).  Lines run along any dimension of images, or along the
middle one of [batch][step][feature].
"""
import math

import torch

own = False

DEV = "cuda:0"
FNS = ["rectify", "logistic", "tanh", "silu", "gelu"]


# ------------------------------------------------------------------------------------------ descriptions
def _gated_images(kind, f, fo, n, fn, **more):
    return dict(kind=kind, layout="maps", f=f, fo=fo, nz=n[0], ny=n[1], nx=n[2], fn=fn, **more)


def _gated_rows(kind, rows, f, fo, fn, **more):
    return dict(kind=kind, layout="rows", rows=rows, f=f, fo=fo, fn=fn, **more)


def _lines(kind, shape, dim, reverse=False, state=False, packed=False, **more):
    """``state``: a state before the first step is given; ``packed``: lines hold several sequences, each begun by a gate that is shut."""
    case = dict(kind=kind, dims=len(shape), dim=dim, reverse=reverse, state=state, packed=packed, **more)
    case.update({"n%d" % i: n for i, n in enumerate(shape)})
    return case


def listed():
    return [
        # One voxel, or one row, in prediction: every weight is read for a single product.
        _gated_rows("gated_fwd", 1, 1024, 4096, "silu", kept=False, name="gated_single_row"),
        # The maps of a 12^3 output patch of a 3D net, in training: one launch on little data, where latency counts.
        _gated_images("gated_fwd", 40, 80, (12, 12, 12), "logistic", kept=True, name="gated_patch"),
        # Training on rows of features, no number round.
        _gated_rows("gated_fwd", 4099, 1001, 2601, "gelu", kept=True, name="gated_rows"),
        # Prediction for the largest images a single GPU is used for.
        _gated_images("gated_fwd", 120, 240, (96, 96, 96), "silu", kept=False, name="gated_widest"),
        # Backward through the branch of a wide 3D layer cut at no round size.
        _gated_images("gated_bwd", 40, 80, (61, 58, 63), "tanh", name="gated_back_maps"),
        # Backward on many rows of many features: what training a wide branch spends its time on.
        _gated_rows("gated_bwd", 8192, 1024, 4096, "silu", name="gated_back_rows"),
        # One step of eight sequences from the state that the step before left: the shortest call there is.
        _lines("lines_fwd", (8, 1, 1024), 1, state=True, name="lines_step"),
        # Along the rows of images, as a net looks at its context line by line.
        _lines("lines_fwd", (40, 60, 60, 60), 3, name="lines_images"),
        # One long sequence of features.
        _lines("lines_fwd", (1, 65536, 512), 1, state=True, name="lines_long"),
        # Backward of the other direction, along the slowest axis of the largest images.
        _lines("lines_bwd", (120, 96, 96, 96), 1, reverse=True, name="lines_back_widest"),
        # Backward on sequences of different lengths in three lines, no number round.
        _lines("lines_bwd", (3, 5003, 1001), 1, state=True, packed=True, name="lines_back_packed"),
        # Backward of a few very long lines: what little runs beside one another has to come from the lines themselves.
        _lines("lines_bwd", (4, 1000003), 1, name="lines_back_signal"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extents(rng):
    if rng.random() < 0.3:
        return 1, _log_int(rng, 24, 320), _log_int(rng, 24, 320)
    e = _log_int(rng, 8, 100)
    return tuple(_log_int(rng, max(6, e // 2), 2 * e) for _ in range(3))


def draw(rng):
    """One more case of the same ranges: from one row, one step or a patch to the largest ones, odd extents as likely as even ones."""
    cases = listed()
    while True:
        kind = rng.choice(["gated_fwd", "gated_bwd", "lines_fwd", "lines_bwd"])
        if kind.startswith("gated"):
            more = {"kept": rng.random() < 0.6} if kind == "gated_fwd" else {}
            fn = rng.choice(FNS)
            if rng.random() < 0.5:
                f = _log_int(rng, 3, 160)
                case = _gated_images(kind, f, _log_int(rng, max(3, f // 2), 4 * f), _extents(rng), fn, **more)
            else:
                f = _log_int(rng, 24, 2048)
                case = _gated_rows(kind, _log_int(rng, 1, 20000), f, _log_int(rng, f, 4 * f), fn, **more)
        else:
            form = rng.choice(["images", "features", "signal"])
            if form == "images":
                shape, dim = (_log_int(rng, 3, 160),) + _extents(rng), rng.choice([1, 2, 3])
            elif form == "features":
                shape, dim = (_log_int(rng, 1, 16), _log_int(rng, 1, 70000), _log_int(rng, 24, 4096)), 1
            else:
                shape, dim = (_log_int(rng, 1, 64), _log_int(rng, 1000, 1100000)), 1
            case = _lines(kind, shape, dim, rng.random() < 0.4, rng.random() < 0.5, rng.random() < 0.3)
        cost = work(case)
        alike = [work(c) for c in cases if c["kind"][:5] == kind[:5]]
        if all(cost[k] <= max(w[k] for w in alike) for k in cost):
            return case


# ---------------------------------------------------------------------------------------------- inputs
def _positions(case):
    return (case["rows"],) if case["layout"] == "rows" else (case["nz"], case["ny"], case["nx"])


def _gated_shape(case, features):
    return _positions(case) + (features,) if case["layout"] == "rows" else (features,) + _positions(case)


def _axis(case):
    return 1 if case["layout"] == "rows" else 0


def _lines_shape(case):
    return tuple(case["n%d" % i] for i in range(case["dims"]))


def _before(w, x, b, axis):
    """W x + b over the features of every position, [2 f'] of them."""
    if axis == 1:
        return x @ w.t() + b
    return (w @ x.reshape(x.shape[0], -1) + b[:, None]).reshape((w.shape[0],) + x.shape[1:])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(size, scale=1.0):
        return torch.randn(size, generator=gen, device=DEV) * scale

    s = {"case": case}
    if case["kind"].startswith("gated"):
        f, fo, axis = case["f"], case["fo"], _axis(case)
        # what a norm with its own weight and bias leaves, a few features large; a corner of every image (some rows) without a signal
        along = (f,) + (1,) * len(_positions(case)) if axis == 0 else (f,)
        x = normal(_gated_shape(case, f)) * (1 + normal(along, 0.2)) + normal(along, 0.1)
        x *= (torch.rand(along, generator=gen, device=DEV) < 0.02).float() * 4 + 1
        if axis == 0:
            x[..., :1, :2] = 0
        else:
            x[96::97] = 0
        s["x"], s["w"], s["b"] = x, normal((2 * fo, f), f ** -0.5), normal((2 * fo,), 0.1)
        if case["kind"] == "gated_bwd":
            s["kept"] = _before(s["w"], x, s["b"], axis)
            s["gy"] = normal(_gated_shape(case, fo), 1e-2)
        return s
    shape, dim = _lines_shape(case), case["dim"]
    # gates that remember a few steps to some hundreds, each feature (or map) around its own number
    along = [1] * len(shape)
    along[0 if len(shape) == 4 or dim == len(shape) - 1 else -1] = -1
    own_gate = normal((shape[0] if along[0] == -1 else shape[-1],), 1.5).view(along)
    s["z"] = normal(shape) + own_gate + 2
    s["x"] = normal(shape)
    if case["packed"]:
        # a gate of minus infinity forgets everything: a new sequence begins
        steps = [1] * len(shape)
        steps[dim] = shape[dim]
        begins = torch.rand(steps, generator=gen, device=DEV) < 4 / shape[dim]
        s["z"] = torch.where(begins, torch.full_like(s["z"], -math.inf), s["z"])
    if case["state"]:
        s["h0"] = normal(shape[:dim] + shape[dim + 1:])
    if case["kind"] == "lines_bwd":
        s["h"] = _lines_fwd(s["z"], s["x"], s.get("h0"), dim, case["reverse"])
        s["gh"] = normal(shape, 1e-2)
    return s


# ---------------------------------------------------------------------------------- the plain operators
def _fn(u, fn):
    """(fn(u), its derivative)"""
    if fn == "rectify":
        return torch.where(u > 0, u, torch.zeros_like(u)), (u > 0).to(u.dtype)
    if fn == "tanh":
        t = torch.tanh(u)
        return t, 1 - t * t
    if fn == "gelu":
        p = 0.5 * torch.erfc(u * -0.5 ** 0.5)
        return u * p, p + u * torch.exp(-0.5 * u * u) * (2 * math.pi) ** -0.5
    s, t = 1 / (1 + torch.exp(-u)), 1 / (1 + torch.exp(u))
    return (s, s * t) if fn == "logistic" else (u * s, s + u * s * t)


def _gated_back(gy, x, w, kept, fn, axis):
    """(gx, gw, gb)"""
    u, v = kept.chunk(2, axis)
    a, d = _fn(u, fn)
    g = torch.cat([gy * v * d, gy * a], axis)
    if axis == 1:
        return g @ w, g.t() @ x, g.sum(0)
    g, m = g.reshape(g.shape[0], -1), x.reshape(x.shape[0], -1)
    return (w.t() @ g).reshape(x.shape), g @ m.t(), g.sum(1)


def _scan(a, b):
    """y_t = a_t y_(t-1) + b_t along the middle dimension: every step of the loop joins twice as many terms."""
    d = 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _as_lines(t, dim, reverse):
    """[outer][step][inner] with the steps in the order they are taken"""
    t = t.reshape(math.prod(t.shape[:dim]), t.shape[dim], -1)
    return t.flip(1) if reverse else t


def _lines_fwd(z, x, h0, dim, reverse):
    zl, xl = _as_lines(z, dim, reverse), _as_lines(x, dim, reverse)
    f = 1 / (1 + torch.exp(-zl))
    b = 1 / (1 + torch.exp(zl)) * xl
    if h0 is not None:
        b[:, 0] += f[:, 0] * h0.reshape(b[:, 0].shape)
    h = _scan(f, b)
    return (h.flip(1) if reverse else h).reshape(z.shape)


def _lines_bwd(gh, z, x, h, h0, dim, reverse):
    gl, zl, xl, hl = (_as_lines(t, dim, reverse) for t in (gh, z, x, h))
    f, k = 1 / (1 + torch.exp(-zl)), 1 / (1 + torch.exp(zl))
    first = torch.zeros_like(hl[:, :1]) if h0 is None else h0.reshape(hl[:, :1].shape)
    before = torch.cat([first, hl[:, :-1]], 1)
    after = torch.cat([f[:, 1:], torch.zeros_like(f[:, :1])], 1)
    g = _scan(after.flip(1), gl.flip(1)).flip(1)
    gz, gx = g * (before - xl) * (f * k), g * k
    out = {n: (t.flip(1) if reverse else t).reshape(z.shape) for n, t in (("gz", gz), ("gx", gx))}
    if h0 is not None:
        out["gh0"] = (f[:, 0] * g[:, 0]).reshape(h0.shape)
    return out


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "gated_fwd":
        kept = _before(s["w"], s["x"], s["b"], _axis(case))
        u, v = kept.chunk(2, _axis(case))
        y = _fn(u, case["fn"])[0] * v
        return {"y": y, "kept": kept} if case["kept"] else {"y": y}
    if kind == "gated_bwd":
        gx, gw, gb = _gated_back(s["gy"], s["x"], s["w"], s["kept"], case["fn"], _axis(case))
        return {"gx": gx, "gw": gw, "gb": gb}
    if kind == "lines_fwd":
        return {"h": _lines_fwd(s["z"], s["x"], s.get("h0"), case["dim"], case["reverse"])}
    return _lines_bwd(s["gh"], s["z"], s["x"], s["h"], s.get("h0"), case["dim"], case["reverse"])


def run(s):
    if not own:
        return _plain(s)
    from paper_1510_06706_amd import binding as znn
    case = s["case"]
    kind = case["kind"]
    if kind == "gated_fwd":
        y, kept = znn.gated_fwd(s["x"], s["w"], s["b"], case["fn"], _axis(case), case["kept"])
        return {"y": y, "kept": kept} if case["kept"] else {"y": y}
    if kind == "gated_bwd":
        gx, gw, gb = znn.gated_bwd(s["gy"], s["x"], s["w"], s["kept"], case["fn"], _axis(case))
        return {"gx": gx, "gw": gw, "gb": gb}
    if kind == "lines_fwd":
        return {"h": znn.recurrence_fwd(s["z"], s["x"], s.get("h0"), case["dim"], case["reverse"])}
    gz, gx, gh0 = znn.recurrence_bwd(s["gh"], s["z"], s["x"], s["h"], s.get("h0"), case["dim"], case["reverse"])
    return {"gz": gz, "gx": gx, "gh0": gh0} if case["state"] else {"gz": gz, "gx": gx}


# ------------------------------------------------------------------------------------------ definitions
def exact(case, seed):
    """The definitions in 64 bits: features as the rows of a matrix; a recurrence step by step, blocks of a long line beside each
    other and then joined."""
    s = prepare(case, seed)
    if case["kind"].startswith("gated"):
        axis, fo = _axis(case), case["fo"]

        def matrix(t):
            return (t.t() if axis == 1 else t.reshape(t.shape[0], -1)).double()

        def back(m):
            return m.t() if axis == 1 else m.reshape((m.shape[0],) + _positions(case))

        x, w = matrix(s["x"]), s["w"].double()
        both = matrix(s["kept"]) if "kept" in s else torch.addmm(s["b"].double()[:, None], w, x)
        u, v = both[:fo], both[fo:]
        fn = case["fn"]
        if fn == "rectify":
            a, d = u.clamp(min=0), (u > 0).double()
        elif fn == "tanh":
            a, d = u.tanh(), u.cosh() ** -2
        elif fn == "logistic":
            a, d = u.sigmoid(), u.sigmoid() * (-u).sigmoid()
        elif fn == "silu":
            a, d = u * u.sigmoid(), u.sigmoid() * (1 + u * (-u).sigmoid())
        else:
            phi = torch.special.ndtr(u)
            a, d = u * phi, phi + u * (-u * u / 2).exp() / math.sqrt(2 * math.pi)
        if case["kind"] == "gated_fwd":
            return {"y": back(a * v), "kept": back(both)} if case["kept"] else {"y": back(a * v)}
        g = matrix(s["gy"])
        gu, gv = g * v * d, g * a
        return {"gx": back(w[:fo].t() @ gu + w[fo:].t() @ gv), "gw": torch.cat([gu @ x.t(), gv @ x.t()]),
                "gb": torch.cat([gu.sum(1), gv.sum(1)])}

    dim, reverse, length = case["dim"], case["reverse"], s["z"].shape[case["dim"]]

    def steps(t):
        # [step][line] in the order of the steps
        t = t.double().movedim(dim, 0)
        return (t.flip(0) if reverse else t).reshape(length, -1)

    def back(t):
        t = t.reshape((length,) + s["z"].shape[:dim] + s["z"].shape[dim + 1:])
        return (t.flip(0) if reverse else t).movedim(0, dim)

    def recur(a, b, state):
        # y_t = a_t y_(t-1) + b_t
        n, lines = a.shape
        block = n if n <= 512 else math.isqrt(n)
        blocks = -(-n // block)
        if blocks * block != n:
            a = torch.cat([a, torch.ones((blocks * block - n, lines), dtype=a.dtype, device=DEV)])
            b = torch.cat([b, torch.zeros((blocks * block - n, lines), dtype=a.dtype, device=DEV)])
        a, y = a.reshape(blocks, block, lines).clone(), b.reshape(blocks, block, lines).clone()
        for t in range(1, block):       # within every block from a state of zero, and what a state before it is multiplied by
            y[:, t] += a[:, t] * y[:, t - 1]
            a[:, t] *= a[:, t - 1]
        states = torch.empty((blocks, lines), dtype=a.dtype, device=DEV)
        for k in range(blocks):
            states[k] = state
            state = y[k, -1] + a[k, -1] * state
        return (y + a * states[:, None]).reshape(blocks * block, lines)[:n]

    z, x = steps(s["z"]), steps(s["x"])
    f, k = torch.sigmoid(z), torch.sigmoid(-z)
    h0 = s["h0"].double().reshape(-1) if case["state"] else torch.zeros(z.shape[1], dtype=torch.float64, device=DEV)
    if case["kind"] == "lines_fwd":
        return {"h": back(recur(f, k * x, h0))}
    g = steps(s["gh"]).flip(0)
    a = torch.cat([torch.zeros_like(f[:1]), f[1:].flip(0)])
    g = recur(a, g, torch.zeros_like(h0)).flip(0)
    before = torch.cat([h0[None], steps(s["h"])[:-1]])
    out = {"gz": back(g * (before - x) * f * k), "gx": back(g * k)}
    if case["state"]:
        out["gh0"] = (f[0] * g[0]).reshape(s["h0"].shape)
    return out


def work(case):
    """Bytes: every operand read once, every result written once.  FLOPs: two per product and sum of the matrix products, and those on
    every element of the recurrence without its exponential."""
    kind = case["kind"]
    if kind.startswith("gated"):
        f, fo, n = case["f"], case["fo"], math.prod(_positions(case))
        weights = 2 * fo * f + 2 * fo
        if kind == "gated_fwd":
            values = f * n + weights + fo * n * (3 if case["kept"] else 1)
            return {"bytes": 4.0 * values, "flops": 4.0 * f * fo * n}
        return {"bytes": 4.0 * (2 * f * n + 3 * fo * n + 2 * weights - 2 * fo), "flops": 8.0 * f * fo * n}
    shape = _lines_shape(case)
    elements = math.prod(shape)
    lines = elements // shape[case["dim"]] if case["state"] else 0
    if kind == "lines_fwd":
        return {"bytes": 4.0 * (3 * elements + lines), "flops": 5.0 * elements}
    return {"bytes": 4.0 * (6 * elements + 2 * lines), "flops": 9.0 * elements}
