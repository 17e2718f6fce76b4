"""Performance cases of the normalisation and regularisation operators: dropout, layer norm and the residual join.

A case is a dict of plain values.  Five kinds of work, each one call of ``binding``:

  dropout   y = x / (1 - p) where an element is kept, 0 elsewhere; its Jacobian is the same call on a gradient
  norm_fwd  layer norm; ``stats`` says whether mean and 1 / deviation are kept (training) or not (prediction)
  norm_bwd  its Jacobian with the gradients of weight and bias, from the kept statistics
  join_fwd  the end of a residual branch: r = x + dropout(h), y = layer norm of r
  join_bwd  its Jacobian: the gradients of x and of h, of weight and bias; ``gr`` says whether r is used behind the
            norm too, so that a gradient arrives there as well

Operands are dense [rows][cols] arrays in 32 bits.  ``maps`` layout: images [map][z][y][x], every voxel normalised
over the maps (axis 0).  ``rows`` layout: rows of features, each normalised by itself (axis 1).
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5


# ------------------------------------------------------------------------------------------ descriptions
def _images(kind, maps, n, **more):
    return dict(kind=kind, layout="maps", maps=maps, nz=n[0], ny=n[1], nx=n[2], **more)


def _rows(kind, rows, features, **more):
    return dict(kind=kind, layout="rows", rows=rows, features=features, **more)


def listed():
    return [
        # Dropout on a node of the six-layer 3D net at its 12^3 output patch: one launch on little data, where latency counts.
        _images("dropout", 40, (12, 12, 12), p=0.5, name="dropout_patch"),
        # On the gradient of an anisotropic layer cut at no round size: maps of an odd number of voxels.
        _images("dropout", 36, (21, 71, 57), p=0.2, name="dropout_ragged"),
        # On the result of the widest layer a single GPU is used for.
        _images("dropout", 120, (90, 90, 90), p=0.1, name="dropout_widest"),
        # The norm on the same small node, in training.
        _images("norm_fwd", 40, (12, 12, 12), stats=True, name="norm_patch"),
        # One row of features in prediction: the shortest call there is.
        _rows("norm_fwd", 1, 1024, stats=False, name="norm_single_row"),
        # Training on the largest images.
        _images("norm_fwd", 120, (96, 96, 96), stats=True, name="norm_widest"),
        # Backward on the result of a wide 3D layer.
        _images("norm_bwd", 40, (60, 60, 60), name="norm_back_wide"),
        # Backward on rows of features, neither number round.
        _rows("norm_bwd", 5003, 1001, name="norm_back_rows"),
        # A residual branch of a wide 2D layer, in training.
        _images("join_fwd", 80, (1, 246, 246), p=0.1, stats=True, name="join_2d"),
        # Prediction for a few rows of many features: nothing is dropped, nothing kept.
        _rows("join_fwd", 16, 4096, p=0.0, stats=False, name="join_few_rows"),
        # Backward through a branch over many short rows, whose sum is also passed on.
        _rows("join_bwd", 16384, 512, p=0.1, gr=True, name="join_back_rows"),
        # Backward through a branch on the largest images.
        _images("join_bwd", 120, (96, 96, 96), p=0.1, gr=True, name="join_back_widest"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: from one row or a patch to the largest images, odd extents as likely as even ones."""
    largest = work(listed()[-1])["bytes"]
    while True:
        kind = rng.choice(["dropout", "norm_fwd", "norm_bwd", "join_fwd", "join_bwd"])
        more = {}
        if kind in ("dropout", "join_fwd", "join_bwd"):
            more["p"] = rng.choice([0.05, 0.1, 0.25, 0.5])
        if kind in ("join_fwd", "join_bwd") and rng.random() < 0.25:
            more["p"] = 0.0
        if kind in ("norm_fwd", "join_fwd"):
            more["stats"] = rng.random() < 0.7
        if kind == "join_bwd":
            more["gr"] = rng.random() < 0.7
        if rng.random() < 0.6:
            e = _log_int(rng, 10, 110)
            if rng.random() < 0.3:
                n = (1, _log_int(rng, 24, 320), _log_int(rng, 24, 320))
            else:
                n = (e, e, e) if rng.random() < 0.4 else tuple(_log_int(rng, max(6, e // 2), 2 * e) for _ in range(3))
            case = _images(kind, _log_int(rng, 3, 240), n, **more)
        else:
            case = _rows(kind, _log_int(rng, 1, 60000), _log_int(rng, 24, 16384), **more)
        if work(case)["bytes"] <= largest:
            return case


# ---------------------------------------------------------------------------------------------- inputs
def _shape(case):
    if case["layout"] == "rows":
        return case["rows"], case["features"]
    return case["maps"], case["nz"], case["ny"], case["nx"]


def _axis(case):
    return 1 if case["layout"] == "rows" else 0


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    shape, axis = _shape(case), _axis(case)
    features = shape[axis]
    along = (features,) + (1,) * (len(shape) - 1) if axis == 0 else (features,)

    def normal(size, scale=1.0):
        return torch.randn(size, generator=gen, device=DEV) * scale

    def image():
        # features of their own scale and offset, a few of them large; a corner of every image (some rows) without a signal
        spread = torch.exp(normal(along, 0.5))
        offset = normal(along, 0.5)
        large = (torch.rand(along, generator=gen, device=DEV) < 0.02).float() * 6 + 1
        x = normal(shape) * spread + offset
        x *= large
        if axis == 0:
            x[..., :1, :2] = 0
        else:
            x[96::97] = 0
        return x

    kind = case["kind"]
    state = {"case": case}
    if case.get("p", 0.0) > 0.0:
        # what the generator goes by: a seed and the number of the round, on the device
        state["random"] = torch.randint(0, 2 ** 62, (2,), generator=gen, device=DEV, dtype=torch.int64)
        state["site"] = 3
    if kind == "dropout":
        state["x"] = normal(shape)
        return state
    state["w"] = 1 + normal((features,), 0.1)
    if kind in ("norm_fwd", "join_fwd"):
        state["b"] = normal((features,), 0.1)
    state["x"] = image()
    if kind == "join_fwd":
        state["h"] = normal(shape, 0.5)
    if kind in ("norm_bwd", "join_bwd"):
        x = state["x"]
        mean = x.mean(axis, dtype=torch.float64)
        deviation = (x - mean.unsqueeze(axis).float()).square().mean(axis, dtype=torch.float64).add(EPS).sqrt()
        state["stats"] = torch.stack([mean.reshape(-1), 1 / deviation.reshape(-1)]).float()
        state["gy"] = normal(shape, 1e-2)
        if case.get("gr"):
            state["gr"] = normal(shape, 1e-2)
    return state


# ---------------------------------------------------------------------------------- the plain operators
def _words(rows, cols, random, site):
    """Words of Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) for a dense array: key the
    seed, counter (column / 4, row, site, round), one word per element; as numbers below 2^32 in 64 bits."""
    low = 0xFFFFFFFF
    quads = (cols + 3) // 4
    c0 = torch.arange(quads, device=DEV).expand(rows, quads)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, quads)
    c2 = torch.full((1, 1), site, device=DEV, dtype=torch.int64)
    c3 = (random[1] & low).reshape(1, 1)
    k0, k1 = random[0] & low, random[0] >> 32 & low
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57       # modulo 2^64
        c0, c1, c2, c3 = p1 >> 32 & low ^ c1 ^ k0, p1 & low, p0 >> 32 & low ^ c3 ^ k1, p0 & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), -1)
    return words.reshape(rows, 4 * quads)[:, :cols]


def _dropped(x, p, random, site):
    if p == 0.0:
        return x
    keep = 2 ** 32 - math.floor(p * 2 ** 32 + 0.5)
    kept = _words(x.shape[0], x.numel() // x.shape[0], random, site) < keep
    return torch.where(kept.reshape(x.shape), x * (2 ** 32 / keep), torch.zeros_like(x))


def _norm(x, w, b, axis):
    """(y, mean, 1 / deviation) in 32 bits."""
    n = x.shape[axis]
    along = (n,) + (1,) * (x.dim() - 1) if axis == 0 else (n,)
    mean = x.sum(axis, keepdim=True) / n
    d = x - mean
    inverse = 1 / ((d * d).sum(axis, keepdim=True) / n + EPS).sqrt()
    return d * inverse * w.view(along) + b.view(along), torch.stack([mean.reshape(-1), inverse.reshape(-1)])


def _norm_back(gy, x, w, stats, axis):
    """(gx, gw, gb) in 32 bits."""
    n = x.shape[axis]
    along = (n,) + (1,) * (x.dim() - 1) if axis == 0 else (n,)
    kept = tuple(1 if a == axis else e for a, e in enumerate(x.shape))
    mean, inverse = stats[0].view(kept), stats[1].view(kept)
    h = (x - mean) * inverse
    a = gy * w.view(along)
    gx = inverse * (a - a.sum(axis, keepdim=True) / n - h * ((a * h).sum(axis, keepdim=True) / n))
    others = [i for i in range(x.dim()) if i != axis]
    return gx, (gy * h).sum(others), gy.sum(others)


def _plain(s):
    case, axis = s["case"], _axis(s["case"])
    p, random, site = case.get("p", 0.0), s.get("random"), s.get("site")
    kind = case["kind"]
    if kind == "dropout":
        return {"y": _dropped(s["x"], p, random, site)}
    if kind == "norm_fwd":
        y, stats = _norm(s["x"], s["w"], s["b"], axis)
        return {"y": y, "stats": stats} if case["stats"] else {"y": y}
    if kind == "norm_bwd":
        gx, gw, gb = _norm_back(s["gy"], s["x"], s["w"], s["stats"], axis)
        return {"gx": gx, "gw": gw, "gb": gb}
    if kind == "join_fwd":
        r = s["x"] + _dropped(s["h"], p, random, site)
        y, stats = _norm(r, s["w"], s["b"], axis)
        return {"r": r, "y": y, "stats": stats} if case["stats"] else {"r": r, "y": y}
    gx, gw, gb = _norm_back(s["gy"], s["x"], s["w"], s["stats"], axis)
    if case["gr"]:
        gx = gx + s["gr"]
    out = {"gx": gx, "gw": gw, "gb": gb}
    if p > 0.0:
        out["gh"] = _dropped(gx, p, random, site)
    return out


def run(s):
    if not own:
        return _plain(s)
    from paper_1510_06706_amd import binding as znn
    case, axis = s["case"], _axis(s["case"])
    p, random, site = case.get("p", 0.0), s.get("random"), s.get("site", 0)
    kind = case["kind"]
    if kind == "dropout":
        return {"y": znn.dropout(s["x"], p, random, site)}
    if kind == "norm_fwd":
        y, stats = znn.layernorm_fwd(s["x"], s["w"], s["b"], EPS, axis, case["stats"])
        return {"y": y, "stats": stats} if case["stats"] else {"y": y}
    if kind == "norm_bwd":
        gx, gw, gb = znn.layernorm_bwd(s["gy"], s["x"], s["w"], s["stats"], axis)
        return {"gx": gx, "gw": gw, "gb": gb}
    if kind == "join_fwd":
        r, y, stats = znn.residual_norm_fwd(s["h"], s["x"], s["w"], s["b"], p, random, site, EPS, axis, case["stats"])
        return {"r": r, "y": y, "stats": stats} if case["stats"] else {"r": r, "y": y}
    gx, gh, gw, gb = znn.residual_norm_bwd(s["gy"], s.get("gr"), s["x"], s["w"], s["stats"], p, random, site, axis)
    out = {"gx": gx, "gw": gw, "gb": gb}
    if p > 0.0:
        out["gh"] = gh
    return out


# ------------------------------------------------------------------------------------------ definitions
def exact(case, seed):
    """The definitions in 64 bits: a dense array as a matrix whose columns are normalised."""
    s = prepare(case, seed)
    axis, kind, p = _axis(case), case["kind"], case.get("p", 0.0)
    shape = s["x"].shape
    rows, cols = shape[0], s["x"].numel() // shape[0]

    def matrix(t):
        t = t.reshape(rows, cols).double()
        return t if axis == 0 else t.t()

    def back(t):
        return (t if axis == 0 else t.t()).reshape(shape)

    def product(a, b):
        # high and low word of a 32 x 32 bit product, from products of 16-bit halves
        a1, a0, b1, b0 = a >> 16, a & 0xFFFF, b >> 16, b & 0xFFFF
        low, one, two = a0 * b0, a0 * b1, a1 * b0
        middle = (low >> 16) + (one & 0xFFFF) + (two & 0xFFFF)
        return a1 * b1 + (one >> 16) + (two >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) + (low & 0xFFFF)

    def factor():
        # what dropout multiplies every element by
        if p == 0.0:
            return 1.0
        seed64, number = (int(v) for v in s["random"])
        key = [seed64 % 2 ** 32, seed64 // 2 ** 32]
        quad = torch.arange((cols + 3) // 4, device=DEV)[None, :]
        row = torch.arange(rows, device=DEV)[:, None]
        c = [quad, row, torch.tensor([[s["site"]]], device=DEV), torch.tensor([[number % 2 ** 32]], device=DEV)]
        for i in range(10):
            h0, l0 = product(c[0], 0xD2511F53)
            h1, l1 = product(c[2], 0xCD9E8D57)
            c = [h1 ^ c[1] ^ (key[0] + i * 0x9E3779B9) % 2 ** 32, l1, h0 ^ c[3] ^ (key[1] + i * 0xBB67AE85) % 2 ** 32, l0]
        keep = 2 ** 32 - math.floor(p * 2 ** 32 + 0.5)
        f = torch.empty((rows, 4 * ((cols + 3) // 4)), dtype=torch.float64, device=DEV)
        for i in range(4):
            f[:, i::4] = torch.where(c[i] < keep, 2 ** 32 / keep, 0.0)
        f = f[:, :cols]
        return f if axis == 0 else f.t()

    if kind == "dropout":
        return {"y": back(matrix(s["x"]) * factor())}
    x, w = matrix(s["x"]), s["w"].double()[:, None]
    if kind in ("norm_fwd", "join_fwd"):
        out = {}
        if kind == "join_fwd":
            x = x + matrix(s["h"]) * factor()
            out["r"] = back(x)
        variance, mean = torch.var_mean(x, 0, correction=0)
        out["y"] = back((x - mean) / torch.sqrt(variance + EPS) * w + s["b"].double()[:, None])
        if case["stats"]:
            out["stats"] = torch.stack([mean, 1 / torch.sqrt(variance + EPS)])
        return out
    mean, inverse = s["stats"].double()
    x = (x - mean) * inverse
    g = matrix(s["gy"])
    out = {"gw": (g * x).sum(1), "gb": g.sum(1)}
    g = g * w
    g = (g - g.mean(0) - x * (g * x).mean(0)) * inverse
    if case.get("gr"):
        g = g + matrix(s["gr"])
    out = {"gx": back(g), **out}
    if kind == "join_bwd" and p > 0.0:
        out["gh"] = back(g * factor())
    return out


def work(case):
    """Bytes: every operand read once, every result written once.  FLOPs: those on the values, without the generator's integers."""
    shape, kind = _shape(case), case["kind"]
    elements, features = math.prod(shape), shape[_axis(case)]
    positions = elements // features
    if kind == "dropout":
        return {"bytes": 8.0 * elements, "flops": 1.0 * elements}
    if kind in ("norm_fwd", "join_fwd"):
        arrays = 2 if kind == "norm_fwd" else 4
        values = arrays * elements + 2 * features + (2 * positions if case["stats"] else 0)
        return {"bytes": 4.0 * values, "flops": (7.0 if kind == "norm_fwd" else 9.0) * elements}
    arrays = 3 + (kind == "join_bwd" and case["gr"]) + (kind == "join_bwd" and case["p"] > 0)
    return {"bytes": 4.0 * (arrays * elements + 3 * features + 2 * positions), "flops": 13.0 * elements}
