"""More operators around the STEM layer and their plain forms: products in 8-bit floating point with a scale for each block of 128, by groups of rows
that have weights of their own, and what brings tokens to such groups (experts) and back.

  linear    y = residual + Q(N(x)) Q(W_g)^T.  Q: blocks of 128 values of a row of x, of 128 x 128 of a matrix; with e the least integer for which the block's
            largest magnitude is at most 448 2^e (and at least -126), the values are those of 8-bit floating point (e4m3, round to nearest even) times 2^e.
            Rows offsets[g] .. offsets[g + 1] meet matrix g; rows behind the last group are left as they were.
  grad      its backward pass: dx = Q(dy) Q(W_g), blocks of 128 along the row of dy; dW_g = Q'(dy)^T Q'(x) over the rows of a group, Q' in blocks of 128 rows of
            the group, column by column.
  ffn       the layer: y = x + Q(SiLU(Q(N(x)) Q(W_gate)^T) * E[ids]) Q(W_down)^T, by groups too.
  dispatch  (token, choice) pairs sorted by expert, stable; src: the pair of each row, place: the row of each pair, -1 where it has no expert; rows of x and the
            token ids in that order.
  combine   y_t = residual_t + sum over the choices of w_tj ys[place_tj]; its backward pass gives every row its w_tj dy_t and every weight <dy_t, ys[place_tj]>;
            without weights it is the backward pass of dispatch.

Sizes are those of the package's own workloads (`paper_2601_10639_amd.inputs.SHAPES`) or generic ones beside them.
"""
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
F32, BF16 = torch.float32, torch.bfloat16
BIG = dict(d=2048, F=8192)     # the 1B-shaped layer
MOST = 2 * 16384 * 2048 * 8192 * 2


def listed():
    return [
        # one user's chat on the 350M-shaped model: a projection of a single token, every weight read once
        dict(name="linear_1", op="linear", T=1, K=1024, N=4096, groups=1, residual=False, norm="none"),
        # one prompt, and a matrix whose sides fit neither block nor tile nor vector
        dict(name="linear_odd", op="linear", T=700, K=1999, N=1001, groups=1, residual=True, norm="none"),
        # the first projection of 16 small experts for a prompt's tokens, which are spread unevenly over them
        dict(name="linear_experts", op="linear", T=8192, K=1024, N=4096, groups=16, residual=False, norm="none"),
        # fine-tuning of a small odd layer's experts on ragged sequences, some of them without a token
        dict(name="grad_experts_odd", op="grad", T=3001, K=520, N=1000, groups=7),
        # the training step of the 350M shape's projection
        dict(name="grad_350m", op="grad", T=16384, K=1024, N=4096, groups=1),
        # the training step of the 1B shape's projection
        dict(name="grad_1b", op="grad", T=16384, K=2048, N=8192, groups=1),
        # one user's chat on the 1B shape: norm, layer and residual of a single token
        dict(name="ffn_1", op="ffn", T=1, V=128256, groups=1, **BIG),
        # a batch of long prompts through the layer
        dict(name="ffn_16384", op="ffn", T=16384, V=128256, groups=1, **BIG),
        # a serving step of 64 users, two of 16 experts each
        dict(name="dispatch_decode", op="dispatch", dtype="bf16", T=64, k=2, experts=16, d=1024),
        # a training batch, two of 64 experts for each token, some tokens padded
        dict(name="dispatch_train", op="dispatch", dtype="bf16", T=16384, k=2, experts=64, d=2048),
        # the same batch's rows back at their tokens, weighted, onto the residual stream
        dict(name="combine_train", op="combine", grad=False, dtype="bf16", weights=True, residual=True, T=16384, k=2, experts=64, d=2048),
        # a small fp32 run's backward pass, a width that fills no vector
        dict(name="combine_grad_f32", op="combine", grad=True, dtype="f32", weights=True, residual=False, T=1999, k=3, experts=5, d=1001),
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def _mult(x, m):
    return max(m, int(round(x / m)) * m)


def draw(rng):
    op = rng.choice(["linear", "linear", "grad", "grad", "ffn", "ffn", "dispatch", "combine", "combine"])
    if op in ("linear", "grad"):
        K, N = int(_log(rng, 64, 8192)), int(_log(rng, 64, 8192))
        if rng.random() < 0.5:
            K, N = _mult(K, 64), _mult(N, 64)
        groups = rng.choice([1, 1, 1, int(_log(rng, 2, 64))])
        groups = max(1, min(groups, 2 ** 28 // (N * K)))
        c = dict(op=op, T=int(min(_log(rng, 1 if op == "linear" else 16, 32768), MOST / ((2 if op == "linear" else 4) * N * K))), K=K, N=N, groups=groups)
        return c if op == "grad" else dict(c, residual=rng.random() < 0.5, norm=rng.choice(["none", "none", "rms", "layer"]))
    if op == "ffn":
        d = _mult(_log(rng, 256, 2048), 64)
        F = min(8192, _mult(d * rng.uniform(2.5, 4.0), 64))
        return dict(op=op, T=int(_log(rng, 1, 16384)), d=d, F=F, V=int(_log(rng, 8000, 128256)), groups=rng.choice([1, 1, 1, 2, 5, 8]))
    dtype, k = rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 2, 4, 8])
    d = int(_log(rng, 16, 8192))
    if rng.random() < 0.7:
        d = _mult(d, 8)
    T = int(max(1, min(_log(rng, 1, 65536), 2 ** 26 / (d * k * (1 if dtype == "bf16" else 2)))))
    c = dict(op=op, dtype=dtype, T=T, k=k, experts=max(k, int(_log(rng, 2, 256))), d=d)
    return c if op == "dispatch" else dict(c, grad=rng.random() < 0.5, weights=rng.random() < 0.8, residual=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _type(c):
    return F32 if c.get("dtype") == "f32" else BF16


def _offsets(T, groups, seed):
    """Rows of each group: uneven, and now and then none; all rows belong to one."""
    rng = random.Random(seed)
    share = [0.0 if rng.random() < 0.1 else rng.lognormvariate(0.0, 0.8) for _ in range(groups)]
    if not any(share):
        share[0] = 1.0
    at, out = 0.0, [0]
    for s in share:
        at += s
        out.append(int(round(T * at / sum(share))))
    return out


def _inputs(c, seed):
    """The tensors of a case, from its seed alone."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, op, T = _type(c), c["op"], c["T"]

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return torch.empty(*shape, device=DEV, dtype=F32).normal_(mean, std, generator=gen).to(dtype)

    if op in ("linear", "grad", "ffn"):
        G = c["groups"]
        bounds = _offsets(T, G, seed)
        s = dict(bounds=bounds, offsets=None if G == 1 else torch.tensor(bounds, dtype=torch.int32).to(DEV))
    if op == "linear":
        K, N = c["K"], c["N"]
        # rows whose sizes differ, as those of activations do
        s.update(x=normal(T, K) * normal(T, 1, std=0.5, mean=1.5), W=normal(G, N, K, std=0.02), res=normal(T, N) if c["residual"] else None,
                 w=normal(K, std=0.2, mean=1.0) if c["norm"] != "none" else None)
        return s
    if op == "grad":
        K, N = c["K"], c["N"]
        # gradients are small, and differ by tokens
        s.update(x=normal(T, K), W=normal(G, N, K, std=0.02), dy=normal(T, N, std=1e-3) * normal(T, 1, std=0.5, mean=1.0))
        return s
    if op == "ffn":
        d, F, V = c["d"], c["F"], c["V"]
        # token ids: a few of the vocabulary take most places, as words do
        ids = (V ** torch.rand(T, device=DEV, generator=gen) - 1.0).to(torch.int32).clamp_(0, V - 1)
        # a table whose rows have grown to what an up projection would give, so that the layer weighs as much as the residual
        s.update(x=normal(T, d), w=normal(d, std=0.2, mean=1.0), ids=ids, Wg=normal(G, F, d, std=0.02), Wd=normal(G, d, F, std=0.02),
                 E=torch.empty(V, F, device=DEV, dtype=dt).normal_(0.0, 1.0, generator=gen))
        return s
    k, n, d = c["k"], c["experts"], c["d"]
    # a router's scores: some experts are liked more than others; one token in 16 is padding and goes nowhere
    scores = normal(T, n, dtype=F32) + normal(n, dtype=F32)
    top, experts = torch.topk(scores, k, dim=1)
    padded = torch.rand(T, 1, device=DEV, generator=gen) < 1 / 16
    experts = torch.where(padded, torch.full_like(experts, -1), experts).to(torch.int32).contiguous()
    if op == "dispatch":
        return dict(experts=experts, x=normal(T, d), ids=torch.randint(0, 32000, (T,), device=DEV, generator=gen).to(torch.int32))
    flat = torch.where(experts.reshape(-1) < 0, n, experts.reshape(-1).long())
    order = torch.sort(flat, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=DEV)
    place = torch.where(flat < n, place, torch.full_like(place, -1)).to(torch.int32).reshape(T, k)
    s = dict(place=place, ys=normal(T * k, d), weights=torch.softmax(top, 1) if c["weights"] else None)
    if c["grad"]:
        s["dy"] = normal(T, d, std=1e-2)
    else:
        s["res"] = normal(T, d, std=2.0) if c["residual"] else None
    return s


_contexts = {}   # a program makes its contexts when it starts


def _context(d, F, V, dtype, T, groups=0, backward=False):
    from paper_2601_10639_amd import stemlib as L
    key = (d, F, V, dtype, T, groups, backward)
    if key not in _contexts:
        _contexts[key] = L.stem_create(d, F, V, dtype, T)
        if groups:
            L.stem_qfloat_reserve(_contexts[key], groups=groups, backward=backward)
    return _contexts[key]


def prepare(case, seed):
    c = case
    s = dict(_inputs(c, seed), case=c)
    op, T, dt = c["op"], c["T"], _type(c)

    def empty(*shape, dtype=dt):
        return torch.zeros(*shape, dtype=dtype, device=DEV)

    if not own:
        # weights are quantised once, when a model is loaded
        for name in ("W", "Wg", "Wd"):
            if name in s:
                s["q" + name] = torch.stack([_square(m) for m in s[name]])
        return s
    from paper_2601_10639_amd import stemlib as L
    code = L.STEM_F32 if dt == F32 else L.STEM_BF16
    kinds = {"rms": L.STEM_NORM_RMS, "layer": L.STEM_NORM_LAYER}
    if op in ("linear", "grad"):
        K, N, G = c["K"], c["N"], c["groups"]
        m = -(-max(K, N) // 64) * 64
        s["ctx"] = _context(64, m, 1000, code, T, G, op == "grad")
        s["pW"] = L.stem_qfloat_weights(s["ctx"], s["W"], backward=op == "grad")
        if op == "grad":
            s.update(dx=empty(T, K), dW=empty(G, N, K, dtype=F32))
        else:
            s.update(y=empty(T, N), norm=None if c["norm"] == "none" else L.stem_norm(kinds[c["norm"]], EPS, s["w"]))
    elif op == "ffn":
        s["ctx"] = _context(c["d"], c["F"], c["V"], code, T, c["groups"])
        s["pWg"], s["pWd"] = L.stem_qfloat_weights(s["ctx"], s["Wg"]), L.stem_qfloat_weights(s["ctx"], s["Wd"])
        s.update(norm=L.stem_norm(L.STEM_NORM_RMS, EPS, s["w"]), y=empty(T, c["d"]))
    else:
        k, d = c["k"], c["d"]
        s["ctx"] = _context(64, 64, 1000, code, T)
        i32 = torch.int32
        if op == "dispatch":
            s.update(src=empty(T * k, dtype=i32), place=empty(T, k, dtype=i32), offsets=empty(c["experts"] + 1, dtype=i32), xs=empty(T * k, d),
                     ids_out=empty(T * k, dtype=i32))
        elif c["grad"]:
            s.update(dys=empty(T * k, d), dw=empty(T, k, dtype=F32) if c["weights"] else None)
        else:
            s["y"] = empty(T, d)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _to_eight(v, top):
    """The values that v has in 8 bits, for the largest magnitudes of their blocks (of v's shape, or one that it is spread over)."""
    bits = top.view(torch.int32)
    exponent = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)      # 448 = 1.75 x 2^8
    exponent = exponent.clamp_min(-126)
    down, up = ((127 - exponent) << 23).view(F32), ((127 + exponent) << 23).view(F32)
    return (v * down).to(torch.float8_e4m3fn).float() * up


def _rows(v):
    """Q along rows."""
    T, K = v.shape
    out = torch.nn.functional.pad(v.float(), (0, -K % 128)).reshape(T, -1, 128)
    return _to_eight(out, out.abs().amax(2, keepdim=True)).reshape(T, -1)[:, :K]


def _square(m):
    """Q of a matrix, in blocks of 128 x 128."""
    N, K = m.shape
    out = torch.nn.functional.pad(m.float(), (0, -K % 128, 0, -N % 128))
    out = out.reshape(out.shape[0] // 128, 128, -1, 128)
    out = _to_eight(out, out.abs().amax((1, 3), keepdim=True))
    return out.reshape(out.shape[0] * 128, -1)[:N, :K].contiguous()


def _normed(v, kind):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v if kind == "none" else v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)


def _by_groups(a, weights, bounds):
    """Rows of a times the transposed matrix of their group."""
    if len(weights) == 1:
        return a @ weights[0].t()
    return torch.cat([a[lo:hi] @ w.t() for w, lo, hi in zip(weights, bounds, bounds[1:])])


def _plain(s):
    c = s["case"]
    op, dt, T = c["op"], _type(c), c["T"]
    if op == "linear":
        n = _normed(s["x"].float(), c["norm"])
        y = _by_groups(_rows(n if s["w"] is None else n * s["w"].float()), s["qW"], s["bounds"])
        return (y if s["res"] is None else y + s["res"].float()).to(dt)
    if op == "grad":
        dx = _by_groups(_rows(s["dy"]), s["qW"].transpose(1, 2), s["bounds"]).to(dt)
        dW = torch.empty(c["groups"], c["N"], c["K"], device=DEV, dtype=F32)
        for g, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
            dW[g] = _rows(s["dy"][lo:hi].t()) @ _rows(s["x"][lo:hi].t()).t() if hi > lo else 0.0
        return dx, dW
    if op == "ffn":
        x = s["x"].float()
        z = _by_groups(_rows(_normed(x, "rms") * s["w"].float()), s["qWg"], s["bounds"])
        h = z / (1.0 + torch.exp(-z)) * s["E"][s["ids"].long()].float()
        return (x + _by_groups(_rows(h), s["qWd"], s["bounds"])).to(dt)
    k, n = c["k"], c["experts"]
    if op == "dispatch":
        flat = s["experts"].reshape(-1).long()
        flat = torch.where(flat < 0, n, flat)
        order = torch.sort(flat, stable=True).indices
        counts = (flat[:, None] == torch.arange(n, device=DEV)).sum(0)
        offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        real = torch.arange(T * k, device=DEV) < offsets[-1]
        place = torch.empty_like(order)
        place[order] = torch.where(real, torch.arange(T * k, device=DEV), -1)
        token = order // k
        xs = torch.where(real[:, None], s["x"][token], 0.0).to(dt)
        return (torch.where(real, order, -1).to(torch.int32), place.to(torch.int32).reshape(T, k), offsets.to(torch.int32), xs,
                torch.where(real, s["ids"][token], 0).to(torch.int32))
    real, at = s["place"] >= 0, s["place"].long().clamp_min(0)
    w = real.float() if s["weights"] is None else torch.where(real, s["weights"], 0.0)
    if not c["grad"]:
        y = torch.zeros(T, c["d"], device=DEV) if s["res"] is None else s["res"].float()
        for j in range(k):
            y = y + w[:, j, None] * s["ys"][at[:, j]].float()
        return y.to(dt)
    dys = torch.zeros(T * k, c["d"], device=DEV, dtype=dt)
    dw = torch.zeros(T, k, device=DEV)
    # (padded tokens' rows are the last ones, which stay zero: they are written there, and zero)
    for j in range(k):
        dw[:, j] = torch.where(real[:, j], (s["dy"].float() * s["ys"][at[:, j]].float()).sum(1), 0.0)
        rows = torch.where(real[:, j], at[:, j], T * k - 1)
        dys.index_add_(0, rows, torch.where(real[:, j, None], w[:, j, None] * s["dy"].float(), 0.0).to(dt))
    return dys, dw if s["weights"] is not None else None


def _own(s):
    from paper_2601_10639_amd import stemlib as L
    c, op = s["case"], s["case"]["op"]
    if op == "linear":
        L.stem_qfloat_linear(s["ctx"], s["x"], s["pW"], s["y"], residual=s["res"], norm=s["norm"], offsets=s["offsets"])
        return s["y"]
    if op == "grad":
        L.stem_qfloat_linear_backward_quantised(s["ctx"], s["dy"], s["x"], s["pW"], s["dx"], s["dW"], offsets=s["offsets"])
        return s["dx"], s["dW"]
    if op == "ffn":
        L.stem_qfloat_ffn_forward(s["ctx"], s["x"], s["ids"], s["pWg"], s["pWd"], s["E"], s["y"], residual=s["x"], norm=s["norm"], offsets=s["offsets"])
        return s["y"]
    if op == "dispatch":
        L.stem_experts_sort(s["ctx"], s["experts"], s["src"], s["place"], s["offsets"])
        L.stem_experts_dispatch(s["ctx"], s["x"], s["src"], s["xs"], choices=c["k"], ids=s["ids"], ids_out=s["ids_out"])
        return s["src"], s["place"], s["offsets"], s["xs"], s["ids_out"]
    if c["grad"]:
        L.stem_experts_combine_backward(s["ctx"], s["dy"], s["place"], s["dys"], ys=s["ys"], weights=s["weights"], dweights=s["dw"])
        return s["dys"], s["dw"]
    L.stem_experts_combine(s["ctx"], s["ys"], s["place"], s["y"], weights=s["weights"], residual=s["res"])
    return s["y"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    c = case
    op, T = c["op"], c["T"]
    if op in ("linear", "grad"):
        K, N = c["K"], c["N"]
        met = min(T, c["groups"])
        if op == "linear":
            return dict(bytes=2 * T * K + met * N * K + 2 * T * N * (2 if c["residual"] else 1), flops=2 * T * K * N)
        return dict(bytes=2 * T * (N + K) + met * N * K + 2 * T * K + 4 * c["groups"] * N * K, flops=4 * T * K * N)
    if op == "ffn":
        d, F, V = c["d"], c["F"], c["V"]
        # rows of the table that this many tokens name, for ids as _inputs draws them
        rows = min(T, V, 0.6 * T ** 0.9)
        return dict(bytes=2 * 2 * T * d + 2 * min(T, c["groups"]) * d * F + 2 * rows * F + 4 * T + 2 * d, flops=4 * T * d * F)
    b = 4 if c["dtype"] == "f32" else 2
    k, d = c["k"], c["d"]
    rows = 15 / 16 * T * k
    if op == "dispatch":
        return dict(bytes=int(b * d * (T + rows) + 4 * (3 * T * k + T + rows)), flops=T * k)
    weights = 4 * T * k if c["weights"] else 0
    if c["grad"]:
        return dict(bytes=int(b * d * (T + rows * (2 if c["weights"] else 1)) + 4 * T * k + 2 * weights), flops=int(3 * rows * d))
    return dict(bytes=int(b * d * (T * (2 if c["residual"] else 1) + rows) + 4 * T * k + weights), flops=int(2 * rows * d))


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _two_to(e):
    """2^e, from its bits (a power function is not always exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _eight64(v, top):
    """Rounded to a multiple of a sixteenth of the power of two above the value, at least 2^-9 of the scale."""
    _, e = torch.frexp(top / 448.0)                     # top / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(448.0 * _two_to(e - 1) >= top, e - 1, e).clamp_min(-126)
    u = v / _two_to(e)
    _, own_e = torch.frexp(u)
    step = _two_to((own_e - 4).clamp_min(-9))
    return torch.round(u / step) * step * _two_to(e)


def _q64(v, dim):
    """Q in blocks of 128 along dim."""
    out = []
    for part in torch.split(v, 128, dim):
        out.append(_eight64(part, part.abs().max(dim, keepdim=True).values))
    return torch.cat(out, dim)


def _weights64(W):
    out = torch.empty(W.shape, device=DEV, dtype=torch.float64)
    for g in range(W.shape[0]):
        for lo in range(0, W.shape[1], 128):
            rows = W[g, lo:lo + 128].double()
            top = torch.stack([p.abs().max() for p in torch.split(rows, 128, 1)]).repeat_interleave(128)[:W.shape[2]]
            out[g, lo:lo + 128] = _eight64(rows, top.expand_as(rows))
    return out


def _norm64(v, kind):
    if kind == "none":
        return v
    if kind == "layer":
        return torch.nn.functional.layer_norm(v, v.shape[-1:], eps=EPS)
    return v / (v.pow(2).sum(-1, keepdim=True) / v.shape[-1] + EPS).sqrt()


def _grouped64(a, W, bounds, n):
    out = torch.zeros(a.shape[0], n, device=DEV, dtype=torch.float64)
    for g in range(len(W)):
        lo, hi = bounds[g], bounds[g + 1]
        if hi > lo:
            out[lo:hi] = torch.mm(a[lo:hi], W[g])
    return out


def exact(case, seed):
    c, op, T = case, case["op"], case["T"]
    s = _inputs(c, seed)
    if op == "linear":
        n = _norm64(s["x"].double(), c["norm"])
        a = _q64(n if s["w"] is None else n * s["w"].double(), 1)
        y = _grouped64(a, _weights64(s["W"]).transpose(1, 2).contiguous(), s["bounds"], c["N"])
        return y if s["res"] is None else y + s["res"].double()
    if op == "grad":
        dx = _grouped64(_q64(s["dy"].double(), 1), _weights64(s["W"]), s["bounds"], c["K"])
        dW = torch.zeros(c["groups"], c["N"], c["K"], device=DEV, dtype=torch.float64)
        for g in range(c["groups"]):
            lo, hi = s["bounds"][g], s["bounds"][g + 1]
            if hi > lo:
                dW[g] = torch.mm(_q64(s["dy"][lo:hi].double(), 0).t().contiguous(), _q64(s["x"][lo:hi].double(), 0))
        return dx, dW
    if op == "ffn":
        x = s["x"].double()
        n = _q64(_norm64(x, "rms") * s["w"].double(), 1)
        z = _grouped64(n, _weights64(s["Wg"]).transpose(1, 2).contiguous(), s["bounds"], c["F"])
        h = torch.nn.functional.silu(z) * s["E"][s["ids"].long()].double()
        return x + _grouped64(_q64(h, 1), _weights64(s["Wd"]).transpose(1, 2).contiguous(), s["bounds"], c["d"])
    k, d = c["k"], c["d"]
    if op == "dispatch":
        pairs = [(e, i) for i, e in enumerate(s["experts"].reshape(-1).tolist()) if e >= 0]
        token = torch.tensor([i // k for _, i in sorted(pairs)], dtype=torch.long).to(DEV)
        xs = torch.zeros(T * k, d, device=DEV, dtype=torch.float64)
        xs[:len(pairs)] = s["x"].double()[token]
        return None, None, None, xs, None
    place, ys = s["place"].long(), s["ys"].double()
    w = None if s["weights"] is None else s["weights"].double()
    # a matrix of no row behind the last one takes what belongs nowhere
    at = torch.where(place < 0, T * k, place)
    if not c["grad"]:
        rows = torch.cat([ys, ys.new_zeros(1, d)])[at]
        y = rows.sum(1) if w is None else (rows * w[:, :, None]).sum(1)
        return y if s["res"] is None else y + s["res"].double()
    dys = torch.zeros(T * k + 1, d, device=DEV, dtype=torch.float64)
    spread = s["dy"].double()[:, None, :].expand(T, k, d)
    dys[at.reshape(-1)] = (spread if w is None else spread * w[:, :, None]).reshape(T * k, d)
    if w is None:
        return dys[:T * k], None
    dw = (spread * torch.cat([ys, ys.new_zeros(1, d)])[at]).sum(2)
    return dys[:T * k], dw
