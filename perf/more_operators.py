"""What stands around a model's MLP layers in a training step, as cases: the normalisation before a layer, the loss over the
vocabulary behind the last one, and the update of the parameters.

Sizes are those of the parameter lists in `paper_2609_33437_gb300.workloads`: a vision tower (width 1024, 257 tokens an
image), a 7B decoder (width 4096, MLP 11008, vocabulary 32000) and a 0.5B decoder (width 896, MLP 4864, vocabulary 151936).
Five operators:

  norm        h = x + r, y = (h - mu) s w + b with s = 1 / sqrt(v + eps): mu and v a row's mean and variance ("layer"), or
              mu = 0 and v its mean square ("rms"); h and the rows' mu and s are kept for the backward pass
  norm_grad   dx = s (a - mean(a) - xh mean(a xh)) + dh, a = dy w, xh = (h - mu) s (without mean(a) for "rms"); dw and db, the
              sums over rows of dy xh and dy
  loss        lse = log sum exp of the logits l = x W^T, and lse - l[target], 0 where the target is to be ignored
  loss_grad   the same, then dx = d W and dW = d^T x with d = g (exp(l - lse) - [target])
  adamw       g = c grad; m1 = b1 m1 + (1 - b1) g; m2 = b2 m2 + (1 - b2) g^2; r = sqrt(m2);
              theta = theta (1 - lr wd) - lr / (1 - b1^t) m1 / (r / sqrt(1 - b2^t) + eps)
              over a list of tensors; m1 and m2 are kept in 32 bits, or m1 and r in 8

8 bits: 256 neighbours of a tensor share a power of two each for m1 and r, 2^(e - 127). With u = 2^(e - 127) a byte's low 7
bits c (m1; bit 7 is its sign) stand for c u below 8, else for (8 + c % 8) 2^(c // 8 - 1) u; a byte c of r stands for c u below
16, else for (16 + c % 16) 2^(c // 16 - 1) u. e is the biased exponent of the largest magnitude of the group less 16 (m1) or 17
(r), 1 at least. A value is rounded up or down with the probability that its place between the two neighbours gives, by 16 bits
of a number made of its place in the list, the step and a seed, so that small changes are not lost from step to step. Tensors
begin at multiples of 256 of the list. What is held in 8 bits is returned as the values it stands for, which bf16 holds exactly.
"""

import math

import torch

own = False

DEVICE = "cuda"
GROUP = 256
IGNORE = -100
EPS = 1e-5
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ADAM = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
_SEED = 1234567


# ----------------------------------------------------------------- the cases ---
def listed():
    return [
        # One token of a decoder on its way into a layer, the residual added: the smallest call, where latency counts.
        _norm("norm_token", "norm", rows=1, cols=4096, kind="rms", residual=True),
        # Sixteen images in a vision tower, weight and bias in fp32.
        _norm("norm_tower", "norm", rows=4112, cols=1024, kind="layer", weights="f32"),
        # Sixteen sequences of 512 tokens in the 7B decoder, the residual added.
        _norm("norm_decoder", "norm", rows=8192, cols=4096, kind="rms", residual=True),
        # Back through a tower's norm with the residual stream's gradient: thirty-two images, an odd number of rows.
        _norm("norm_grad_tower", "norm_grad", rows=8223, cols=1024, kind="layer", residual=True),
        # The 0.5B list trains in fp32: an odd number of tokens back through its norm.
        _norm("norm_grad_f32", "norm_grad", rows=4099, cols=896, kind="rms", dtype="f32"),
        # Scoring: a few candidates' last positions against the 7B decoder's vocabulary.
        _loss("loss_score", "loss", rows=24, k=4096, n=32000),
        # Evaluation of the 0.5B decoder on an odd number of tokens, over its large vocabulary.
        _loss("loss_eval", "loss", rows=2049, k=896, n=151936, ignored=0.1),
        # A training step's end in the 7B decoder: sixteen sequences of 512 tokens. The largest call.
        _loss("loss_grad_7b", "loss_grad", rows=8192, k=4096, n=32000, ignored=0.05),
        # The same in the 0.5B decoder, in fp32 as its list has it, one ragged sequence of which half is a prompt.
        _loss("loss_grad_f32", "loss_grad", rows=515, k=896, n=32000, dtype="f32", ignored=0.5),
        # Adapters on the projections of three layers in fp32: a small list, where latency counts.
        _adamw("adamw_adapters", tensors=24, low=32768, high=32768, dtype="f32", grads="f32", bits=32),
        # A vision tower of 24 layers in bf16, matrices, norms and biases, moments in 8 bits.
        _adamw("adamw_tower_8", tensors=288, low=1024, high=4194304, dtype="bf16", grads="bf16", bits=8),
        # The 0.5B decoder's list in fp32, moments in 32 bits.
        _adamw("adamw_decoder_32", tensors=216, low=128, high=16777216, dtype="f32", grads="f32", bits=32),
    ]


def _norm(name, op, rows, cols, kind, dtype="bf16", weights="same", residual=False):
    return dict(name=name, op=op, rows=rows, cols=cols, kind=kind, dtype=dtype, weights=weights, residual=residual)


def _loss(name, op, rows, k, n, dtype="bf16", ignored=0.0):
    return dict(name=name, op=op, rows=rows, k=k, n=n, dtype=dtype, ignored=ignored)


def _adamw(name, tensors, low, high, dtype, grads, bits):
    return dict(name=name, op="adamw", tensors=tensors, low=low, high=high, dtype=dtype, grads=grads, bits=bits)


def _size(rng, low, high):
    """A size spread over its logarithm: odd ones, multiples of 8 and of 128."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice((1, 1, 8, 128))
    return min(high, max(low, (v + step // 2) // step * step))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "loss", "loss_grad", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("norm", "norm_grad"):
        c = _norm("", op, rows=_size(rng, 1, 16384), cols=_size(rng, 16, 11008), kind=rng.choice(("layer", "rms")), dtype=dtype,
                  weights=rng.choice(("same", "f32")), residual=rng.random() < 0.5)
    elif op in ("loss", "loss_grad"):
        c = _loss("", op, rows=_size(rng, 1, 8192), k=_size(rng, 64, 4096), n=_size(rng, 500, 151936), dtype=dtype,
                  ignored=rng.choice((0.0, 0.1, 0.5)))
        # at most half of the largest listed one, a tenth of it in fp32, which has no matrix instructions of its width
        most = 8192 * 4096 * 32000 // (10 if dtype == "f32" else 2)
        while c["rows"] * c["k"] * c["n"] > most:
            c["rows"] = max(1, c["rows"] * 2 // 3)
            c["n"] = max(500, c["n"] * 3 // 4)
    else:
        low = _size(rng, 1, 65536)
        c = _adamw("", tensors=_size(rng, 1, 200), low=low, high=low * rng.choice((1, 8, 64)), dtype=dtype,
                   grads=rng.choice((dtype, "f32")), bits=rng.choice((8, 32)))
    del c["name"]
    return c


def _sizes(case):
    """The list's tensors: sizes from low to high over their logarithm, large and small ones in turn, none like the next."""
    n, low, high = case["tensors"], case["low"], case["high"]
    out = []
    for i in range(n):
        at = (i * 7 % n) / max(1, n - 1)
        v = int(round(low * (high / low) ** at))
        out.append(v if high == low or i % 3 else v + 1)
    return out


def _starts(sizes):
    """Where each tensor begins in the list, and the list's length."""
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // GROUP) * GROUP
    return out, at


# ----------------------------------------------------------------- the inputs ---
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _stream(g, rows, cols):
    """Activations: normal, with one column in 64 eight times as large, as trained networks have them."""
    x = _normal(g, rows, cols)
    x[:, ::64] *= 8.0
    return x


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op, dt = case["op"], _TYPES[case["dtype"]]
    s = {"case": case}
    if op in ("norm", "norm_grad"):
        m, n = case["rows"], case["cols"]
        wt = torch.float32 if case["weights"] == "f32" else dt
        s["x"] = (_stream(g, m, n) + 0.5).to(dt)
        s["w"] = (1.0 + 0.2 * _normal(g, n)).to(wt)
        s["b"] = (0.1 * _normal(g, n)).to(wt) if case["kind"] == "layer" else None
        if op == "norm":
            s["r"] = _normal(g, m, n).to(dt) if case["residual"] else None
        else:
            s["dy"] = (1e-2 * _normal(g, m, n)).to(dt)
            s["dh"] = (1e-2 * _normal(g, m, n)).to(dt) if case["residual"] else None
            s["stats"] = _stats(s["x"].float(), case["kind"])  # as the forward pass kept them
        return s
    if op in ("loss", "loss_grad"):
        m, k, n = case["rows"], case["k"], case["n"]
        s["w"] = (2.0 / math.sqrt(k) * _normal(g, n, k)).to(dt)
        # frequent and rare words; the last layer's output leans towards the right one, as a trained model's does
        t = (n * torch.rand(m, generator=g, device=DEVICE, dtype=torch.float64) ** 3).long().clamp_(max=n - 1)
        s["x"] = (_normal(g, m, k) + 3.0 * s["w"][t].float()).to(dt)
        s["t"] = torch.where(torch.rand(m, generator=g, device=DEVICE) < case["ignored"], IGNORE, t)
        # the mean over the tokens that count
        s["g"] = torch.full((m,), 1.0 / max(1.0, m * (1.0 - case["ignored"])), device=DEVICE)
        return s
    sizes = _sizes(case)
    starts, total = _starts(sizes)
    gt = _TYPES[case["grads"]]
    s["sizes"], s["starts"] = sizes, starts
    length, first = torch.tensor(sizes, device=DEVICE), torch.tensor(starts, device=DEVICE)
    place = torch.arange(total, device=DEVICE)
    which = torch.bucketize(place, first, right=True) - 1
    there = place - first[which] < length[which]  # not between two tensors
    del which, place
    # gradients of a tensor spread over some orders of magnitude; moments that went before them
    spread = torch.exp(1.5 * _normal(g, total)) * 1e-3 * there
    s["p"] = (0.02 * _normal(g, total) * there).to(dt)
    s["g"] = (spread * _normal(g, total)).to(gt)
    m1, m2 = 0.2 * spread * _normal(g, total), spread * spread * (0.5 + torch.rand(total, generator=g, device=DEVICE))
    del spread, there
    s["scale"] = torch.full((), 0.5, device=DEVICE)
    if case["bits"] == 8:
        # byte by byte as an earlier step left them
        s["q1"], s["e1"], s["q2"], s["e2"] = _pack(m1, torch.sqrt(m2), _dither(total, 9, DEVICE))
    else:
        s["m1"], s["m2"] = m1, m2
    if own:  # the handle that a program keeps for its optimizer
        from paper_2609_33437_gb300 import optim as O

        s["params"] = [s["p"][a:a + n] for a, n in zip(starts, sizes)]
        s["grads"] = [s["g"][a:a + n] for a, n in zip(starts, sizes)]
        s["moments"] = O.Moments(s["params"], bits=case["bits"])
        for name, t in s["moments"].buffers().items():
            t.copy_(s[name])
            s[name] = t
    return s


# ------------------------------------------------------------ the plain forms ---
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _stats(h, kind):
    if kind == "layer":
        mu = h.mean(1)
        v = (h - mu[:, None]).square().mean(1)
        return torch.stack([mu, 1.0 / torch.sqrt(v + EPS)])
    return (1.0 / torch.sqrt(h.square().mean(1) + EPS))[None]


def _run_plain(s):
    c = s["case"]
    dt, op = _TYPES[c["dtype"]], c["op"]
    if op == "norm":
        h = s["x"].float()
        if s["r"] is not None:
            h = (h + s["r"].float()).to(dt).float()
        stats = _stats(h, c["kind"])
        y = h - stats[0][:, None] if c["kind"] == "layer" else h
        y = y * stats[-1][:, None] * s["w"].float()
        if s["b"] is not None:
            y = y + s["b"].float()
        out = {"y": y.to(dt), "stats": stats}
        if s["r"] is not None:
            out["h"] = h.to(dt)
        return out
    if op == "norm_grad":
        h, dy, rs = s["x"].float(), s["dy"].float(), s["stats"][-1][:, None]
        xh = (h - s["stats"][0][:, None] if c["kind"] == "layer" else h) * rs
        a = dy * s["w"].float()
        dx = a - xh * (a * xh).mean(1, keepdim=True)
        if c["kind"] == "layer":
            dx = dx - a.mean(1, keepdim=True)
        dx = dx * rs
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        out = {"dx": dx.to(dt), "dw": (dy * xh).sum(0).to(s["w"].dtype)}
        if s["b"] is not None:
            out["db"] = dy.sum(0).to(s["b"].dtype)
        return out
    if op in ("loss", "loss_grad"):
        x, w, t = s["x"].float(), s["w"].float(), s["t"]
        counts = t != IGNORE
        at = torch.where(counts, t, 0)[:, None]
        l = x @ w.T
        top = l.amax(1)
        lse = top + torch.log(torch.exp(l - top[:, None]).sum(1))
        loss = torch.where(counts, lse - l.gather(1, at)[:, 0], 0.0)
        if op == "loss":
            return {"loss": loss, "lse": lse}
        d = torch.exp(l - lse[:, None])
        d.scatter_add_(1, at, torch.full_like(at, -1, dtype=d.dtype))
        d = d * torch.where(counts, s["g"], 0.0)[:, None]
        return {"loss": loss, "dx": (d @ w).to(dt), "dw": (d.T @ x).to(dt)}
    a = _ADAM
    p, g = s["p"].float(), s["g"].float() * s["scale"]
    if c["bits"] == 8:
        m1, r0 = _unpack1(s["q1"], s["e1"]), _unpack2(s["q2"], s["e2"])
        m2 = r0 * r0
    else:
        m1, m2 = s["m1"], s["m2"]
    t = 100
    m1 = a["beta1"] * m1 + (1.0 - a["beta1"]) * g
    m2 = a["beta2"] * m2 + (1.0 - a["beta2"]) * (g * g)
    r = torch.sqrt(m2)
    p = p * (1.0 - a["lr"] * a["weight_decay"])
    p = p - a["lr"] / (1.0 - a["beta1"] ** t) * (m1 / (r / math.sqrt(1.0 - a["beta2"] ** t) + a["eps"]))
    s["p"].copy_(p)
    if c["bits"] == 32:
        s["m1"].copy_(m1)
        s["m2"].copy_(m2)
        return {"p": s["p"], "m1": s["m1"], "m2": s["m2"]}
    for name, v in zip(("q1", "e1", "q2", "e2"), _pack(m1, r, _dither(m1.numel(), t, m1.device))):
        s[name].copy_(v)
    return {"p": s["p"], "m1": _unpack1(s["q1"], s["e1"]).to(torch.bfloat16),
            "r": _unpack2(s["q2"], s["e2"]).to(torch.bfloat16)}


_LOW = (1 << 32) - 1


def _mix(h):
    """The 32-bit finaliser of MurmurHash3 (A. Appleby), on whole numbers below 2^32."""
    h = h ^ (h >> 16)
    h = h * 0x85EBCA6B & _LOW
    h = h ^ (h >> 13)
    h = h * 0xC2B2AE35 & _LOW
    return h ^ (h >> 16)


def _dither(n, step, device):
    """A 32-bit number for each of the list's n < 2^32 places: the low half rounds m1, the high half r."""
    key = _mix(_mix(_mix(_SEED & _LOW) ^ (_SEED >> 32)) ^ step)
    return _mix(torch.arange(n, device=device) ^ _mix(key))


def _power(e):
    """2^(e - 127) of bytes e >= 1, a group's for each of its values."""
    return (e.to(torch.int32) << 23).view(torch.float32).repeat_interleave(GROUP)


def _rounded(v, e, part, places):
    """The codes of v >= 0 of `places` binary places with the units 2^(e - 127); `part`: 16 bits for each."""
    f = v * _power(254 - e.to(torch.int32))
    u = (part.float() + 0.5) * 2.0 ** -16
    one = float(1 << places)
    at = torch.where(f >= one, (f.view(torch.int32) >> 23) - 127 - places, 0)
    up = torch.floor(f * ((127 - at) << 23).view(torch.float32) + u).to(torch.int32)
    return ((at << places) + up).to(torch.uint8)


def _exponent(v, less):
    top = v.view(-1, GROUP).amax(1).view(torch.int32) >> 23
    return (top - less).clamp(min=1).to(torch.uint8)


def _pack(m1, r, dither):
    """(q1, e1, q2, e2) of the first moments and the roots of the second, see the head of this file."""
    size = m1.abs()
    e1, e2 = _exponent(size, 16), _exponent(r, 17)
    q1 = _rounded(size, e1, dither & 0xFFFF, 3) | torch.where(m1 < 0, 128, 0).to(torch.uint8)
    return q1, e1, _rounded(r, e2, dither >> 16, 4), e2


def _unpack(c, e, places):
    c = c.to(torch.int32)
    one = 1 << places
    high = c >> places
    v = torch.where(high > 0, ((one + c % one) << (high - 1).clamp(min=0)), c).float()
    return v * _power(e)


def _unpack1(q, e):
    v = _unpack(q & 127, e, 3)
    return torch.where(q >= 128, -v, v)


def _unpack2(q, e):
    return _unpack(q, e, 4)


# ---------------------------------------------------- the framework's operators ---
def _run_own(s):
    c = s["case"]
    op = c["op"]
    if op in ("norm", "norm_grad"):
        from paper_2609_33437_gb300 import norm as N

        if op == "norm":
            got = N.norm(s["x"], s["w"], s["b"], residual=s["r"], kind=c["kind"], eps=EPS, save=True)
            return {"y": got[0], "stats": got[-1]} if s["r"] is None else {"y": got[0], "stats": got[-1], "h": got[1]}
        dx, dw, db = N.norm_grad(s["dy"], s["x"], s["stats"], s["w"], bias=s["b"] is not None, kind=c["kind"], dh=s["dh"])
        return {"dx": dx, "dw": dw, "db": db} if s["b"] is not None else {"dx": dx, "dw": dw}
    if op in ("loss", "loss_grad"):
        from paper_2609_33437_gb300 import loss as T

        loss, lse = T.token_loss(s["x"], s["w"], s["t"], ignore=IGNORE)
        if op == "loss":
            return {"loss": loss, "lse": lse}
        dx, dw = T.token_loss_grad(s["g"], s["x"], s["w"], s["t"], lse, ignore=IGNORE)
        return {"loss": loss, "dx": dx, "dw": dw}
    from paper_2609_33437_gb300 import optim as O

    O.adamw(s["params"], s["grads"], s["moments"], step=100, seed=_SEED, scale=s["scale"], **_ADAM)
    if c["bits"] == 32:
        return {"p": s["p"], "m1": s["m1"], "m2": s["m2"]}
    m1, r = s["moments"].values()
    return {"p": s["p"], "m1": m1, "r": r}


# ------------------------------------------------------------------- the work ---
def work(case):
    op = case["op"]
    b = 2 if case["dtype"] == "bf16" else 4
    if op == "adamw":
        n = sum(_sizes(case))
        each = 2 * b + (2 if case["grads"] == "bf16" else 4)
        # moments read and written; those in 8 bits then read once more and returned as values
        each += 16 if case["bits"] == 32 else 4 + 2 + 4
        return {"bytes": each * n, "flops": 14 * n}
    m = case["rows"]
    if op in ("norm", "norm_grad"):
        n = case["cols"]
        w = 4 if case["weights"] == "f32" else b
        layer = case["kind"] == "layer"
        if op == "norm":
            return {"bytes": b * m * n * (4 if case["residual"] else 2) + w * n * (2 if layer else 1) + 4 * m * (2 if layer else 1),
                    "flops": 8 * m * n}
        return {"bytes": b * m * n * (4 if case["residual"] else 3) + w * n * (3 if layer else 2) + 4 * m * (2 if layer else 1),
                "flops": 14 * m * n}
    k, n = case["k"], case["n"]
    if op == "loss":
        return {"bytes": b * (m * k + n * k) + 16 * m, "flops": 2.0 * m * n * k}
    return {"bytes": 2 * b * (m * k + n * k) + 20 * m, "flops": 6.0 * m * n * k}


# ------------------------------------------------------- the definition, 64 bits ---
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "norm":
        h = wide["x"]
        if s["r"] is not None:
            h = (h + wide["r"]).to(s["x"].dtype).double()
        mu = torch.einsum("ij->i", h) / h.shape[1] if case["kind"] == "layer" else torch.zeros_like(h[:, 0])
        off = h - mu.unsqueeze(1)
        inv = torch.rsqrt(torch.einsum("ij,ij->i", off, off) / h.shape[1] + EPS)
        y = torch.einsum("ij,i,j->ij", off, inv, wide["w"])
        out = {"y": y + wide["b"] if s["b"] is not None else y,
               "stats": torch.stack([mu, inv]) if case["kind"] == "layer" else inv.unsqueeze(0)}
        if s["r"] is not None:
            out["h"] = h
        return out
    if op == "norm_grad":
        inv, n = wide["stats"][-1], case["cols"]
        off = wide["x"] - wide["stats"][0].unsqueeze(1) if case["kind"] == "layer" else wide["x"]
        hat = torch.einsum("ij,i->ij", off, inv)
        a = torch.einsum("ij,j->ij", wide["dy"], wide["w"])
        inner = a - torch.einsum("ij,i->ij", hat, torch.einsum("ij,ij->i", a, hat) / n)
        if case["kind"] == "layer":
            inner -= (torch.einsum("ij->i", a) / n).unsqueeze(1)
        dx = torch.einsum("ij,i->ij", inner, inv)
        out = {"dx": dx + wide["dh"] if s["dh"] is not None else dx, "dw": torch.einsum("ij,ij->j", wide["dy"], hat)}
        if s["b"] is not None:
            out["db"] = torch.einsum("ij->j", wide["dy"])
        return out
    if op in ("loss", "loss_grad"):
        m, n = case["rows"], case["n"]
        l = torch.einsum("mk,nk->mn", wide["x"], wide["w"])
        lse = torch.logsumexp(l, 1)
        hot = torch.arange(m, device=DEVICE)[s["t"] != IGNORE]
        right = s["t"][hot]
        loss = torch.zeros_like(lse)
        loss[hot] = lse[hot] - l[hot, right]
        if op == "loss":
            return {"loss": loss, "lse": lse}
        weight = torch.zeros_like(lse)
        weight[hot] = wide["g"][hot]
        l.sub_(lse.unsqueeze(1)).exp_().mul_(weight.unsqueeze(1))
        l[hot, right] -= weight[hot]
        return {"loss": loss, "dx": torch.einsum("mn,nk->mk", l, wide["w"]), "dw": torch.einsum("mn,mk->nk", l, wide["x"])}
    b1, b2, t = _ADAM["beta1"], _ADAM["beta2"], 100
    g = wide["g"] * wide["scale"]
    if case["bits"] == 8:
        first, root = _table(3)[s["q1"].int() & 127], _table(4)[s["q2"].int()]
        first = torch.where(s["q1"] > 127, -first, first) * _unit64(s["e1"])
        second = (root * _unit64(s["e2"])).square()
    else:
        first, second = wide["m1"], wide["m2"]
    first = torch.lerp(g, first, b1)
    second = torch.lerp(g.square(), second, b2)
    root = second.sqrt()
    p = wide["p"] * (1 - _ADAM["lr"] * _ADAM["weight_decay"])
    p -= _ADAM["lr"] / (1 - b1 ** t) * first / (root / math.sqrt(1 - b2 ** t) + _ADAM["eps"])
    if case["bits"] == 32:
        return {"p": p, "m1": first, "m2": second}
    number = _dither(p.numel(), t, DEVICE)
    return {"p": p, "m1": first.sign() * _held64(first.abs(), number & 0xFFFF, 3, 16), "r": _held64(root, number >> 16, 4, 17)}


def _table(places):
    """The values of the codes of so many binary places, in units."""
    one = 1 << places
    return torch.tensor([float(c) if c < one else math.ldexp(one + c % one, c // one - 1) for c in range(16 * one)],
                        dtype=torch.float64, device=DEVICE)


def _power64(power):
    """2^power from its bits: a power function's last bit would move a border."""
    return ((power.to(torch.int64) + 1023) << 52).view(torch.float64)


def _unit64(e):
    return _power64(e.int() - 127).repeat_interleave(GROUP)


def _held64(v, number, places, less):
    """v >= 0 as 8 bits hold it, from the definition: the neighbour below or above, by the number's place between 0 and 1."""
    v = v.view(-1, GROUP)
    top = v.amax(1)
    power = (torch.frexp(top)[1] - 1 - less).clamp(min=-126)
    unit = _power64(power).unsqueeze(1)
    f = v / unit
    step = _power64((torch.frexp(f)[1] - 1 - places).clamp(min=0))
    u = (number.double().view(-1, GROUP) + 0.5) / 65536
    return (torch.floor(f / step + u) * step * unit).view(-1)
