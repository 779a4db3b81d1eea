"""A linear layer's products with what surrounds them, and activations saved in 8 bits, as cases.

The layers are those of the parameter lists in `paper_2609_33437_gb300.workloads`: a vision tower
(width 1024, MLP 4096, 257 tokens an image, patches of 588 values), a 7B decoder (4096, MLP 11008) and a
0.5B decoder (896, MLP 4864). Four operators:

  linear       y = act(x W^T + b) + r, and on request the pre-activation h = x W^T + b saved in 8 bits
  checkpoint   a tensor saved in 8 bits and read back, through an activation on request
  grad_input   dx = (dy W) * act'(h^), h^ read from its 8 bits
  grad_weight  dW = dy^T x^ and db = the sums of dy over rows; x^ read from 8 bits, through an activation
               on request, or x as it is; added to an older dW on request

8 bits: each row in groups of 32 columns (the last one may be shorter), a power of two 2^(e - 127) per
group and q = round(x / 2^(e - 127)), ties to even. 2^(e - 127) is the smallest power of two, from 2^-126
on, with which every |q| is at most 127. A value saved in 8 bits is returned as q 2^(e - 127), which bf16
holds exactly.
"""

import math

import torch

own = False

DEVICE = "cuda"
GROUP = 32
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ACTS = ("none", "relu", "gelu", "gelu_tanh", "quick_gelu", "silu")

# every key that a case can have, with the value that stands for "not said"
_DEFAULTS = dict(dtype="bf16", act="none", bias=False, residual=False, save=False, packed=False, accumulate=False)


# ----------------------------------------------------------------- the cases ---
def listed():
    return [
        # One token through the decoder's attention output, onto the residual stream: the smallest product,
        # where latency counts.
        _case("linear_token", "linear", rows=1, k=4096, n=4096, residual=True),
        # A few sequences decoded together through the gate projection.
        _case("linear_few_rows", "linear", rows=24, k=4096, n=11008, act="silu"),
        # Eight images through a tower's first MLP layer, its pre-activation saved for the backward pass.
        _case("linear_fc1_saved", "linear", rows=2056, k=1024, n=4096, bias=True, act="quick_gelu", save=True),
        # Sixteen images' patches: rows of 588 values, which no 16-byte boundary meets.
        _case("linear_patches", "linear", rows=4096, k=588, n=1024, bias=True),
        # Sixteen sequences of 512 tokens through the decoder's down projection: the largest call.
        _case("linear_down", "linear", rows=8192, k=11008, n=4096, residual=True),
        # The 0.5B list trains in fp32: an odd number of tokens through its gate projection.
        _case("linear_f32", "linear", rows=515, k=896, n=4864, dtype="f32", act="silu"),
        # The input of one tower layer saved and read back, one image: latency.
        _case("checkpoint_image", "checkpoint", rows=257, n=1024),
        # A decoder MLP's activations saved, and read back through the activation.
        _case("checkpoint_decoder", "checkpoint", rows=8191, n=11008, act="silu"),
        # Sixteen images back through a tower's second MLP layer and its activation.
        _case("grad_input_fc2", "grad_input", rows=4112, k=4096, n=1024, act="quick_gelu"),
        # One short sequence back through the 0.5B decoder's gate projection.
        _case("grad_input_short", "grad_input", rows=77, k=896, n=4864),
        # Thirty-two images: the second MLP layer's weight gradient, its input recomputed from the saved
        # pre-activation.
        _case("grad_weight_fc2", "grad_weight", rows=8224, k=4096, n=1024, bias=True, act="quick_gelu", packed=True),
        # A further micro-batch of an odd number of tokens added to a square projection's gradient.
        _case("grad_weight_more", "grad_weight", rows=4099, k=4096, n=4096, packed=True, accumulate=True),
    ]


def _case(name, op, **kw):
    return {"name": name, "op": op, **_DEFAULTS, **kw}


def _size(rng, low, high):
    """A size spread over its logarithm: odd ones, multiples of 8 and of 128."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice((1, 1, 8, 128))
    v = min(high, max(low, (v + step // 2) // step * step))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("linear", "linear", "checkpoint", "grad_input", "grad_weight"))
    c = dict(_DEFAULTS, op=op, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
    c["rows"] = _size(rng, 1, 8192)
    c["n"] = _size(rng, 64, 11008)
    if op == "checkpoint":
        c["act"] = rng.choice(("none", "none") + _ACTS[1:])
        return c
    c["k"] = _size(rng, 64, 11008)
    # at most a tenth of the largest listed product in fp32, which has no matrix instructions of its width
    most = 8192 * 11008 * 4096 // (10 if c["dtype"] == "f32" else 1)
    while c["rows"] * c["n"] * c["k"] > most:
        c["rows"] = max(1, c["rows"] * 2 // 3)
        c["n"] = max(64, c["n"] * 2 // 3)
    c["rows"] += c["rows"] == 3072
    c["n"] += c["n"] == 3072
    c["act"] = rng.choice(_ACTS)
    c["bias"] = op != "grad_input" and rng.random() < 0.6
    if op == "linear":
        c["residual"] = rng.random() < 0.4
        c["save"] = rng.random() < 0.4
    elif op == "grad_weight":
        c["packed"] = rng.random() < 0.6
        c["act"] = c["act"] if c["packed"] else "none"
        c["accumulate"] = rng.random() < 0.4
    return c


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
    dt, op, m, n = _TYPES[case["dtype"]], case["op"], case["rows"], case["n"]
    s = {"case": case}
    if op == "checkpoint":
        s["x"] = _stream(g, m, n).to(dt)
        return s
    k = case["k"]
    if op in ("linear", "grad_input"):
        s["w"] = (_normal(g, n, k) / math.sqrt(k)).to(dt)
    if op == "linear":
        s["x"] = _stream(g, m, k).to(dt)
        s["b"] = (0.1 * _normal(g, n)).to(dt) if case["bias"] else None
        s["r"] = _normal(g, m, n).to(dt) if case["residual"] else None
        return s
    s["dy"] = (1e-3 * _normal(g, m, n)).to(dt)
    if op == "grad_input":
        # the pre-activation of the layer before, as the forward pass saved it
        s["q"], s["e"] = _pack(1.5 * _normal(g, m, k)) if case["act"] != "none" else (None, None)
    else:
        x = _stream(g, m, k)
        s["x"], (s["q"], s["e"]) = (None, _pack(x)) if case["packed"] else (x.to(dt), (None, None))
        s["old"] = (1e-2 * _normal(g, n, k)).to(dt) if case["accumulate"] else None
    return s


# ------------------------------------------------------------ the plain forms ---
def _pack(x):
    """(q int8 [rows, cols], e uint8 [rows, groups]) of x, see the head of this file."""
    x = x.float()
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    v = torch.nn.functional.pad(x, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    top = v.abs().amax(-1)
    # the largest value's exponent less 6; one more where it would round to 128
    e = (((top.view(torch.int32) + 0x10000) >> 23) - 6).clamp(min=1)
    q = torch.round(v * (((254 - e) << 23).view(torch.float32)).unsqueeze(-1)).to(torch.int8)
    return q.view(rows, groups * GROUP)[:, :cols].contiguous(), e.to(torch.uint8)


def _unpack(q, e):
    scale = (e.to(torch.int32) << 23).view(torch.float32)
    return q.float() * scale.repeat_interleave(GROUP, 1)[:, :q.shape[1]]


def _act(name, h):
    if name == "relu":
        return torch.where(h > 0, h, torch.zeros_like(h))
    if name == "gelu":
        return 0.5 * h * (1.0 + torch.erf(h * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * h * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (h + 0.044715 * h * h * h)))
    if name == "quick_gelu":
        return h / (1.0 + torch.exp(-1.702 * h))
    if name == "silu":
        return h / (1.0 + torch.exp(-h))
    return h


def _act_grad(name, h):
    if name == "relu":
        return (h > 0).to(h.dtype)
    if name == "gelu":
        return (0.5 * (1.0 + torch.erf(h * math.sqrt(0.5)))
                + h * torch.exp(-0.5 * h * h) * (1.0 / math.sqrt(2.0 * math.pi)))
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (h + 0.044715 * h * h * h))
        return 0.5 * (1.0 + t) + 0.5 * h * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * h * h)
    if name in ("quick_gelu", "silu"):
        c = 1.702 if name == "quick_gelu" else 1.0
        s = 1.0 / (1.0 + torch.exp(-c * h))
        return s * (1.0 + c * h * (1.0 - s))
    return torch.ones_like(h)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["case"]
    dt, op = _TYPES[c["dtype"]], c["op"]
    if op == "linear":
        h = s["x"].float() @ s["w"].float().T
        if s["b"] is not None:
            h = h + s["b"].float()
        y = _act(c["act"], h)
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(dt), "saved": _unpack(*_pack(h)).to(torch.bfloat16)} if c["save"] else {"y": y.to(dt)}
    if op == "checkpoint":
        return {"x": _act(c["act"], _unpack(*_pack(s["x"]))).to(dt)}
    dy = s["dy"].float()
    if op == "grad_input":
        dx = dy @ s["w"].float()
        if c["act"] != "none":
            dx = dx * _act_grad(c["act"], _unpack(s["q"], s["e"]))
        return {"dx": dx.to(dt)}
    # the layer's input has its own type, whatever it was saved in
    x = _act(c["act"], _unpack(s["q"], s["e"])).to(dt).float() if c["packed"] else s["x"].float()
    dw = dy.T @ x
    if s["old"] is not None:
        dw = dw + s["old"].float()
    return {"dw": dw.to(dt), "db": dy.sum(0).to(dt)} if c["bias"] else {"dw": dw.to(dt)}


# ---------------------------------------------------- the framework's operators ---
def _run_own(s):
    from paper_2609_33437_gb300 import linear as L

    c = s["case"]
    dt, op = _TYPES[c["dtype"]], c["op"]
    if op == "linear":
        if not c["save"]:
            return {"y": L.linear(s["x"], s["w"], bias=s["b"], act=c["act"], residual=s["r"])}
        y, saved = L.linear(s["x"], s["w"], bias=s["b"], act=c["act"], residual=s["r"], save=True)
        return {"y": y, "saved": L.unpack8(saved, dtype=torch.bfloat16)}
    if op == "checkpoint":
        return {"x": L.unpack8(L.pack8(s["x"]), act=c["act"], dtype=dt)}
    if op == "grad_input":
        saved = L.Packed8(s["q"], s["e"]) if c["act"] != "none" else None
        return {"dx": L.linear_grad_input(s["dy"], s["w"], act=c["act"], saved=saved)}
    x = L.Packed8(s["q"], s["e"]) if c["packed"] else s["x"]
    # a gradient that is added to is the caller's buffer: a copy of it, so that the state can be used again
    out = s["old"].clone() if s["old"] is not None else None
    dw, db = L.linear_grad_weight(s["dy"], x, act=c["act"], bias=c["bias"], out=out, accumulate=c["accumulate"])
    return {"dw": dw, "db": db} if c["bias"] else {"dw": dw}


# ------------------------------------------------------------------- the work ---
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    m, n, op = case["rows"], case["n"], case["op"]
    if op == "checkpoint":
        eight = m * n + m * -(-n // GROUP)  # written, then read
        return {"bytes": 2 * b * m * n + 2 * eight, "flops": 0}
    k = case["k"]
    flops = 2.0 * m * n * k
    if op == "linear":
        moved = b * (m * k + n * k + m * n)
        moved += b * n * case["bias"] + b * m * n * case["residual"]
        if case["save"]:  # written, then read and returned as values
            moved += 2 * (m * n + m * -(-n // GROUP)) + 2 * m * n
    elif op == "grad_input":
        moved = b * (m * n + n * k + m * k)
        moved += (m * k + m * -(-k // GROUP)) if case["act"] != "none" else 0
    else:
        moved = b * (m * n + n * k) + (m * k + m * -(-k // GROUP) if case["packed"] else b * m * k)
        moved += b * n * case["bias"] + b * n * k * case["accumulate"]
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------- the definition, 64 bits ---
def exact(case, seed):
    s = prepare(case, seed)
    op, act = case["op"], case["act"]

    def wide(t):
        return None if t is None else t.double()

    if op == "checkpoint":
        return {"x": _value64(act, _saved64(wide(s["x"])))}
    if op == "linear":
        h = torch.einsum("mk,nk->mn", wide(s["x"]), wide(s["w"]))
        if s["b"] is not None:
            h += wide(s["b"])
        y = _value64(act, h)
        if s["r"] is not None:
            y = y + wide(s["r"])
        return {"y": y, "saved": _saved64(h)} if case["save"] else {"y": y}
    dy = wide(s["dy"])
    if op == "grad_input":
        dx = torch.einsum("mn,nk->mk", dy, wide(s["w"]))
        return {"dx": dx if act == "none" else dx * _slope64(act, _read64(s["q"], s["e"]))}
    x = wide(s["x"]) if s["x"] is not None else _value64(act, _read64(s["q"], s["e"]))
    dw = torch.einsum("mn,mk->nk", dy, x)
    if s["old"] is not None:
        dw += wide(s["old"])
    return {"dw": dw, "db": torch.einsum("mn->n", dy)} if case["bias"] else {"dw": dw}


def _saved64(x):
    """x as its 8 bits stand for it, from the definition: a power of two per group of 32."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    for a in range(0, cols, 4096):
        v = x[:, a:a + 4096]
        width = v.shape[1]
        spare = -width % GROUP
        v = torch.cat([v, v.new_zeros(rows, spare)], 1).reshape(rows, -1, GROUP)
        top = v.abs().max(-1, keepdim=True).values
        _, power = torch.frexp(top)  # top < 2^power
        step = _power64((power - 7).clamp(min=-126))
        step = torch.where(torch.round(top / step) > 127, 2 * step, step)
        out[:, a:a + 4096] = (torch.round(v / step) * step).reshape(rows, -1)[:, :width]
    return out


def _read64(q, e):
    power = e.to(torch.int32) - 127
    power = power[:, torch.arange(q.shape[1], device=q.device) // GROUP]
    return q.double() * _power64(power)


def _power64(power):
    """2^power from its bits: a power function's last bit would move ties."""
    return ((power.to(torch.int64) + 1023) << 52).view(torch.float64)


def _value64(act, h):
    if act == "none":
        return h
    if act == "relu":
        return h.clamp(min=0)
    if act == "gelu":
        return h * torch.special.ndtr(h)
    if act == "gelu_tanh":
        return h * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3))
    return h * torch.sigmoid((1.702 if act == "quick_gelu" else 1.0) * h)


def _slope64(act, h):
    if act == "relu":
        return torch.heaviside(h, torch.zeros_like(h))
    if act == "gelu":
        return torch.special.ndtr(h) + h * torch.exp(-h * h / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(c * (h + 0.044715 * h ** 3))
        return s + h * s * (1 - s) * c * (1 + 3 * 0.044715 * h ** 2)
    c = 1.702 if act == "quick_gelu" else 1.0
    s = torch.sigmoid(c * h)
    return s + c * h * s * (1 - s)
