"""The AdamW step over many tensors on the GPU (include/smat.h, "AdamW"): bit for bit against the definition in fp32
(`_adamw_ref`), against 64 bits with every rounding counted, over ragged lists, both types and widths of moments, addresses off
every boundary, gradients that are missing, special values, what the device holds, graphs, long lists and long tensors; the
optimizer class, its state, and the periodic schedule around it."""

import copy

import numpy as np
import pytest
import torch

import _adamw_ref as A
from paper_2609_33437_gb300 import optim as O
from paper_2609_33437_gb300 import smat as S

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SIZES = [1, 255, 256, 257, 0, 1000, 7, 4099, 512, 2048, 70001, 3]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def _tensors(seed, sizes, dtype, scale, off=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n in sizes:
        t = torch.empty(n + off, device="cuda", dtype=dtype)[off:]
        t.copy_(torch.randn(n, generator=g, device="cuda") * torch.exp(2 * torch.randn(n, generator=g, device="cuda")) * scale)
        out.append(t)
    return out


def _flat(ts, sizes):
    """fp32 numpy by place, 0 between tensors."""
    at, total = A.starts(sizes)
    out = np.zeros(total, np.float32)
    for a, n, t in zip(at, sizes, ts):
        if t is not None:
            out[a:a + n] = t.float().cpu().numpy()
    return out


def _there(sizes, given):
    at, total = A.starts(sizes)
    out = np.zeros(total, bool)
    for a, n, t in zip(at, sizes, given):
        out[a:a + n] = t is not None
    return out


def _same(a, b):
    a, b = np.asarray(a), np.asarray(b)
    return a.shape == b.shape and bool(((a == b) | (np.isnan(a) & np.isnan(b))).all())


class Model:
    """The list and its moments on the CPU, stepped by the definition."""

    def __init__(self, sizes, bits):
        self.sizes, self.bits = sizes, bits
        _, total = A.starts(sizes)
        if bits == 8:
            z = np.zeros(total, np.uint8)
            self.state = [z, np.ones(total // A.GROUP, np.uint8), z.copy(), np.ones(total // A.GROUP, np.uint8)]
        else:
            self.state = [np.zeros(total, np.float32), np.zeros(total, np.float32)]

    def step(self, params, grads, t, seed=0, scale=1.0, **hyper):
        """The parameters as they will be, by place, in fp32 before their rounding; the state is stepped."""
        there = _there(self.sizes, grads)
        groups = there.reshape(-1, A.GROUP).any(1)
        p, g = _flat(params, self.sizes), _flat(grads, self.sizes)
        if self.bits == 8:
            m1, r = (v.astype(np.float32) for v in A.unpack(*self.state))
            m2 = r * r
        else:
            m1, m2 = self.state
        c = A.constants(t, **hyper)
        q, m1, m2, r = A.step(p, g, m1, m2, c, scale)
        with np.errstate(all="ignore"):
            self.taken = np.abs(c["step"] * (m1 / (r / c["bc2"] + c["eps"])))
        zero = np.float32(0)
        if self.bits == 8:
            new = A.pack(np.where(there, m1, zero), np.where(there, r, zero), t, seed)
            wide = np.repeat(groups, A.GROUP)
            self.state = [np.where(wide if n.size == wide.size else groups, n, o) for n, o in zip(new, self.state)]
        else:
            self.state = [np.where(there, n, o) for n, o in zip((m1, m2), self.state)]
        return q, there

    def check(self, params, moments, want, there, dtype):
        got = _flat(params, self.sizes)
        exact = want.astype(np.float64)
        want = torch.from_numpy(want).to(dtype).float().numpy()
        bad = ~((got == want) | (np.isnan(got) & np.isnan(want))) & there
        if self.bits == 8:
            # what is subtracted is off by 3 units in its last place (a reciprocal's 1, three roundings), the definition's by its
            # own four roundings, 2 units; either difference is rounded in fp32, and the kernel's to the type
            with np.errstate(all="ignore"):
                off = 5 * 2.0 ** -23 * self.taken + 2.0 ** -23 * np.abs(exact)
                bad &= ~(np.abs(got - exact) <= off + (2.0 ** -8 if dtype == BF else 0.0) * (np.abs(exact) + off))
        assert not bad.any(), f"{bad.sum()} parameters, first at {np.nonzero(bad)[0][0]}: {got[bad][0]} for {want[bad][0]}"
        for (name, b), ref in zip(moments.buffers().items(), self.state):
            b = b.cpu().numpy()
            assert _same(b, ref), f"{name}: {(b != ref).sum()} off, first at {np.nonzero(b != ref)[0][:1]}"


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dt,gt", [(F32, F32), (BF, BF), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("off", [0, 1, 8])
def test_steps_bit_for_bit(bits, dt, gt, off):
    params = _tensors(0, SIZES, dt, 0.1, off)
    moments, model = O.Moments(params, bits=bits), Model(SIZES, bits)
    for t in (1, 2, 3):
        grads = _tensors(10 + t, SIZES, gt, 1e-3, off if t > 1 else 0)
        want, there = model.step(params, grads, t, seed=5 << 33 | 17, scale=0.5, **HYPER)
        O.adamw(params, grads, moments, t, seed=5 << 33 | 17, scale=0.5, **HYPER)
        model.check(params, moments, want, there, dt)
    if bits == 8:
        m1, r = moments.values()
        for got, ref in zip((m1, r), A.unpack(*model.state)):
            assert _same(got.double().cpu().numpy(), ref)
        assert sum(t.numel() * t.element_size() for t in moments.buffers().values()) == moments.nbytes() <= 2.01 * moments.places
    else:
        assert moments.values()[0] is moments.buffers()["m1"]


def test_against_64_bits():
    """Every operation rounds by 2^-24 of its result at most, and the constants by as much."""
    sizes = [70001, 300]
    params, grads = _tensors(0, sizes, F32, 0.1), _tensors(1, sizes, F32, 1e-3)
    moments = O.Moments(params)
    m1, m2 = moments.values()
    m1.copy_(torch.randn(m1.numel(), device="cuda") * 1e-3)
    m2.copy_(torch.rand(m1.numel(), device="cuda") * 1e-6)
    p, g, a, b = (v.astype(np.float64) for v in (_flat(params, sizes), _flat(grads, sizes), m1.cpu().numpy(), m2.cpu().numpy()))
    O.adamw(params, grads, moments, 7, scale=0.25, **HYPER)
    u, h = 2.0 ** -24, HYPER
    g = g * 0.25
    x, y = h["beta1"] * a, (1 - h["beta1"]) * g
    m = x + y
    e_m = 4 * u * (abs(x) + abs(y))
    v = h["beta2"] * b + (1 - h["beta2"]) * g * g
    d = np.sqrt(v) / np.sqrt(1 - h["beta2"] ** 7) + h["eps"]
    k = h["lr"] / (1 - h["beta1"] ** 7)
    want = p * (1 - h["lr"] * h["weight_decay"]) - k * m / d
    tol = 4 * u * abs(p) + k * (e_m / d + 10 * u * abs(m) / d)  # v: 5 roundings, half of them left by the root; r, / bc2, + eps
    there = _there(sizes, params)
    for got, ref, e in ((_flat(params, sizes), want, tol), (m1.cpu().numpy(), m, e_m), (m2.cpu().numpy(), v, 6 * u * v)):
        assert bool((abs(got - ref) <= 1.01 * e + 1e-40)[there].all())


@pytest.mark.parametrize("bits", [8, 32])
def test_missing_gradients_and_what_lies_beside(bits):
    """Tensors without a gradient, their moments, and the elements beside a tensor stay as they are."""
    sizes = [300, 5, 0, 1024, 77, 256]
    whole = [torch.full((n + 16,), 7.0, device="cuda", dtype=BF) for n in sizes]
    params = [w[8:8 + n] for w, n in zip(whole, sizes)]
    moments, model = O.Moments(params, bits=bits), Model(sizes, bits)
    for t, skip in ((1, ()), (2, (0, 3)), (3, (5,)), (4, (1, 4)), (5, range(6))):
        grads = [None if k in skip else g for k, g in enumerate(_tensors(t, sizes, F32, 1e-2))]
        want, there = model.step(params, grads, t, **HYPER)
        O.adamw(params, grads, moments, t, **HYPER)
        model.check(params, moments, want, there, BF)
    for w, n in zip(whole, sizes):
        assert bool((w[:8] == 7).all()) and bool((w[8 + n:] == 7).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_special_values(bits):
    """Zeros, subnormal and huge gradients; an infinity or NaN is seen in its element, and in 8 bits in its group."""
    sizes = [600, 256]
    params = _tensors(0, sizes, F32, 1.0)
    moments, model = O.Moments(params, bits=bits), Model(sizes, bits)
    for t, plant in ((1, {}), (2, {3: 1e-42, 4: -1e-30, 5: 1e18, 300: -1e-44}), (3, {10: float("inf")}), (4, {400: float("nan")}),
                     (5, {})):
        grads = [torch.zeros(n, device="cuda") for n in sizes]
        for i, v in plant.items():
            grads[0][i] = v
        want, there = model.step(params, grads, t, **HYPER)
        O.adamw(params, grads, moments, t, **HYPER)
        model.check(params, moments, want, there, F32)
    m1 = moments.values()[0][:600].float()
    if bits == 8:
        assert bool(m1[:512].isnan().all()) and not bool(m1[512:].isnan().any())
    else:
        assert int((~torch.isfinite(m1)).sum()) == 2
    assert bool(torch.isfinite(moments.values()[0][768:].float()).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_many_tensors(bits):
    """More tensors than one launch takes."""
    sizes = [1 + k % 5 * 80 for k in range(2701)]
    params, grads = _tensors(0, sizes, BF, 0.1), _tensors(1, sizes, BF, 1e-3)
    moments, model = O.Moments(params, bits=bits), Model(sizes, bits)
    want, there = model.step(params, grads, 1, seed=3, **HYPER)
    O.adamw(params, grads, moments, 1, seed=3, **HYPER)
    model.check(params, moments, want, there, BF)


@pytest.mark.parametrize("bits", [8, 32])
def test_what_the_device_holds(bits):
    """step, lr and scale on the device: as the same numbers from the host, and read anew by a replay."""
    sizes = [1000, 33]
    start, grads = _tensors(0, sizes, F32, 0.1), _tensors(1, sizes, F32, 1e-3)
    hyper = {k: v for k, v in HYPER.items() if k != "lr"}
    lr, scale = torch.full((), 0.0078125, device="cuda"), torch.full((1,), 0.5, device="cuda")
    one, two = ([t.clone() for t in start] for _ in range(2))
    m_one, m_two = O.Moments(one, bits=bits), O.Moments(two, bits=bits)
    step = torch.ones((), dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # captured, not run
        O.adamw(two, grads, m_two, step, lr=lr, scale=scale, seed=9, **hyper)
        step.add_(1)
    for t in (1, 2, 3):
        O.adamw(one, grads, m_one, t, lr=0.0078125 * t, scale=0.5, seed=9, **hyper)
        lr.fill_(0.0078125 * t)
        graph.replay()
    assert int(step) == 4
    # the constants are made in double on either side and rounded once: off by a unit in the last place at most where the two
    # functions differ, and a byte by a step
    for a, b in zip(one, two):
        assert float((a - b).abs().max()) <= 3 * 2.0 ** -22 * 0.03 + 2.0 ** -23 * float(a.abs().max())
    if bits == 32:
        for a, b in zip(m_one.values(), m_two.values()):
            assert torch.equal(a, b)
    three, m_three = [t.clone() for t in start], O.Moments(start, bits=bits)
    O.adamw(three, grads, m_three, 1, lr=lr, scale=0.5, seed=9, **hyper)
    four, m_four = [t.clone() for t in start], O.Moments(start, bits=bits)
    O.adamw(four, grads, m_four, 1, lr=float(lr), scale=0.5, seed=9, **hyper)
    assert all(torch.equal(a, b) for a, b in zip(three, four))


def test_streams_and_repeats():
    sizes = [4096, 100]
    start, grads = _tensors(0, sizes, BF, 0.1), _tensors(1, sizes, BF, 1e-3)
    outs = []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, side):
        p = [t.clone() for t in start]
        m = O.Moments(p, bits=8)
        torch.cuda.synchronize()
        for t in (1, 2):
            O.adamw(p, grads, m, t, stream=stream, **HYPER)
        v = m.values(stream=stream)
        torch.cuda.synchronize()
        outs.append((*p, *v))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_long_tensor_in_8_bits():
    """Places past 2^31 and offsets past 32 bits: the ends of a long tensor and the tensor after it."""
    n = (1 << 31) + 777
    big, small = torch.zeros(n, device="cuda", dtype=BF), torch.zeros(100, device="cuda", dtype=BF)
    grad, gsmall = torch.zeros(n, device="cuda", dtype=BF), _tensors(2, [100], BF, 1e-3)[0]
    tail = _tensors(1, [5000], BF, 1e-3)[0]
    grad[-5000:] = tail
    moments = O.Moments([big, small], bits=8)
    O.adamw([big, small], [grad, gsmall], moments, 1, seed=4, **HYPER)
    first = (n - 5000) // A.GROUP * A.GROUP
    g = np.zeros(moments.places - first, np.float32)
    g[n - 5000 - first:n - first] = tail.float().cpu().numpy()
    g[moments.starts[1] - first:moments.starts[1] - first + 100] = gsmall.float().cpu().numpy()
    z = np.zeros_like(g)
    p, m1, _, r = A.step(z, g, z, z, A.constants(1, **HYPER))
    for (name, b), ref in zip(moments.buffers().items(), A.pack(m1, r, 1, 4, first)):
        assert _same(b[-ref.size:].cpu().numpy(), ref), name
    got = torch.cat([big[first:], torch.zeros(moments.starts[1] - n, device="cuda", dtype=BF), small]).cpu()
    want = torch.from_numpy(p[:got.numel()]).double()
    assert bool(((got.double() - want).abs() <= (2.0 ** -8 + 7 * 2.0 ** -23) * want.abs()).all())  # see Model.check
    assert not bool(big[:1 << 20].any()) and int(moments.buffers()["q1"][:first].max()) == 0


def test_optimizer_matches_torch():
    """optim.AdamW against torch.optim.AdamW in fp32: the same formula, a few roundings apart after ten steps."""
    torch.manual_seed(0)
    a = [torch.nn.Parameter(torch.randn(33, 7, device="cuda")), torch.nn.Parameter(torch.randn(40, device="cuda"))]
    b = [torch.nn.Parameter(t.detach().clone()) for t in a]
    groups = lambda ps: [dict(params=ps[:1], weight_decay=0.1), dict(params=ps[1:], lr=3e-3)]  # noqa: E731
    mine, ref = O.AdamW(groups(a), lr=1e-2), torch.optim.AdamW(groups(b), lr=1e-2)
    for t in range(10):
        for p, q in zip(a, b):
            q.grad = torch.randn_like(q)
            p.grad = q.grad.clone()
        mine.step()
        ref.step()
    for p, q in zip(a, b):
        # ten steps of at most lr each, with about 12 roundings a step of their size, and two a step of the parameter
        assert float((p - q).abs().max()) <= 10 * (12 * 1e-2 + 2 * 4.0) * 2.0 ** -24


@pytest.mark.parametrize("bits", [8, 32])
def test_optimizer_state_goes_on(bits):
    """A saved and loaded state goes on with the same bits; mixed types make a list each."""
    def make():
        torch.manual_seed(1)
        return [torch.nn.Parameter(torch.randn(300, device="cuda")), torch.nn.Parameter(torch.randn(4, 5, device="cuda").to(BF))]

    def grads(ps, t):
        g = torch.Generator(device="cuda").manual_seed(t)
        for p in ps:
            p.grad = torch.randn(p.shape, generator=g, device="cuda").to(p.dtype)

    one = make()
    opt = O.AdamW(one, lr=1e-2, bits=bits, seed=3)
    for t in range(4):
        grads(one, t)
        opt.step()
        if t == 1:
            saved = {k: v for k, v in opt.state_dict().items()}
            saved["moments"] = [{k: v.cpu().clone() if torch.is_tensor(v) else v for k, v in m.items()} for m in saved["moments"]]
            two = [torch.nn.Parameter(p.detach().clone()) for p in one]
    assert len(opt.lists()) == 2
    again = O.AdamW(two, lr=1.0, bits=bits)
    again.load_state_dict(saved)
    for t in (2, 3):
        grads(two, t)
        again.step()
    assert all(torch.equal(p, q) for p, q in zip(one, two)) and again.steps == 4
    with pytest.raises(ValueError, match="other"):
        O.AdamW(two, bits=40 - bits).load_state_dict(saved)


def test_a_graph_that_saved_a_parameter_notices():
    w = torch.nn.Parameter(torch.randn(8, 8, device="cuda"))
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    loss = (x @ w).sum()
    w.grad = torch.ones_like(w)
    O.AdamW([w]).step()
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()


@pytest.mark.parametrize("dt", [F32, BF])
def test_schedule_takes_the_step_into_the_gradient_map(dt):
    """PeriodicSmat.optimizer_step with an AdamW of 32 bits: the same bits as the mapped gradient and a step of its own (the
    hyperparameters are powers of two, which the two calls' constants agree on)."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    def run(fused):
        torch.manual_seed(2)
        params = [torch.nn.Parameter((torch.randn(n, device="cuda") * 0.1).to(dt)) for n in (700, 64)]
        theta0 = [(p.detach() + 0.01).to(dt) for p in params]
        sched = PeriodicSmat(params, [0.5, 1.0], [1e-3] * 2, theta0=theta0, period=2, seed=1, alpha_min=0.5, alpha_max=1.0,
                             alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
        opt = O.AdamW(params, lr=2.0 ** -9, betas=(0.5, 0.75), eps=2.0 ** -20, weight_decay=2.0 ** -4)
        for step in range(4):
            sched.before_forward(step)
            sum((p.float() ** 2).sum() for p in params).backward()
            if fused:
                sched.optimizer_step(step, opt)
            else:
                sched.after_backward(step)
                opt.step()
            opt.zero_grad()
        assert opt.steps == 4
        sched.close()
        return [p.detach().clone() for p in params] + [v.clone() for v in opt.lists()[0][2].values()]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


@pytest.mark.parametrize("bits", [8, 32])
def test_moments_moved_away_and_back(bits):
    """Buffers taken to the host and back, and given other storage: the step goes on with the bits of one that stayed."""
    sizes = [700, 33]
    start = _tensors(0, sizes, F32, 0.1)
    lists, kept = [], []
    for moved in (False, True):
        params = [t.clone() for t in start]
        moments = O.Moments(params, bits=bits)
        for t in (1, 2, 3):
            O.adamw(params, _tensors(t, sizes, F32, 1e-3), moments, t, **HYPER)
            if moved:
                for b in moments.buffers().values():
                    kept.append(b.data)  # nobody else gets its place: a step that went there would be seen
                    b.data = b.data.cpu()
                with pytest.raises(ValueError, match="moments"):
                    O.adamw(params, params, moments, t + 1, **HYPER)
                for b in moments.buffers().values():
                    b.data = b.data.cuda()
        lists.append([*params, *moments.buffers().values()])
    assert all(torch.equal(a, b) for a, b in zip(*lists))


def test_a_parameter_without_a_gradient_is_untouched():
    """The step leaves it as it is: a graph that saved it goes on."""
    w, v = torch.nn.Parameter(torch.randn(8, 8, device="cuda")), torch.nn.Parameter(torch.randn(8, 8, device="cuda"))
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    loss = (x @ w).sum()
    v.grad = torch.ones_like(v)
    versions = w._version, v._version
    O.AdamW([w, v]).step()
    assert w._version == versions[0] and v._version > versions[1]
    loss.backward()
    assert torch.equal(x.grad, torch.ones(4, 8, device="cuda") @ w.detach().T)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("why", ["eps of 0", "a gradient in its parameter's place", "a parameter that is not contiguous"])
def test_a_refused_step_moves_nothing(why, bits):
    """What is refused of a later list leaves the first as it was; the step is then as if it had been the first try."""
    def make():
        torch.manual_seed(3)
        ps = [torch.nn.Parameter(torch.randn(300, device="cuda")), torch.nn.Parameter(torch.randn(16, 5, device="cuda").to(BF)),
              torch.nn.Parameter(torch.randn(70, device="cuda").to(BF))]
        return ps, O.AdamW([dict(params=ps[:1]), dict(params=ps[1:])], lr=1e-2, bits=bits, seed=5)

    def grads(ps, t):
        g = torch.Generator(device="cuda").manual_seed(t)
        for p in ps:
            p.grad = torch.randn(p.shape, generator=g, device="cuda").to(p.dtype)

    ends = []
    for interrupted in (False, True):
        ps, opt = make()
        for t in (1, 2):
            grads(ps, t)
            if interrupted:
                before = [p.detach().clone() for p in ps] + [b.clone() for _, _, m in opt.lists() for b in m.buffers().values()]
                was = ps[1].data, opt.param_groups[1]["eps"], ps[2].grad
                if why == "eps of 0":
                    opt.param_groups[1]["eps"] = 0.0
                elif why == "a gradient in its parameter's place":
                    ps[2].grad = ps[2].data
                else:
                    ps[1].data = torch.randn(5, 16, device="cuda").to(BF).t()
                with pytest.raises((ValueError, S.SmatError)):
                    opt.step()
                ps[1].data, opt.param_groups[1]["eps"], ps[2].grad = was
                after = [p.detach().clone() for p in ps] + [b.clone() for _, _, m in opt.lists() for b in m.buffers().values()]
                assert opt.steps == t - 1 and all(torch.equal(a, b) for a, b in zip(before, after))
            opt.step()
        ends.append([p.detach().clone() for p in ps] + [b for _, _, m in opt.lists() for b in m.buffers().values()])
    assert all(torch.equal(a, b) for a, b in zip(*ends))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_first_gradient_that_comes_late(bits):
    """Each parameter's step count is of its own gradients: a late one moves as it would by itself, and as with torch's."""
    def make():
        torch.manual_seed(4)
        return [torch.nn.Parameter(torch.randn(300, device="cuda")) for _ in range(3)]

    def grad(t, i):
        g = torch.Generator(device="cuda").manual_seed(10 * t + i)
        return torch.randn(300, generator=g, device="cuda")

    there = lambda t, i: i == 0 or (i == 1 and t > 6) or (i == 2 and t % 3 == 0)  # noqa: E731
    together, ref = make(), make()
    opt, theirs = O.AdamW(together, lr=1e-2, bits=bits), torch.optim.AdamW(ref, lr=1e-2)
    for t in range(1, 13):
        for i in range(3):
            together[i].grad = grad(t, i) if there(t, i) else None
            ref[i].grad = grad(t, i) if there(t, i) else None
        opt.step()
        theirs.step()
    assert opt.steps == 12 and opt.counts == [[12, 6, 4]]
    state = opt.state_dict()
    assert state["counts"] == [[12, 6, 4]]
    if bits == 32:
        for p, q in zip(together, ref):  # see test_optimizer_matches_torch
            assert float((p - q).abs().max()) <= 12 * (12 * 1e-2 + 2 * 4.0) * 2.0 ** -24
        for i in range(3):
            alone = make()[i]
            one = O.AdamW([alone], lr=1e-2)
            for t in range(1, 13):
                if there(t, i):
                    alone.grad = grad(t, i)
                    one.step()
            assert torch.equal(alone, together[i])
    else:
        # a first step is one of lr, whenever it comes
        alone = make()
        late = O.AdamW(alone, lr=1e-2, bits=8, weight_decay=0.0)
        for t in range(1, 4):
            alone[0].grad = grad(t, 0)
            late.step()
        alone[1].grad, before = grad(9, 1), alone[1].detach().clone()
        late.step()
        assert float(((alone[1] - before).abs() - 1e-2).abs().max()) < 1e-5
    again = O.AdamW(together, bits=bits)
    again.load_state_dict(state)
    assert again.counts == [[12, 6, 4]]
    old = {k: v for k, v in state.items() if k != "counts"}
    again.load_state_dict(old)
    assert again.counts == [[12, 12, 12]]


def test_schedule_with_step_counts_apart():
    """A parameter whose gradients began later: the fused step has one count for all and is not taken."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    def run(fused):
        torch.manual_seed(5)
        params = [torch.nn.Parameter(torch.randn(n, device="cuda") * 0.1) for n in (700, 64)]
        theta0 = [p.detach() + 0.01 for p in params]
        sched = PeriodicSmat(params, [0.5, 1.0], [1e-3] * 2, theta0=theta0, period=2, seed=1, alpha_min=0.5, alpha_max=1.0,
                             alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
        opt = O.AdamW(params, lr=1e-2)
        for step in range(4):
            sched.before_forward(step)
            sum((p.float() ** 2).sum() for p in (params[:1] if step == 0 else params)).backward()
            if fused:
                sched.optimizer_step(step, opt)
            else:
                sched.after_backward(step)
                opt.step()
            opt.zero_grad()
        assert opt.steps == 4 and opt.counts == [[4, 3]]
        sched.close()
        return [p.detach().clone() for p in params] + [v.clone() for v in opt.lists()[0][2].values()]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_copy_goes_on(bits):
    """A deep copy of a model and its optimizer goes on with the same bits, each with its own state."""
    ps = [torch.nn.Parameter(p) for p in _tensors(0, [300, 40], F32, 0.1)]
    opt = O.AdamW(ps, lr=1e-2, bits=bits, seed=2)
    for t in (1, 2):
        for p, g in zip(ps, _tensors(t, [300, 40], F32, 1e-3)):
            p.grad = g
        opt.step()
    qs, new = copy.deepcopy((ps, opt))
    for params, o in ((ps, opt), (qs, new)):
        for p, g in zip(params, _tensors(3, [300, 40], F32, 1e-3)):
            p.grad = g
        o.step()
    assert new.counts == opt.counts == [[3, 3]] and all(torch.equal(p, q) and p is not q for p, q in zip(ps, qs))
    for a, b in zip(opt.lists()[0][2].buffers().values(), new.lists()[0][2].buffers().values()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_group_added_between_steps(bits):
    """A layer that is trained from a later step on: it and what was there move as with torch's optimizer."""
    torch.manual_seed(6)
    ps = [torch.nn.Parameter(torch.randn(300, device="cuda")) for _ in range(2)]
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    opt, ref = O.AdamW(ps[:1], lr=1e-2, bits=bits), torch.optim.AdamW(qs[:1], lr=1e-2)
    for t in range(1, 7):
        if t == 3:
            opt.add_param_group(dict(params=ps[1:], lr=5e-3))
            ref.add_param_group(dict(params=qs[1:], lr=5e-3))
        for p, q, g in zip(ps, qs, _tensors(t, [300, 300], F32, 1.0)):
            p.grad, q.grad = g.clone(), g.clone()
        opt.step()
        ref.step()
    assert opt.counts == [[6], [4]]
    # 32 bits: see test_optimizer_matches_torch; 8 bits: m1 and r are held to a step of 1/16 and 1/32 of their size, or of a group's
    # largest / 2^16, so that an update, at most lr (1 - beta1) / sqrt(1 - beta2) = 3.2 lr, is off by 10% at most after each step
    for p, q in zip(ps, qs):
        tol = 6 * (12 * 1e-2 + 2 * 4.0) * 2.0 ** -24 if bits == 32 else 6 * 0.1 * 3.2e-2
        assert float((p - q).abs().max()) <= tol


@pytest.mark.parametrize("make", [O.AdamW, torch.optim.AdamW])
def test_a_graph_notices_the_fused_step(make):
    """The step inside the gradient map raises the parameters' version, as an optimizer's own step does."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    w = torch.nn.Parameter(torch.randn(8, 8, device="cuda"))
    sched = PeriodicSmat([w], [0.5], [1e-3], theta0=[w.detach() + 0.01], period=1, seed=1, alpha_min=0.5, alpha_max=1.0,
                         alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
    opt = make([w], lr=1e-2)
    sched.before_forward(0)
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    loss = (x @ w).sum()
    w.grad = torch.ones_like(w)
    fused, session = [], sched.session
    call = session.grad_map_adamw_multi
    session.grad_map_adamw_multi = lambda *a, **k: (fused.append(1), call(*a, **k))
    sched.optimizer_step(0, opt)
    assert fused == [1]
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()
    sched.close()


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("hyper", [dict(lr=1e-3), dict(lr=3e-4, betas=(0.9, 0.95), eps=1e-6, weight_decay=0.1)])
def test_fused_step_has_the_list_steps_constants(hyper, dt):
    """With hyperparameters that fp32 does not hold: the gradient map with the step inside, and the map and a step of its own, the
    same bits, over steps of either kind."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    def run(fused):
        torch.manual_seed(2)
        params = [torch.nn.Parameter((torch.randn(n, device="cuda") * 0.1).to(dt)) for n in (7000, 64)]
        theta0 = [(p.detach() + 0.01).to(dt) for p in params]
        sched = PeriodicSmat(params, [0.5, 1.0], [1e-3] * 2, theta0=theta0, period=2, seed=1, alpha_min=0.5, alpha_max=1.0,
                             alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
        opt = O.AdamW(params, **hyper)
        for step in range(6):
            sched.before_forward(step)
            sum((p.float() ** 2).sum() for p in params).backward()
            if fused:
                sched.optimizer_step(step, opt)
            else:
                sched.after_backward(step)
                opt.step()
            opt.zero_grad()
        sched.close()
        return [p.detach().clone() for p in params] + [v.clone() for v in opt.lists()[0][2].values()]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


def test_fused_step_in_double_refuses():
    theta = [torch.ones(300, device="cuda")]
    sim, theta0, g, m1, m2 = ([torch.full((300,), v, device="cuda")] for v in (0.0, 0.5, 1.0, 0.0, 0.0))
    session = S.SmatSession(theta, theta0, sim, [0.5], [1e-3])
    session.simulate_multi(0)
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, adam_step=1)
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=1e39), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-39),
                dict(weight_decay=-1.0), dict(adam_step=0), dict(adam_step=1 << 31)):
        with pytest.raises(S.SmatError):
            session.grad_map_adamw_multi(0, g, m1, m2, **{**good, **bad}, double=True)
    assert bool((theta[0] == 1).all()) and not bool(m1[0].any())
    session.grad_map_adamw_multi(0, g, m1, m2, **good, double=True)
    assert bool((theta[0] != 1).any()) and bool(m1[0].any())
    session.close()


@pytest.mark.parametrize("make", [O.AdamW, torch.optim.AdamW])
def test_a_refused_fused_step_may_be_tried_again(make):
    """The parameters' storage and the optimizer are as before the refusal, and the step is then as at the first try."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    def run(refused):
        torch.manual_seed(2)
        params = [torch.nn.Parameter(torch.randn(n, device="cuda") * 0.1) for n in (700, 64)]
        sched = PeriodicSmat(params, [0.5, 1.0], [1e-3] * 2, theta0=[p.detach() + 0.01 for p in params], period=2, seed=1,
                             alpha_min=0.5, alpha_max=1.0, alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
        opt = make(params, lr=1e-2)
        for step in range(4):
            sched.before_forward(step)
            sum((p.float() ** 2).sum() for p in params).backward()
            if refused and step % 2:
                there = [p.data_ptr() for p in params]
                opt.param_groups[0]["eps"] = 0.0
                with pytest.raises(S.SmatError):
                    sched.optimizer_step(step, opt)
                opt.param_groups[0]["eps"] = 1e-8
                assert [p.data_ptr() for p in params] == there
            sched.optimizer_step(step, opt)
            opt.zero_grad()
        sched.close()
        return [p.detach().clone() for p in params]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


def test_schedule_around_moments_in_8_bits():
    """The fused step holds 32 bits: on a simulated-loss step the gradient is mapped and an AdamW of 8 bits makes a step of its own."""
    from paper_2609_33437_gb300.schedule import PeriodicSmat

    def run(by_schedule):
        torch.manual_seed(2)
        params = [torch.nn.Parameter((torch.randn(n, device="cuda") * 0.1).to(BF)) for n in (700, 64)]
        sched = PeriodicSmat(params, [0.5, 1.0], [1e-3] * 2, theta0=[(p.detach() + 0.01).to(BF) for p in params], period=2, seed=1,
                             alpha_min=0.5, alpha_max=1.0, alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
        opt = O.AdamW(params, lr=1e-2, bits=8, seed=3)
        for step in range(4):
            sched.before_forward(step)
            sum((p.float() ** 2).sum() for p in params).backward()
            if by_schedule:
                sched.optimizer_step(step, opt)
            else:
                sched.after_backward(step)
                opt.step()
            opt.zero_grad()
        assert opt.steps == 4 and opt.counts == [[4, 4]]
        sched.close()
        return [p.detach().clone() for p in params] + list(opt.lists()[0][2].buffers().values())

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("device", [False, True])
def test_optimizer_step_scale_closure_and_strided_gradients(device, bits):
    """A scale, gradients that are not contiguous and a closure: the bits of the call with these gradients."""
    start, g = torch.randn(24, 40, device="cuda"), torch.randn(40, 24, device="cuda")
    p = torch.nn.Parameter(start.clone())
    opt = O.AdamW([p], lr=1e-2, bits=bits, seed=9)
    scale = torch.full((1,), 0.25, device="cuda") if device else 0.25

    def closure():
        assert torch.is_grad_enabled()
        p.grad = g.t()
        return torch.tensor(3.0)

    q, moments = start.clone(), O.Moments([start], bits=bits)
    for t in (1, 2, 3):
        assert float(opt.step(closure, scale=scale)) == 3.0
        assert not p.grad.is_contiguous() and torch.equal(p.grad, g.t())
        O.adamw([q], [g.t().contiguous()], moments, t, lr=1e-2, scale=0.25, seed=9)
        assert torch.equal(p.detach(), q)
    for a, b in zip(opt.lists()[0][2].buffers().values(), moments.buffers().values()):
        assert torch.equal(a, b)
