"""CPU-only checks of the AdamW step over many tensors: what the C ABI and the binding refuse before anything reaches a GPU
(pointers here are numbers; none is read), and the 8-bit form's definition in `_adamw_ref`."""

import copy
import ctypes
import pickle
import struct

import numpy as np
import pytest
import torch

import _adamw_ref as A
from paper_2609_33437_gb300 import optim as O
from paper_2609_33437_gb300 import smat as S

INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 3
BASE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return S.load_library()


def _call(lib, params=(BASE, BASE + 0x1000), grads=(2 * BASE, 2 * BASE + 0x1000), numels=(300, 5), **kw):
    n = len(numels)
    arrays = [ctypes.create_string_buffer(struct.pack(f"{n}{c}", *v)) for c, v in (("P", params), ("P", grads), ("q", numels))]
    v = dict(params_at=ctypes.addressof(arrays[0]), grads_at=ctypes.addressof(arrays[1]), numels_at=ctypes.addressof(arrays[2]), m1=3 * BASE,
             m2=4 * BASE, e1=0, e2=0, scale_at=0, lr_at=0, step_at=0, scale=1.0, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, wd=0.0,
             step=1, seed=0, n=n, dtype=1, gdtype=1, bits=32)
    v.update(kw)
    return lib.smat_adamw_step(O._ADAMW.pack(*v.values()), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(gdtype=-1), UNSUPPORTED), (dict(bits=16), UNSUPPORTED), (dict(lr=-1.0), INVALID),
    (dict(lr=float("inf")), INVALID), (dict(lr=float("nan")), INVALID), (dict(beta1=1.0), INVALID), (dict(beta2=-0.1), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(wd=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(step=0), INVALID), (dict(step=1 << 31), INVALID), (dict(n=-1), INVALID), (dict(params_at=0), INVALID), (dict(numels_at=0), INVALID),
    (dict(numels=(-1, 5)), INVALID), (dict(numels=(1 << 41, 5)), INVALID), (dict(m1=0), INVALID), (dict(m2=4 * BASE + 16), ALIGNMENT),
    (dict(e1=5 * BASE), INVALID), (dict(bits=8), INVALID), (dict(bits=8, e1=5 * BASE), INVALID),
    (dict(bits=8, e1=5 * BASE, e2=5 * BASE), INVALID), (dict(m2=3 * BASE), INVALID), (dict(m1=BASE), INVALID),
    (dict(scale_at=4 * BASE), INVALID), (dict(lr_at=4 * BASE), INVALID), (dict(step_at=3 * BASE), INVALID),
    (dict(step_at=6 * BASE + 4), ALIGNMENT),
])
def test_refuses(lib, bad, code):
    kw = dict(bad)
    lists = {k: kw.pop(k) for k in ("numels",) if k in kw}
    assert _call(lib, **lists, **kw) == code
    assert lib.smat_last_error()


def test_refuses_pointers(lib):
    assert _call(lib, params=(BASE, 0)) == INVALID
    assert _call(lib, params=(BASE, BASE + 0x1001)) == ALIGNMENT
    assert _call(lib, params=(BASE, BASE)) == INVALID            # the same tensor twice
    assert _call(lib, params=(BASE, BASE + 598)) == INVALID      # 300 bf16 end at 600
    assert _call(lib, grads=(BASE, 2 * BASE)) == INVALID         # a gradient in its parameter
    assert _call(lib, grads=(0, 0)) == 0                         # nothing to do
    assert _call(lib, numels=(0, 0), params=(0, 0), grads=(0, 0)) == 0
    assert lib.smat_adamw_step(None, None) == INVALID
    assert _call(lib, numels=(1 << 32, 5), bits=8, e1=5 * BASE, e2=6 * BASE) == INVALID


def test_places_and_values(lib):
    numels = struct.pack("3q", 1, 256, 257)
    assert lib.smat_adamw_places(numels, 3) == 256 + 256 + 512
    assert lib.smat_adamw_places(None, 0) == 0 and lib.smat_adamw_places(numels, -1) == 0
    b = [BASE * k for k in range(1, 7)]
    assert lib.smat_adamw_values(*b, 100, None) == INVALID and lib.smat_adamw_values(*b, -256, None) == INVALID
    assert lib.smat_adamw_values(*b, 0, None) == 0
    assert lib.smat_adamw_values(b[0], b[1], b[2], b[3], b[0], b[5], 256, None) == INVALID
    assert lib.smat_adamw_values(b[0] + 4, *b[1:], 256, None) == ALIGNMENT


def test_binding_refuses():
    p = torch.zeros(4)
    with pytest.raises(ValueError, match="bits"):
        O.Moments([p], bits=16)
    with pytest.raises(ValueError, match="at least one"):
        O.Moments([])
    m = O.Moments([p])
    assert m.places == 256 and m.starts == [0] and [v.shape for v in m.views("m1")] == [(4,)]
    with pytest.raises(ValueError, match="moments of 1"):
        O.adamw([p, p], [p], m, 1)
    with pytest.raises(ValueError, match="CUDA"):
        O.adamw([p], [p], m, 1)
    with pytest.raises(ValueError, match=r"grads\[1\]"):
        O._addresses("grads", [p, p[:2]], [4, 4], -1, True)
    with pytest.raises(ValueError, match=r"params\[0\]"):
        O._addresses("params", [torch.zeros(4, 2).t()], [8], -1, False)
    with pytest.raises(ValueError, match="step"):
        O._one("step", torch.zeros(2, dtype=torch.int64), torch.int64, p.device)
    with pytest.raises(ValueError, match="bits"):
        O.AdamW([p], bits=4)


def test_the_8_bit_form():
    """Every code reads back and packs to itself; a value in between is rounded up as often as its place says."""
    q = np.arange(256, dtype=np.uint8)
    for places, less, count in ((3, 16, 120), (4, 17, 240)):
        v = np.zeros(A.GROUP)
        v[:count] = A.table(places)[:count]  # up to the largest code a group's largest magnitude can have
        e = np.array([90], np.uint8)
        values = (v * 2.0 ** (90 - 127)).astype(np.float32)
        for part in (0, 65535):
            got, ge = A.codes(values, np.full(A.GROUP, part), places, less)
            assert ge[0] == e[0] and bool((got[:count] == q[:count]).all())
        assert bool((A.values(got, ge, places) == values).all())
    v = np.full(A.GROUP, 1.0, np.float32)
    v[1:] = 0.6 + 1 / 64 * 0.3  # steps are 1/16 of 1/2 there
    rng = np.random.default_rng(0)
    ups, n = 0, 400
    for _ in range(n):
        got, e = A.codes(v, rng.integers(0, 65536, A.GROUP), 3, 16)
        back = A.values(got, e, 3)[1:]
        ups += int((back > v[1:]).sum())
        assert bool((abs(back - v[1:]) < 1 / 16).all())
    low = np.floor(float(v[1]) * 16) / 16
    p = (float(v[1]) - low) * 16
    assert abs(ups / (n * 255) - p) < 5 * (p * (1 - p) / (n * 255)) ** 0.5


@pytest.mark.parametrize("bits", [8, 32])
def test_moments_where_they_lie(bits):
    """A buffer that was given other storage: a step takes that one, and refuses one of another size or stride."""
    m = O.Moments([torch.zeros(300), torch.zeros(5)], bits=bits)
    names = ("q1", "q2", "e1", "e2") if bits == 8 else ("m1", "m2")
    keep = []
    for k, name in enumerate(names):
        t = m.buffers()[name]
        keep.append(t.data)
        t.data = t.data.clone()
        assert t.data_ptr() != keep[-1].data_ptr() and m._addresses()[k] == t.data_ptr()
    assert bits == 8 or m._addresses()[2:] == (0, 0)
    t = m.buffers()[names[0]]
    for bad in (t.data[:-1].clone(), t.data.repeat_interleave(2)[::2]):
        was, t.data = t.data, bad
        with pytest.raises(ValueError, match=f"moments: {names[0]}"):
            m._addresses()
        t.data = was
    t.data = t.data[:0]
    with pytest.raises(ValueError, match="moments"):
        m.values() if bits == 8 else m._addresses()


class _CheckOnly:
    """A library whose step is the check alone."""

    def __init__(self, lib):
        self.smat_adamw_step, self.smat_last_error = lambda args, _: lib.smat_adamw_check(args), lib.smat_last_error


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(bits=16), UNSUPPORTED), (dict(lr=-1.0), INVALID), (dict(beta1=1.0), INVALID),
    (dict(eps=0.0), INVALID), (dict(step=0), INVALID), (dict(numels_at=0), INVALID), (dict(m2=4 * BASE + 16), ALIGNMENT),
    (dict(bits=8, e1=5 * BASE, e2=5 * BASE), INVALID), (dict(lr_at=4 * BASE), INVALID),
])
def test_the_check_alone_refuses_the_same(lib, bad, code):
    assert _call(_CheckOnly(lib), **bad) == _call(lib, **bad) == code
    assert _call(_CheckOnly(lib), params=(BASE, BASE)) == INVALID
    assert _call(_CheckOnly(lib), grads=(0, 0)) == 0
    assert lib.smat_adamw_check(None) == INVALID


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("laid_out", [False, True])
@pytest.mark.parametrize("how", [copy.deepcopy, lambda v: pickle.loads(pickle.dumps(v))], ids=["deepcopy", "pickle"])
def test_copies(how, laid_out, bits):
    """A copied or pickled optimizer has its own parameters, moments and counts, which belong together as the original's do."""
    ps = [torch.nn.Parameter(torch.ones(300)), torch.nn.Parameter(torch.ones(5, dtype=torch.bfloat16))]
    opt = O.AdamW([dict(params=ps[:1]), dict(params=ps[1:], lr=0.5)], lr=0.25, bits=bits, seed=7)
    if laid_out:
        first = opt.lists()[0][2].buffers()
        for k, b in enumerate(first.values()):
            b.fill_(k + 2)
        opt.steps, opt.counts[0][0] = 4, 3
    new = how(opt)
    assert (new.bits, new.seed, new.steps, new.counts) == (bits, 7, 4 if laid_out else 0, [[3], [0]] if laid_out else [])
    assert [g["lr"] for g in new.param_groups] == [0.25, 0.5] and (new._lists is None) is not laid_out
    lists = new.lists()
    for (group, qs, moments), (_, _, old), mine in zip(lists, opt.lists(), new.param_groups):
        assert group is mine and qs[0] is mine["params"][0] and qs[0] is not ps[0] and moments.sizes == old.sizes
        for name, b in moments.buffers().items():
            assert torch.equal(b, old.buffers()[name]) and b.data_ptr() != old.buffers()[name].data_ptr()
        assert moments._addresses() != old._addresses()
    new.counts[0][0] += 1
    assert opt.counts[0][0] == (3 if laid_out else 0)
    one = how(O.Moments(ps[:1], bits=bits))
    assert one.sizes == [300] and one.places == 512


def test_groups_may_be_added():
    """Before the moments are laid out, after (a saved state or `lists` lays them out), and after steps; what is there stays."""
    ps = [torch.nn.Parameter(torch.ones(n)) for n in (300, 5, 7)]
    opt = O.AdamW(ps[:1], lr=0.25, seed=7)
    assert len(opt.state_dict()["moments"]) == 1
    first = opt.lists()[0][2]
    first.buffers()["m1"].fill_(2.0)
    opt.counts[0][0] = 3
    opt.add_param_group(dict(params=[ps[1], torch.nn.Parameter(torch.ones(4, dtype=torch.bfloat16))], lr=0.5))
    assert [len(q) for _, q, _ in opt.lists()] == [1, 1, 1] and opt.counts == [[3], [0], [0]]
    assert opt.lists()[0][2] is first and opt.lists()[1][0] is opt.param_groups[1] and opt.lists()[1][0]["lr"] == 0.5
    with pytest.raises(ValueError):  # a parameter that is there
        opt.add_param_group(dict(params=[ps[0]]))
    with pytest.raises(ValueError, match="one device"):
        opt.add_param_group(dict(params=[ps[2], torch.nn.Parameter(torch.ones(4, device="meta"))]))
    assert len(opt.param_groups) == 2 and len(opt.lists()) == 3
    opt.add_param_group(dict(params=[ps[2]]))
    assert len(opt.param_groups) == 3 and opt.counts == [[3], [0], [0], [0]]
    again = O.AdamW(ps[:1])
    again.add_param_group(dict(params=ps[1:]))
    assert [len(q) for _, q, _ in again.lists()] == [1, 2]
    wrong = O.AdamW([ps[0], torch.nn.Parameter(torch.ones(4, device="meta"))])
    for _ in range(2):
        with pytest.raises(ValueError, match="one device"):
            wrong.lists()


def test_the_fused_step_in_double_refuses(lib):
    opt = S.AdamWDouble(1e-3, 0.9, 0.999, 1e-8, 0.0, 1)
    assert lib.smat_grad_map_adamw_double_multi(None, 0, None, None, None, 0, ctypes.byref(opt), None) == INVALID


@pytest.mark.parametrize("bits", [8, 32])
def test_a_state_that_does_not_fit_changes_nothing(bits):
    ps = [torch.nn.Parameter(torch.ones(300)), torch.nn.Parameter(torch.ones(5))]
    opt, other = (O.AdamW(ps, lr=lr, bits=bits, seed=seed) for lr, seed in ((0.25, 7), (0.5, 8)))
    opt.lists()[0][2].buffers()["e1" if bits == 8 else "m1"].fill_(9)
    opt.counts[0][:] = [3, 2]
    other.lists()
    name = "q1" if bits == 8 else "m2"

    def state(**change):
        s = opt.state_dict()
        s.update(change)
        return s

    moments = opt.state_dict()["moments"][0]
    wrong = [state(counts=[[3]]), state(counts=[]), state(counts=[[3, 2], [1]]), state(param_groups=[]), state(bits=40 - bits),
             state(moments=[{k: v for k, v in moments.items() if k != name}]),
             state(moments=[{**moments, name: moments[name][:-1]}]), state(moments=[{**moments, name: moments[name].double()}])]
    before = {k: v.clone() for k, v in other.lists()[0][2].buffers().items()}
    for s in wrong:
        with pytest.raises(ValueError, match="state"):
            other.load_state_dict(s)
        assert (other.counts, other.seed, other.param_groups[0]["lr"]) == ([[0, 0]], 8, 0.5)
        assert all(torch.equal(v, before[k]) for k, v in other.lists()[0][2].buffers().items())
    other.load_state_dict(state())
    assert (other.counts, other.seed, other.param_groups[0]["lr"]) == ([[3, 2]], 7, 0.25)
    assert all(torch.equal(v, moments[k]) for k, v in other.lists()[0][2].buffers().items())
