"""AdamW over many tensors: against the formulas in 64 bits, its 8-bit states against separately rounded float operations, and its
refusals (which need no GPU)."""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_21271_b200 as eq
from paper_2607_21271_b200 import binding
from tests.harness import torch_dtype, eql_dtype

U = 2.0 ** -24                       # half a step of float
BLOCK = 256
SIZES = (1, 3, 255, 256, 257, 0, 2048, 5003)


# ------------------------------------------------------------------------------------------------ refusals

def fake(**change):
    """A tensor at made-up addresses: nothing of it is read before it is refused."""
    args = dict(param=1 << 20, grad=2 << 20, exp_avg=3 << 20, exp_avg_sq=4 << 20, numel=1000, param_dtype=eq.EQL_FP32, grad_dtype=eq.EQL_FP32)
    args.update(change)
    return eq.eqlinear_adamw_tensor(**args)


def refused(tensors, bits=32, workspace=1 << 30, bytes_=1 << 20):
    with pytest.raises(eq.EqlError) as e:
        eq.eqlinear_adamw(tensors, bits, workspace, bytes_)
    return e.value.status


@pytest.mark.parametrize("change,status", [
    (dict(param=None), binding.EQL_ERR_INVALID_ARG),
    (dict(grad=None), binding.EQL_ERR_INVALID_ARG),
    (dict(exp_avg=None), binding.EQL_ERR_INVALID_ARG),
    (dict(exp_avg_sq=None), binding.EQL_ERR_INVALID_ARG),
    (dict(numel=-1), binding.EQL_ERR_INVALID_ARG),
    (dict(numel=(1 << 40) + 1), binding.EQL_ERR_UNSUPPORTED),
    (dict(param_dtype=3), binding.EQL_ERR_INVALID_ARG),
    (dict(grad_dtype=-1), binding.EQL_ERR_INVALID_ARG),
    (dict(weight_decay=-0.1), binding.EQL_ERR_INVALID_ARG),
    (dict(weight_decay=math.nan), binding.EQL_ERR_INVALID_ARG),
    (dict(lr_scale=math.inf), binding.EQL_ERR_INVALID_ARG),
    (dict(exp_avg_scale=5 << 20, exp_avg_sq_scale=6 << 20), binding.EQL_ERR_INVALID_ARG),     # scales without 8-bit states
    (dict(param=(1 << 20) + 8), binding.EQL_ERR_ALIGNMENT),
    (dict(grad=(2 << 20) + 4), binding.EQL_ERR_ALIGNMENT),
    (dict(master=(7 << 20) + 4), binding.EQL_ERR_ALIGNMENT),
    (dict(exp_avg=(1 << 20) + 3984), binding.EQL_ERR_INVALID_ARG),                             # the last elements of param
    (dict(grad=(1 << 20) + 16), binding.EQL_ERR_INVALID_ARG),                                  # a gradient under the parameter
    (dict(master=1 << 30), binding.EQL_ERR_INVALID_ARG),                                       # in the workspace
])
def test_tensors_that_cannot_be_updated_are_refused(change, status):
    assert refused([fake(**change)]) == status
    assert refused([fake(param=8 << 20, grad=9 << 20, exp_avg=10 << 20, exp_avg_sq=11 << 20), fake(**change)]) == status


def test_eight_bit_states_need_their_scales():
    assert refused([fake()], bits=8) == binding.EQL_ERR_INVALID_ARG
    assert refused([fake(exp_avg_scale=5 << 20)], bits=8) == binding.EQL_ERR_INVALID_ARG
    assert refused([fake(exp_avg_scale=(5 << 20) + 2, exp_avg_sq_scale=6 << 20)], bits=8) == binding.EQL_ERR_ALIGNMENT
    assert refused([fake(exp_avg_scale=5 << 20, exp_avg_sq_scale=(5 << 20) + 12)], bits=8) == binding.EQL_ERR_INVALID_ARG   # four scales each


def test_the_same_tensor_twice_is_refused():
    assert refused([fake(), fake()]) == binding.EQL_ERR_INVALID_ARG


def test_optimisers_that_cannot_be_built_are_refused():
    assert refused([]) == binding.EQL_ERR_INVALID_ARG
    assert refused([fake()], bits=16) == binding.EQL_ERR_INVALID_ARG
    assert refused([fake()], workspace=None) == binding.EQL_ERR_INVALID_ARG
    assert refused([fake()], workspace=(1 << 30) + 16) == binding.EQL_ERR_ALIGNMENT
    need = eq.eqlinear_adamw_workspace_bytes([fake()], 32)
    assert refused([fake()], bytes_=need - 1) == binding.EQL_ERR_WORKSPACE
    lib, h = eq.load_library(), ctypes.c_void_p(99)
    assert lib.eqlinear_adamw(ctypes.byref(h), None, 1, 32, 1 << 30, 1 << 20, None) == binding.EQL_ERR_INVALID_ARG
    assert h.value is None
    assert lib.eqlinear_adamw_workspace_bytes(None, 1, 32, ctypes.byref(ctypes.c_size_t())) == binding.EQL_ERR_INVALID_ARG
    for call in (lambda: eq.eqlinear_adamw_step(None, 1e-3), lambda: eq.eqlinear_adamw_clip(None, 1.0),
                 lambda: eq.eqlinear_adamw_set_step(None, 0), lambda: eq.eqlinear_adamw_info(None)):
        with pytest.raises(eq.EqlError) as e:
            call()
        assert e.value.status == binding.EQL_ERR_INVALID_ARG
    eq.eqlinear_adamw_destroy(None)


# ------------------------------------------------------------------------------------------------ on the GPU

class Optimiser:
    """Tensors with guard elements around every buffer, and the library's optimiser over them."""

    def __init__(self, sizes, dtype, grad, bits, master, seed=0, decay=0.1, empty_states=False):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits = sizes, bits
        self.stream = torch.cuda.current_stream().cuda_stream
        self.buffers, self.parts, table = [], [], []
        td, gd = torch_dtype(dtype), torch_dtype(grad)
        for i, n in enumerate(sizes):
            blocks = -(-n // BLOCK)
            g = rng.standard_normal(n) * np.exp(rng.standard_normal(n)) * 10.0 ** rng.integers(-4, 1)
            g[rng.random(n) < 0.1] = 0.0
            scale = 0.0 if empty_states else np.sqrt(np.mean(g ** 2)) if n else 0.0
            t = {"p": self.new(0.1 * rng.standard_normal(n), td), "g": self.new(g, gd),
                 "m": self.new(0.5 * scale * rng.standard_normal(n), torch.float32),
                 "v": self.new(scale ** 2 * rng.chisquare(1, n), torch.float32)}
            if master:
                t["w"] = self.new(t["p"].double().cpu().numpy(), torch.float32)
            if bits == 8:
                for k, kind, top in (("m", torch.float8_e4m3fn, 448.0), ("v", torch.float8_e5m2, 57344.0)):
                    codes, s = encode(t[k].cpu().numpy(), top, kind)
                    t[k], t[k + "s"] = self.new(codes.float().numpy(), kind), self.new(s, torch.float32)
            self.parts.append(t)
            table.append(eq.eqlinear_adamw_tensor(t["p"], t["g"], t["m"], t["v"], n, eql_dtype(dtype), eql_dtype(grad), master=t.get("w"),
                                                  exp_avg_scale=t.get("ms"), exp_avg_sq_scale=t.get("vs"),
                                                  weight_decay=decay if i % 2 == 0 else 0.0, lr_scale=1.0 if i % 3 else 0.5))
        self.table = table
        bytes_ = eq.eqlinear_adamw_workspace_bytes(table, bits)
        self.workspace = torch.full((bytes_ + 256,), 0xAB, dtype=torch.uint8, device="cuda")
        self.h = eq.eqlinear_adamw(table, bits, self.workspace, bytes_, self.stream)
        self.bytes = bytes_

    def new(self, values, kind):
        n, size = len(values), kind.itemsize
        raw = torch.full((-(-n * size // 16) * 16 + 64 + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        part = raw[64:64 + n * size].view(kind)
        if n:
            part.copy_(torch.from_numpy(np.ascontiguousarray(values)).to("cuda").to(kind))
        self.buffers.append((raw, 64, 64 + n * size))
        return part

    def check_guards(self):
        torch.cuda.synchronize()
        for raw, a, b in self.buffers:
            assert bool((raw[:a] == 0x5A).all()) and bool((raw[b:] == 0x5A).all()), "wrote beside a tensor"
        assert bool((self.workspace[self.bytes:] == 0xAB).all())

    def snapshot(self):
        torch.cuda.synchronize()
        return [{k: x.view(torch.uint8).cpu().clone() for k, x in t.items()} for t in self.parts]

    def close(self):
        torch.cuda.synchronize()
        eq.eqlinear_adamw_destroy(self.h)


def encode(values, top, kind):
    """Blocks of 256 as codes and scales, by separately rounded float operations in numpy."""
    f = np.float32
    n = len(values)
    padded = np.zeros(-(-n // BLOCK) * BLOCK, f)
    padded[:n] = values
    b = padded.reshape(-1, BLOCK)
    most = np.abs(b).max(1) if n else np.zeros(0, f)
    fine = most >= f(2.0 ** -100)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        scale = np.where(fine, most / f(top), f(0)).astype(f)
        inverse = np.where(fine, f(top) / np.where(fine, most, f(1)), f(0)).astype(f)
    q = (b * inverse[:, None]).astype(f)
    if kind == torch.float8_e5m2:
        q = np.where((b > 0) & fine[:, None], np.maximum(q, f(2.0 ** -16)), q)
    q = np.clip(q, -f(top), f(top)).reshape(-1)[:n]
    return torch.from_numpy(np.ascontiguousarray(q)).to(kind), scale


def decode(codes, scale, n):
    return codes.float().cpu().numpy() * np.repeat(scale.cpu().numpy(), BLOCK)[:n]


def reference(o, t_number, lr, b1, b2, eps, factor=1.0):
    """The step in 64 bits from what the buffers hold now: per tensor (p, m, v) and the bounds of their errors."""
    out = []
    for desc, t, n in zip(o.table, o.parts, o.sizes):
        g = t["g"].double().cpu().numpy() * factor
        if o.bits == 8:
            m, v = (decode(t[k], t[k + "s"], n).astype(np.float64) for k in ("m", "v"))
        else:
            m, v = (t[k].double().cpu().numpy() for k in ("m", "v"))
        p = t.get("w", t["p"]).double().cpu().numpy()
        rate = lr * desc.lr_scale
        mag = b1 * np.abs(m) + (1 - b1) * np.abs(g)
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        down = np.sqrt(v / (1 - b2 ** t_number)) + eps
        new = p * (1 - rate * desc.weight_decay) - rate * m / (1 - b1 ** t_number) / down
        # m: two products, a sum, two rounded coefficients, the factor (its own rounding and the product); v: the square of the gradient twice as much
        em, ev = 8 * U * mag, 12 * U * v + 2.0 ** -148
        # the update: m's 8, rate and bias correction 6, half of v's 12, square root 2, its correction 4, product and sum 2, quotient 4
        ep = 4 * U * (np.abs(p) + np.abs(new)) + 34 * U * rate * mag / (1 - b1 ** t_number) / down
        out.append(((new, ep), (m, em), (v, ev)))
    return out


def within(got, want, bound, half_step=0.0, least=0.0):
    off = np.abs(got.double().cpu().numpy() - want)
    limit = bound + half_step * (np.abs(want) + bound) + least
    assert np.all(off <= limit), f"off by {float(off.max())}, {float((off / np.maximum(limit, 1e-300)).max())} of the bound"


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad,master", [("fp32", "fp32", False), ("fp16", "fp32", True), ("bf16", "bf16", True), ("bf16", "fp32", False),
                                               ("fp16", "fp16", False), ("fp32", "bf16", True)])
def test_steps_against_the_formulas(dtype, grad, master, bits):
    o = Optimiser(SIZES, dtype, grad, bits, master, seed=3)
    try:
        for t in range(1, 4):
            want = reference(o, t, 2e-3, 0.9, 0.99, 1e-8)
            eq.eqlinear_adamw_step(o.h, 2e-3, 0.9, 0.99, 1e-8, stream=o.stream)
            o.check_guards()
            for part, n, ((p, ep), (m, em), (v, ev)) in zip(o.parts, o.sizes, want):
                if n == 0:
                    continue
                half = torch.finfo(torch_dtype(dtype)).eps / 2
                least = 2.0 ** -25 if dtype == "fp16" else 0.0                       # half a step of the subnormal halves
                within(part["p"], p, ep, half if dtype != "fp32" else 0.0, least)
                if master:
                    within(part["w"], p, ep)
                    assert torch.equal(part["p"], part["w"].to(part["p"].dtype))     # the master's value, rounded once
                if bits == 32:
                    within(part["m"], m, em)
                    within(part["v"], v, ev)
                else:                                                                # half a step of the codes, or of their subnormals
                    for k, x, ex, half_code, sub in (("m", m, em, 2.0 ** -4, 2.0 ** -10), ("v", v, ev, 2.0 ** -3, 2.0 ** -16)):
                        s = np.repeat(part[k + "s"].double().cpu().numpy(), BLOCK)[:n]
                        got = torch.from_numpy(part[k].float().cpu().double().numpy() * s)
                        within(got, x, ex, half_code + 4 * U, sub * s)
        info = eq.eqlinear_adamw_info(o.h, o.stream)
        assert (info.step, info.skipped, info.skip) == (3, 0, 0)
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
def test_eight_bit_states_hold_the_codes_of_float_operations(grad):
    """Bit for bit: the moments by rounded products and sums, the codes by rounded products with the block's inverse scale."""
    f = np.float32
    o = Optimiser((1, 300, 4096, 777), "fp32", grad, 8, False, seed=4)
    try:
        o.parts[2]["g"][256:512] = 0.0                        # a block that only decays
        o.parts[2]["m"][512:768] = 0.0
        o.parts[2]["ms"][2] = 0.0
        o.parts[2]["g"][512:768] = 1e-33                      # held as zeros: below 2^-100
        o.parts[2]["vs"][2] = 0.0
        for _ in range(3):
            want = []
            for part, n in zip(o.parts, o.sizes):
                g = part["g"].float().cpu().numpy()
                m = decode(part["m"], part["ms"], n) * f(0.9) + g * f(1.0 - 0.9)
                v = decode(part["v"], part["vs"], n) * f(0.95) + (g * g) * f(1.0 - 0.95)
                want.append((encode(m, 448.0, torch.float8_e4m3fn), encode(v, 57344.0, torch.float8_e5m2), v))
            eq.eqlinear_adamw_step(o.h, 1e-3, 0.9, 0.95, 1e-8, stream=o.stream)
            o.check_guards()
            for part, ((mc, ms), (vc, vs), v) in zip(o.parts, want):
                assert np.array_equal(part["ms"].cpu().numpy(), ms) and np.array_equal(part["vs"].cpu().numpy(), vs)
                assert torch.equal(part["m"].view(torch.uint8).cpu(), mc.view(torch.uint8))
                assert torch.equal(part["v"].view(torch.uint8).cpu(), vc.view(torch.uint8))
                codes, held = part["v"].float().cpu().numpy(), np.repeat(vs > 0, BLOCK)[:len(v)]
                assert np.all(codes[(v > 0) & held] > 0)      # a second moment that is not zero is not held as zero
        assert float(o.parts[2]["ms"][2]) == 0.0 and not o.parts[2]["m"][512:768].float().any()
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits,grad,scale,max_norm", [(32, "fp32", None, 1.0), (32, "fp16", 64.0, math.inf), (8, "bf16", 1024.0, 1e-3), (32, "fp32", 8.0, 1e9)])
def test_clipping_and_loss_scale(bits, grad, scale, max_norm):
    o = Optimiser(SIZES, "fp32", grad, bits, False, seed=5)
    try:
        loss_scale = None if scale is None else torch.full((1,), scale, device="cuda")
        norm = torch.zeros(1, device="cuda")
        total = math.sqrt(sum(float(t["g"].double().square().sum()) for t in o.parts)) / (scale or 1.0)
        factor = min(1.0, max_norm / (total + 1e-6)) / (scale or 1.0)
        want = reference(o, 1, 1e-3, 0.9, 0.999, 1e-8, factor)
        before = o.snapshot()
        eq.eqlinear_adamw_clip(o.h, max_norm, loss_scale, norm, stream=o.stream)
        assert abs(float(norm) - total) <= U * total * 1.001                          # one rounding of a double sum
        for a, b in zip(before, o.snapshot()):
            assert all(torch.equal(a[k], b[k]) for k in a)                            # the norm changes nothing
        eq.eqlinear_adamw_step(o.h, 1e-3, 0.9, 0.999, 1e-8, stream=o.stream)
        o.check_guards()
        for part, n, ((p, ep), (m, em), (v, ev)) in zip(o.parts, o.sizes, want):
            within(part["p"], p, ep)
            if bits == 32:
                within(part["m"], m, em)
                within(part["v"], v, ev)
        # used up: the next step takes the gradients as they are
        want = reference(o, 2, 1e-3, 0.9, 0.999, 1e-8)
        eq.eqlinear_adamw_step(o.h, 1e-3, 0.9, 0.999, 1e-8, stream=o.stream)
        torch.cuda.synchronize()
        for part, ((p, ep), _, _) in zip(o.parts, want):
            within(part["p"], p, ep)
        first = norm.clone()
        eq.eqlinear_adamw_clip(o.h, max_norm, loss_scale, norm, stream=o.stream)
        assert torch.equal(first, norm)                                               # the same gradients, the same bits
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("what", ["inf", "nan", "-inf", "scale zero", "scale inf"])
def test_a_step_with_gradients_that_are_not_finite_changes_nothing(what, bits):
    o = Optimiser(SIZES, "bf16", "fp32", bits, True, seed=6)
    try:
        eq.eqlinear_adamw_set_step(o.h, 41, o.stream)
        loss_scale = torch.full((1,), {"scale zero": 0.0, "scale inf": math.inf}.get(what, 2.0), device="cuda")
        good = o.parts[7]["g"][5002].clone()
        if not what.startswith("scale"):
            o.parts[7]["g"][5002] = float(what)                                       # the last element of an odd tensor
        before = o.snapshot()
        eq.eqlinear_adamw_clip(o.h, 1.0, loss_scale, stream=o.stream)
        assert eq.eqlinear_adamw_info(o.h, o.stream).skip == 1
        eq.eqlinear_adamw_step(o.h, 1e-3, stream=o.stream)
        o.check_guards()
        for a, b in zip(before, o.snapshot()):
            assert all(torch.equal(a[k], b[k]) for k in a)
        info = eq.eqlinear_adamw_info(o.h, o.stream)
        assert (info.step, info.skipped, info.skip) == (41, 1, 0)
        o.parts[7]["g"][5002] = good                                                  # and the next step is number 42
        loss_scale.fill_(1.0)
        want = reference(o, 42, 1e-3, 0.9, 0.999, 1e-8)
        eq.eqlinear_adamw_clip(o.h, math.inf, loss_scale, stream=o.stream)
        eq.eqlinear_adamw_step(o.h, 1e-3, stream=o.stream)
        torch.cuda.synchronize()
        for part, ((p, ep), _, _) in zip(o.parts, want):
            within(part["w"], p, ep)
        assert eq.eqlinear_adamw_info(o.h, o.stream).step == 42
    finally:
        o.close()


@pytest.mark.gpu
def test_first_step_from_empty_states_and_edges_of_the_rates():
    o = Optimiser((1000, 17), "fp32", "fp32", 8, False, seed=7, empty_states=True)
    try:
        assert not any(t["m"].float().any() or t["v"].float().any() for t in o.parts)
        want = reference(o, 1, 1e-2, 0.0, 0.0, 1e-12)                                 # no memory at all: a step of lr against the sign
        eq.eqlinear_adamw_step(o.h, 1e-2, 0.0, 0.0, 1e-12, stream=o.stream)
        torch.cuda.synchronize()
        for part, ((p, ep), _, _) in zip(o.parts, want):
            within(part["p"], p, ep)
        kept = [t["p"].clone() for t in o.parts]
        eq.eqlinear_adamw_step(o.h, 0.0, stream=o.stream)                             # a learning rate of zero moves no weight
        torch.cuda.synchronize()
        assert all(torch.equal(a, t["p"]) for a, t in zip(kept, o.parts))
        for bad in (dict(lr=-1e-3), dict(lr=math.nan), dict(lr=1e-3, beta1=1.0), dict(lr=1e-3, beta2=-0.1), dict(lr=1e-3, eps=0.0),
                    dict(lr=1e-3, eps=1e-60), dict(lr=1e-3, eps=1e-40), dict(lr=1e-3, eps=math.inf), dict(lr=math.inf), dict(lr=1e39)):
            with pytest.raises(eq.EqlError) as e:
                eq.eqlinear_adamw_step(o.h, **bad)
            assert e.value.status == binding.EQL_ERR_INVALID_ARG
        for bad in (0.0, -1.0, math.nan):
            with pytest.raises(eq.EqlError) as e:
                eq.eqlinear_adamw_clip(o.h, bad)
            assert e.value.status == binding.EQL_ERR_INVALID_ARG
        with pytest.raises(eq.EqlError):
            eq.eqlinear_adamw_set_step(o.h, -1)
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_steps_are_the_steps_themselves(bits):
    """A captured clip and step, replayed with another learning rate each time, next to the same calls made one by one on another stream."""
    a, b = (Optimiser((4000, 77, 2049), "bf16", "fp32", bits, True, seed=8) for _ in range(2))
    try:
        lr = torch.zeros(1, device="cuda")
        loss_scale = torch.full((1,), 2.0, device="cuda")
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            s = torch.cuda.current_stream().cuda_stream
            eq.eqlinear_adamw_clip(a.h, 0.5, loss_scale, stream=s)
            eq.eqlinear_adamw_step(a.h, 7.0, lr_device=lr, stream=s)
            with pytest.raises(eq.EqlError):                                          # an optimiser cannot be built here
                eq.eqlinear_adamw(a.table, bits, a.workspace, a.bytes, s)
        for i in range(4):
            lr.fill_(1e-3 * (i + 1))
            if i == 2:
                a.parts[0]["g"][0] = b.parts[0]["g"][0] = math.inf                    # a step that is left out on the way
            if i == 3:
                a.parts[0]["g"][0] = b.parts[0]["g"][0] = 0.5
            torch.cuda.synchronize()
            graph.replay()
            with torch.cuda.stream(side):
                eq.eqlinear_adamw_clip(b.h, 0.5, loss_scale, stream=side.cuda_stream)
                eq.eqlinear_adamw_step(b.h, float(lr), stream=side.cuda_stream)
            torch.cuda.synchronize()
            for x, y in zip(a.snapshot(), b.snapshot()):
                assert all(torch.equal(x[k], y[k]) for k in x)
        info = eq.eqlinear_adamw_info(a.h, a.stream)
        assert (info.step, info.skipped) == (3, 1)
    finally:
        a.close()
        b.close()


@pytest.mark.gpu
def test_many_tensors_of_every_size():
    """More tensors than CTAs, and one long one: every element is updated once."""
    sizes = [int(n) for n in np.random.default_rng(9).integers(1, 3000, 900)] + [3_000_001]
    o = Optimiser(sizes, "fp32", "fp32", 32, False, seed=9)
    try:
        want = reference(o, 1, 1e-3, 0.9, 0.999, 1e-8)
        eq.eqlinear_adamw_step(o.h, 1e-3, stream=o.stream)
        o.check_guards()
        for part, ((p, ep), (m, em), (v, ev)) in zip(o.parts, want):
            within(part["p"], p, ep)
            within(part["m"], m, em)
            within(part["v"], v, ev)
    finally:
        o.close()


@pytest.mark.gpu
def test_tensors_of_different_types_and_none_with_elements():
    """One optimiser over parameters and gradients of several types gives the bits of one for each; one over empty tensors only counts."""
    kinds = [("fp32", "fp32", False), ("bf16", "fp32", True), ("fp16", "fp16", False), ("bf16", "bf16", True)]
    parts = [Optimiser((5000, 33), d, g, 8, m, seed=20 + i) for i, (d, g, m) in enumerate(kinds)]
    same = [Optimiser((5000, 33), d, g, 8, m, seed=20 + i) for i, (d, g, m) in enumerate(kinds)]
    table = [t for o in same for t in o.table]
    bytes_ = eq.eqlinear_adamw_workspace_bytes(table, 8)
    workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    h = eq.eqlinear_adamw(table, 8, workspace, bytes_, s)
    try:
        for _ in range(2):
            eq.eqlinear_adamw_step(h, 1e-3, stream=s)
            for o in parts:
                eq.eqlinear_adamw_step(o.h, 1e-3, stream=s)
        for a, b in zip(parts, same):
            b.check_guards()
            for x, y in zip(a.snapshot(), b.snapshot()):
                assert all(torch.equal(x[k], y[k]) for k in x)
    finally:
        torch.cuda.synchronize()
        eq.eqlinear_adamw_destroy(h)
        for o in parts + same:
            o.close()
    o = Optimiser((0, 0), "fp32", "fp32", 32, False, seed=30)
    try:
        norm = torch.full((1,), 9.0, device="cuda")
        eq.eqlinear_adamw_clip(o.h, 1.0, norm=norm, stream=o.stream)
        eq.eqlinear_adamw_step(o.h, 1e-3, stream=o.stream)
        o.check_guards()
        assert float(norm) == 0.0 and eq.eqlinear_adamw_info(o.h, o.stream).step == 1
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["param", "master", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"])
def test_memory_of_the_host_is_refused(which):
    n = 512
    args = {k: torch.zeros(n, device="cuda") for k in ("param", "master", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")}
    for host in (torch.zeros(n + 16), torch.zeros(n + 16).pin_memory()):
        at = (-host.data_ptr() % 16) // 4
        table = [eq.eqlinear_adamw_tensor(**{**args, which: host[at:]}, numel=n, param_dtype=eq.EQL_FP32, grad_dtype=eq.EQL_FP32)]
        bytes_ = eq.eqlinear_adamw_workspace_bytes(table, 8)
        workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
        assert refused(table, 8, workspace, bytes_) == binding.EQL_ERR_INVALID_ARG
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("pinned", [False, True])
def test_a_workspace_of_the_host_is_refused(pinned):
    args = {k: torch.zeros(512, device="cuda") for k in ("param", "grad", "exp_avg", "exp_avg_sq")}
    table = [eq.eqlinear_adamw_tensor(**args, numel=512, param_dtype=eq.EQL_FP32, grad_dtype=eq.EQL_FP32)]
    bytes_ = eq.eqlinear_adamw_workspace_bytes(table, 32)
    host = torch.zeros(bytes_ + 256, dtype=torch.uint8)
    host = host.pin_memory() if pinned else host
    assert refused(table, 32, host[-host.data_ptr() % 256:], bytes_) == binding.EQL_ERR_INVALID_ARG
    assert not host.any()


@pytest.mark.gpu
def test_counters_are_not_read_during_capture():
    """The call waits for its stream: refused, and the capture goes on."""
    o = Optimiser((300,), "fp32", "fp32", 32, False, seed=12)
    try:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            s = torch.cuda.current_stream().cuda_stream
            eq.eqlinear_adamw_step(o.h, 1e-3, stream=s)
            with pytest.raises(eq.EqlError) as e:
                eq.eqlinear_adamw_info(o.h, s)
            assert e.value.status == binding.EQL_ERR_INVALID_ARG
        graph.replay()
        torch.cuda.synchronize()
        assert eq.eqlinear_adamw_info(o.h, o.stream).step == 1
    finally:
        o.close()


@pytest.mark.gpu
def test_a_loss_scale_whose_reciprocal_is_not_finite_changes_nothing():
    """1 / 1e-40 is beyond float, and gradients of zero (norm 0) times that would be NaN."""
    o = Optimiser((300, 7), "fp32", "fp32", 32, False, seed=13)
    try:
        for t in o.parts:
            t["g"].zero_()
        before = o.snapshot()
        eq.eqlinear_adamw_clip(o.h, 1.0, torch.full((1,), 1e-40, device="cuda"), stream=o.stream)
        assert eq.eqlinear_adamw_info(o.h, o.stream).skip == 1
        eq.eqlinear_adamw_step(o.h, 1e-3, stream=o.stream)
        info = eq.eqlinear_adamw_info(o.h, o.stream)
        assert (info.step, info.skipped) == (0, 1)
        assert all(torch.equal(a[k], b[k]) for a, b in zip(before, o.snapshot()) for k in a)
    finally:
        o.close()


@pytest.mark.gpu
def test_scalars_that_a_kernel_cannot_reach_are_refused():
    """A learning rate, loss scale or norm in ordinary memory of the host is refused before any launch; pinned memory is read and written."""
    o = Optimiser((300, 7), "fp32", "fp32", 32, False, seed=14)
    try:
        host, before = torch.full((1,), 1e-3), o.snapshot()
        for call in (lambda: eq.eqlinear_adamw_step(o.h, 1e-3, lr_device=host, stream=o.stream),
                     lambda: eq.eqlinear_adamw_clip(o.h, 1.0, loss_scale=host, stream=o.stream),
                     lambda: eq.eqlinear_adamw_clip(o.h, 1.0, norm=host, stream=o.stream)):
            with pytest.raises(eq.EqlError) as e:
                call()
            assert e.value.status == binding.EQL_ERR_INVALID_ARG
        info = eq.eqlinear_adamw_info(o.h, o.stream)
        assert (info.step, info.skipped, info.skip) == (0, 0, 0) and float(host) == float(torch.tensor(1e-3))
        assert all(torch.equal(a[k], b[k]) for a, b in zip(before, o.snapshot()) for k in a)
        norm, lr = torch.zeros(1).pin_memory(), torch.full((1,), 1e-3).pin_memory()
        want = reference(o, 1, float(lr), 0.9, 0.999, 1e-8)
        eq.eqlinear_adamw_clip(o.h, math.inf, norm=norm, stream=o.stream)
        eq.eqlinear_adamw_step(o.h, 7.0, lr_device=lr, stream=o.stream)
        o.check_guards()
        total = math.sqrt(sum(float(t["g"].double().square().sum()) for t in o.parts))
        assert abs(float(norm) - total) <= U * total * 1.001
        for part, ((p, ep), _, _) in zip(o.parts, want):
            within(part["p"], p, ep)
    finally:
        o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("beta2", [0.8, 0.9, 0.95])
def test_eight_bit_second_moments_follow_changing_gradients(beta2):
    """Hundreds of steps, then gradients of a quarter of each block three times smaller and of another quarter three times larger: sqrt(v) stays
    near that of 64 bits.

    Codes lie 14 to 25 % apart, so a step's rounding moves v by an error of standard deviation 0.25 / sqrt(12) of v at most, which
    decays by beta2 a step: 0.25 / sqrt(12 (1 - beta2^2)) altogether if the roundings are independent, half of that for the root."""
    blocks, steps = 24, 600
    n = blocks * BLOCK
    gen = torch.Generator(device="cuda").manual_seed(15)
    rand = lambda: torch.randn(n, device="cuda", generator=gen)                       # noqa: E731
    p, g = rand(), torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(blocks, device="cuda") for _ in range(2))
    table = [eq.eqlinear_adamw_tensor(p, g, m, v, n, eq.EQL_FP32, eq.EQL_FP32, exp_avg_scale=ms, exp_avg_sq_scale=vs)]
    bytes_ = eq.eqlinear_adamw_workspace_bytes(table, 8)
    workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    h = eq.eqlinear_adamw(table, 8, workspace, bytes_, s)
    try:
        size, part = torch.exp(rand()), torch.arange(n, device="cuda") % 4
        want = torch.zeros(n, dtype=torch.float64, device="cuda")
        sigma = 0.5 * 0.25 / math.sqrt(12 * (1 - beta2 ** 2))
        for factors in ((1.0, 1.0), (1 / 3, 3.0)):
            now = torch.where(part == 0, size * factors[0], torch.where(part == 1, size * factors[1], size))
            for _ in range(steps):
                g.copy_(now * rand())
                want.mul_(beta2).add_(g.double().square(), alpha=1 - beta2)
                eq.eqlinear_adamw_step(h, 1e-3, 0.9, beta2, stream=s)
            held = v.view(torch.float8_e5m2).double() * vs.double().repeat_interleave(BLOCK)
            off = torch.log(held / want) / 2                                          # of the root, relative
            for k in range(4):
                assert float(off[part == k].mean().abs()) < sigma / 3                 # a mean over 1536 of them: nothing drags behind
            assert float(off.std()) < 1.5 * sigma and float(off.abs().max()) < 6 * sigma
    finally:
        torch.cuda.synchronize()
        eq.eqlinear_adamw_destroy(h)
