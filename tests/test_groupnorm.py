"""Group norm with an activation, forward and backward: against the formulas in 64 bits, with bounds from the roundings of float,
and its refusals (which need no GPU)."""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_21271_b200 as eq
from paper_2607_21271_b200 import binding
from tests.harness import eql_dtype, torch_dtype

U = 2.0 ** -24                                   # half a step of float
ACTS = {"none": eq.EQL_ACT_NONE, "gelu": eq.EQL_ACT_GELU, "silu": eq.EQL_ACT_SILU}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ refusals

def fwd_status(change=(), x=1 << 20, gamma=None, beta=None, lengths=None, y=2 << 20, stats=None, scratch=1 << 30, bytes_=1 << 24, desc=None):
    d = desc or eq.eqlinear_groupnorm_desc(4, 8, 2, eq.EQL_FP32, 2, 64)
    for k, v in dict(change).items():
        setattr(d, k, v)
    return eq.load_library().eqlinear_groupnorm_fwd(ctypes.byref(d), x, gamma, beta, lengths, y, stats, scratch, bytes_, None)


def bwd_status(change=(), x=1 << 20, dy=2 << 20, gamma=None, beta=None, lengths=None, stats=3 << 20, dx=4 << 20, dgamma=None, dbeta=None,
               scratch=1 << 30, bytes_=1 << 24):
    d = eq.eqlinear_groupnorm_desc(4, 8, 2, eq.EQL_FP32, 2, 64)
    for k, v in dict(change).items():
        setattr(d, k, v)
    return eq.load_library().eqlinear_groupnorm_bwd(ctypes.byref(d), x, dy, gamma, beta, lengths, stats, dx, dgamma, dbeta, scratch, bytes_, None)


BAD_SHAPES = [
    (dict(T=0), binding.EQL_ERR_INVALID_ARG), (dict(T=65, C=4), binding.EQL_ERR_UNSUPPORTED), (dict(C=0), binding.EQL_ERR_INVALID_ARG),
    (dict(groups=0), binding.EQL_ERR_INVALID_ARG), (dict(groups=3), binding.EQL_ERR_INVALID_ARG), (dict(dtype=3), binding.EQL_ERR_INVALID_ARG),
    (dict(act=3), binding.EQL_ERR_INVALID_ARG), (dict(act=-1), binding.EQL_ERR_INVALID_ARG), (dict(eps=0.0), binding.EQL_ERR_INVALID_ARG),
    (dict(eps=math.nan), binding.EQL_ERR_INVALID_ARG), (dict(eps=math.inf), binding.EQL_ERR_INVALID_ARG),
    (dict(batch=-1), binding.EQL_ERR_INVALID_ARG), (dict(positions=-1), binding.EQL_ERR_INVALID_ARG),
    (dict(batch=1 << 20, positions=1 << 20), binding.EQL_ERR_UNSUPPORTED), (dict(batch=1 << 40), binding.EQL_ERR_UNSUPPORTED),
    (dict(C=1 << 20), binding.EQL_ERR_UNSUPPORTED), (dict(T=1, C=6), binding.EQL_ERR_ALIGNMENT), (dict(T=1, C=4, dtype=1), binding.EQL_ERR_ALIGNMENT),
]


@pytest.mark.parametrize("change,status", BAD_SHAPES)
def test_shapes_that_are_refused(change, status):
    assert fwd_status(change) == status
    assert bwd_status(change) == status
    d = eq.eqlinear_groupnorm_desc(4, 8, 2, eq.EQL_FP32, 2, 64)
    for k, v in change.items():
        setattr(d, k, v)
    with pytest.raises(eq.EqlError) as e:
        eq.eqlinear_groupnorm_scratch_bytes(d)
    assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), binding.EQL_ERR_INVALID_ARG), (dict(y=None), binding.EQL_ERR_INVALID_ARG), (dict(y=1 << 20), binding.EQL_ERR_INVALID_ARG),
    (dict(y=(1 << 20) + 16368), binding.EQL_ERR_INVALID_ARG),          # over the last bytes of x
    (dict(x=(1 << 20) + 8), binding.EQL_ERR_ALIGNMENT), (dict(y=(2 << 20) + 4), binding.EQL_ERR_ALIGNMENT),
    (dict(gamma=4), binding.EQL_ERR_ALIGNMENT), (dict(beta=8), binding.EQL_ERR_ALIGNMENT), (dict(lengths=4), binding.EQL_ERR_ALIGNMENT),
    (dict(stats=8), binding.EQL_ERR_ALIGNMENT),
])
def test_forward_arguments_that_are_refused(change, status):
    assert fwd_status(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), binding.EQL_ERR_INVALID_ARG), (dict(dy=None), binding.EQL_ERR_INVALID_ARG), (dict(dx=None), binding.EQL_ERR_INVALID_ARG),
    (dict(stats=None), binding.EQL_ERR_INVALID_ARG), (dict(dx=1 << 20), binding.EQL_ERR_INVALID_ARG), (dict(dx=2 << 20), binding.EQL_ERR_INVALID_ARG),
    (dict(dx=(4 << 20) + 8), binding.EQL_ERR_ALIGNMENT), (dict(dgamma=5 << 20, dbeta=(5 << 20) + 16), binding.EQL_ERR_INVALID_ARG), (dict(dgamma=12), binding.EQL_ERR_ALIGNMENT), (dict(dbeta=20), binding.EQL_ERR_ALIGNMENT),
])
def test_backward_arguments_that_are_refused(change, status):
    assert bwd_status(**change) == status


def test_scratch_that_is_refused():
    d = eq.eqlinear_groupnorm_desc(16, 64, 1, eq.EQL_FP16, 1, 65536)
    need = eq.eqlinear_groupnorm_scratch_bytes(d)
    assert need > 0
    big = 1 << 40
    assert fwd_status(desc=d, y=big, scratch=None) == binding.EQL_ERR_INVALID_ARG
    assert fwd_status(desc=d, y=big, scratch=(1 << 30) + 16) == binding.EQL_ERR_ALIGNMENT
    assert fwd_status(desc=d, y=big, bytes_=16) == binding.EQL_ERR_WORKSPACE
    lib = eq.load_library()
    assert lib.eqlinear_groupnorm_fwd(None, 1, None, None, None, 1, None, None, 0, None) == binding.EQL_ERR_INVALID_ARG
    assert lib.eqlinear_groupnorm_scratch_bytes(ctypes.byref(d), None) == binding.EQL_ERR_INVALID_ARG


def test_no_rows_are_a_success():
    for change in (dict(batch=0), dict(positions=0)):
        assert fwd_status(change, x=None, y=None, scratch=None, bytes_=0) == binding.EQL_OK
        assert bwd_status(change, x=None, dy=None, dx=None, stats=None, scratch=None, bytes_=0) == binding.EQL_OK


# ------------------------------------------------------------------------------------------------ the formulas in 64 bits

def phi(z):
    return np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def cdf(z):
    return torch.special.ndtr(torch.from_numpy(np.ascontiguousarray(z))).numpy()


def act64(z, act):
    return z if act == "none" else z * cdf(z) if act == "gelu" else z * torch.sigmoid(torch.from_numpy(z)).numpy()


def slope64(z, act):
    if act == "none":
        return np.ones_like(z)
    if act == "gelu":
        return cdf(z) + z * phi(z)
    p = torch.sigmoid(torch.from_numpy(z)).numpy()
    return p * (1 + z * (1 - p))


def reference(x, gamma, beta, lengths, T, groups, act, dy=None, eps=EPS):
    """x [B, S, D] in 64 bits -> (value, bound of the float arithmetic's error) of every output."""
    B, S, D = x.shape
    C, w = D // T, D // groups
    ge, be = np.repeat(gamma, T), np.repeat(beta, T)
    out = {k: [np.zeros(x.shape), np.zeros(x.shape)] for k in ("y", "dx")}
    stats, stats_bound = np.zeros((B, groups, 2)), np.zeros((B, groups, 2))
    stats[:, :, 1] = eps ** -0.5
    stats_bound[:, :, 1] = 4 * U * eps ** -0.5
    sums = {k: [np.zeros(C), np.zeros(C)] for k in ("dgamma", "dbeta")}
    chains = np.zeros((C, 2))
    for b in range(B):
        n = S if lengths is None else int(np.clip(lengths[b], 0, S))
        if n == 0:
            continue
        for g in range(groups):
            cols = slice(g * w, (g + 1) * w)
            v = x[b, :n, cols]
            mean = v.mean()
            centred = v - mean
            var = (centred ** 2).mean()
            r = 1 / math.sqrt(var + eps)
            xh = centred * r
            # The mean comes from a running mean and merged partial means, each step of which moves it by a share of what it adds: its roundings
            # are those of values no larger than A, 64 at most at their full size; the sum of squares likewise, relative to itself (all terms
            # are positive), and to the mean's error, squared.
            A = np.abs(v).max()
            emean, er = 64 * U * A, 64 * U * r + r ** 3 * (64 * U * A) ** 2
            exh = r * (emean + U * np.abs(v)) + np.abs(centred) * er + 2 * U * np.abs(xh)
            stats[b, g], stats_bound[b, g] = (mean, r), (emean, er)
            z = xh * ge[cols] + be[cols]
            ez = np.abs(ge[cols]) * exh + 4 * U * (np.abs(xh * ge[cols]) + np.abs(be[cols]))
            # the activation's slope is below 1.13; its own evaluation: an exponential or error function of z, good to a few roundings of
            # values below 1 and, through the rounding of its argument, |z| or z^2 more; both fall faster than that grows
            y = act64(z, act)
            ey = 1.13 * ez + (0 if act == "none" else 16 * U * np.abs(z))
            out["y"][0][b, :n, cols], out["y"][1][b, :n, cols] = y, ey
            if dy is None:
                continue
            d = dy[b, :n, cols]
            k = slope64(z, act)
            dz = d * k
            edz = np.abs(d) * ((0 if act == "none" else 1.13 * ez + 24 * U) + U * np.abs(k))
            chan = np.arange(g * w, (g + 1) * w) // T
            np.add.at(sums["dbeta"][0], chan, dz.sum(0))
            np.add.at(sums["dgamma"][0], chan, (dz * xh).sum(0))
            # sums: 256 additions one after the other at most (rows of a thread, then lanes, ranges, instances)
            np.add.at(sums["dbeta"][1], chan, (edz + 256 * U * np.abs(dz)).sum(0))
            np.add.at(sums["dgamma"][1], chan, (edz * np.abs(xh) + np.abs(dz) * exh + 256 * U * np.abs(dz * xh)).sum(0))
            m = n * w
            s1, s2 = (ge[cols] * dz).sum() / m, (ge[cols] * dz * xh).sum() / m
            G = np.abs(ge[cols])
            e1 = (G * (edz + 260 * U * np.abs(dz))).sum() / m
            e2 = (G * (edz * np.abs(xh) + np.abs(dz) * exh + 260 * U * np.abs(dz * xh))).sum() / m
            dx = r * (ge[cols] * dz - s1 - xh * s2)
            edx = r * (G * edz + e1 + np.abs(xh) * e2 + exh * abs(s2) + 6 * U * (np.abs(ge[cols] * dz) + abs(s1) + np.abs(xh * s2))) + np.abs(dx) * er / r
            out["dx"][0][b, :n, cols], out["dx"][1][b, :n, cols] = dx, edx
    return {"y": out["y"], "dx": out["dx"], "stats": (stats, stats_bound), **sums}


# ------------------------------------------------------------------------------------------------ on the GPU

class Guarded:
    """Device buffers with guard bytes on both sides."""

    def __init__(self):
        self.all = []

    def new(self, shape, kind, values=None, fill=None):
        n = int(np.prod(shape)) * kind.itemsize
        raw = torch.full((256 + -(-n // 256) * 256 + 256,), 0x5A, dtype=torch.uint8, device="cuda")
        part = raw[256:256 + n].view(kind).view(*shape)
        if values is not None and n:
            part.copy_(torch.from_numpy(np.ascontiguousarray(values)).to("cuda").to(kind))
        elif fill is not None and n:
            part.fill_(fill)
        self.all.append((raw, 256, 256 + n))
        return part

    def check(self):
        torch.cuda.synchronize()
        for raw, a, b in self.all:
            assert bool((raw[:a] == 0x5A).all()) and bool((raw[b:] == 0x5A).all()), "wrote beside a buffer"


class Norm:
    def __init__(self, T, C, groups, B, S, dtype, act, lengths=None, seed=0, affine=True, x=None, dy=None):
        rng = np.random.default_rng(seed)
        self.args = (T, C, groups, B, S, dtype, act)
        self.guard = Guarded()
        kind, D = torch_dtype(dtype), C * T
        if x is None:
            x = rng.standard_normal((B, S, C, T)) * np.exp(0.5 * rng.standard_normal((C, 1))) + rng.standard_normal((C, 1))
        dy = rng.standard_normal((B, S, D)) if dy is None else dy
        self.x = self.guard.new((B, S, D), kind, np.asarray(x).reshape(B, S, D))
        self.dy = self.guard.new((B, S, D), kind, dy)
        self.gamma = self.guard.new((C,), kind, 1 + 0.3 * rng.standard_normal(C)) if affine else None
        self.beta = self.guard.new((C,), kind, 0.3 * rng.standard_normal(C)) if affine else None
        self.lengths = None if lengths is None else self.guard.new((B,), torch.int32, np.asarray(lengths, np.int32))
        self.y, self.dx = (self.guard.new((B, S, D), kind, fill=-7.0) for _ in range(2))
        self.stats = self.guard.new((B, groups, 2), torch.float32, fill=math.nan)
        self.dgamma, self.dbeta = (self.guard.new((C,), torch.float32, fill=math.nan) for _ in range(2))
        self.desc = eq.eqlinear_groupnorm_desc(T, C, groups, eql_dtype(dtype), B, S, act=ACTS[act], eps=EPS)
        self.bytes = eq.eqlinear_groupnorm_scratch_bytes(self.desc)
        self.scratch = self.guard.new((self.bytes,), torch.uint8, fill=0xFF) if self.bytes else None
        self.pad = None
        if lengths is not None:
            self.pad = (torch.arange(S, device="cuda")[None, :] >= self.lengths.clamp(0, S)[:, None]).view(B, S, 1).expand(B, S, D)
        torch.cuda.synchronize()

    def fwd(self, stream=None, stats=True):
        s = torch.cuda.current_stream().cuda_stream if stream is None else stream
        eq.eqlinear_groupnorm_fwd(self.desc, self.x, self.gamma, self.beta, self.lengths, self.y, self.stats if stats else None, self.scratch,
                                  self.bytes, stream=s)

    def bwd(self, stream=None):
        s = torch.cuda.current_stream().cuda_stream if stream is None else stream
        eq.eqlinear_groupnorm_bwd(self.desc, self.x, self.dy, self.gamma, self.beta, self.lengths, self.stats, self.dx, self.dgamma, self.dbeta,
                                  self.scratch, self.bytes, stream=s)

    def outputs(self):
        torch.cuda.synchronize()
        return {k: getattr(self, k).clone() for k in ("y", "stats", "dx", "dgamma", "dbeta")}

    def expected(self):
        T, C, groups, B, S, dtype, act = self.args
        host = lambda t: t.double().cpu().numpy()                                    # noqa: E731
        x, dy = host(self.x), host(self.dy)
        gamma = np.ones(C) if self.gamma is None else host(self.gamma)
        beta = np.zeros(C) if self.beta is None else host(self.beta)
        return reference(x, gamma, beta, None if self.lengths is None else self.lengths.cpu().numpy(), T, groups, act, dy)

    def check(self, what=("y", "stats", "dx", "dgamma", "dbeta")):
        self.guard.check()
        want, dtype = self.expected(), self.args[5]
        half = torch.finfo(torch_dtype(dtype)).eps / 2
        least = 2.0 ** -25 if dtype == "fp16" else 0.0                               # half a step of the subnormal halves
        for k in what:
            value, bound = want[k]
            got = getattr(self, k).double().cpu().numpy()
            if self.pad is not None and k in ("y", "dx"):
                rest = self.pad.cpu().numpy()
                assert np.all(got[rest] == -7.0), f"{k}: rows of padding were written"
                got = np.where(rest, value, got)
            limit = bound + 1e-30
            if k in ("y", "dx") and dtype != "fp32":
                limit = limit + half * (np.abs(value) + bound) + least
            off = np.abs(got - value)
            assert np.all(off <= limit), f"{k}: off by {np.nanmax(off)}, {np.nanmax(off / limit)} of the bound, NaN: {np.isnan(off).sum()}"

    def step(self, what=("y", "stats", "dx", "dgamma", "dbeta")):
        self.fwd()
        self.bwd()
        self.check(what)


# (T, C, groups, B, S): one token to long maps; groups whose borders fall inside a 16-byte vector, at its end, beyond rows of 256 vectors
SHAPES = [
    (4, 8, 2, 1, 64), (8, 96, 32, 3, 197), (4, 24, 8, 2, 500), (1, 320, 32, 2, 49), (3, 16, 4, 2, 33), (5, 8, 8, 2, 7), (5, 8, 4, 3, 1),
    (16, 64, 1, 37, 1), (2, 4, 1, 5, 1), (1, 8, 1, 3, 1), (32, 33, 11, 2, 5), (12, 10, 5, 1, 130), (1, 4096, 1, 2, 3), (6, 4, 2, 1, 3000),
    (8, 96, 1, 130, 1), (2, 8, 8, 300, 2), (64, 2, 2, 4, 31), (1, 16, 16, 2, 1100), (7, 40, 8, 3, 64), (4, 24, 1, 1, 5000),
    (1, 1000, 8, 2, 70), (8, 1100, 2, 2, 9), (1, 2056, 257, 3, 4),
    (12, 700, 2, 2, 40), (3, 2736, 1, 2, 70), (4, 24, 8, 1, 20000), (1, 16, 16, 1, 40001),
]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T{}_C{}_g{}_B{}_S{}".format(*s))
def test_forward_and_gradients_against_the_formulas(shape, dtype, act):
    Norm(*shape, dtype, act, seed=sum(shape)).step()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,act", [("fp32", "gelu"), ("bf16", "silu"), ("fp16", "none")])
@pytest.mark.parametrize("shape", [(8, 96, 32, 7, 197), (4, 24, 8, 6, 70), (1, 320, 32, 5, 9), (3, 16, 1, 9, 3), (8, 16, 2, 40, 1), (4, 24, 1, 3, 2000)],
                         ids=lambda s: "T{}_C{}_g{}_B{}_S{}".format(*s))
def test_padded_batches(shape, dtype, act):
    """Lengths from none to all; what stands in the padding, NaN and infinities, is never read into anything."""
    B, S = shape[3:]
    lengths = np.random.default_rng(1).integers(0, S + 1, B)
    lengths[:3] = (0, S, 1)
    if B > 4:
        lengths[3], lengths[4] = -5, S + 9                   # taken as none and all
    n = Norm(*shape, dtype, act, lengths=lengths, seed=2)
    keep = n.x.clone(), n.dy.clone()
    n.step()
    first = n.outputs()
    n.x.masked_fill_(n.pad, math.nan)
    n.dy.masked_fill_(n.pad, math.inf)
    n.fwd()
    n.bwd()
    again = n.outputs()
    assert all(torch.equal(first[k], again[k]) for k in first)
    n.x.copy_(keep[0])
    n.dy.copy_(keep[1])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 96, 32, 3, 197), (16, 64, 1, 70, 1), (4, 24, 1, 1, 5000)])
def test_without_gamma_beta_or_their_gradients(shape):
    n = Norm(*shape, "fp32", "gelu", seed=3, affine=False)
    n.step()
    first = n.outputs()
    n.dgamma.fill_(5.0)
    n.dx.fill_(0.0)
    s = torch.cuda.current_stream().cuda_stream
    eq.eqlinear_groupnorm_bwd(n.desc, n.x, n.dy, None, None, None, n.stats, n.dx, None, None, n.scratch, n.bytes, stream=s)
    n.guard.check()
    assert torch.equal(n.dx, first["dx"]) and bool((n.dgamma == 5.0).all())
    n.y.fill_(0.0)
    n.stats.fill_(3.0)
    n.fwd(stats=False)                                       # inference
    torch.cuda.synchronize()
    assert torch.equal(n.y, first["y"]) and bool((n.stats == 3.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 96, 32, 2, 197), (16, 64, 1, 20, 1), (4, 24, 1, 1, 5000), (1, 320, 32, 2, 49)])
def test_values_far_from_zero_and_single_far_values(shape):
    T, C, groups, B, S = shape
    rng = np.random.default_rng(4)
    x = 1000.0 + rng.standard_normal((B, S, C, T))           # the spread is a thousandth of the mean
    Norm(*shape, "fp32", "none", seed=4, x=x).step()
    x = rng.standard_normal((B, S, C, T))
    x[:, 0, 0, 0] = 300.0                                    # the first value of every instance, which others could be compared to
    Norm(*shape, "fp32", "silu", seed=5, x=x).step()
    x = np.full((B, S, C, T), 3.0)                           # no spread at all
    n = Norm(*shape, "fp32", "none", seed=6, x=x)
    n.step()
    assert torch.equal(n.y, n.beta.repeat_interleave(T).expand(B, S, C * T))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("shape", [(8, 96, 32, 3, 197), (16, 64, 1, 20, 1), (4, 24, 2, 2, 3000), (1, 320, 32, 2, 49), (3, 16, 16, 2, 60), (4, 24, 8, 1, 20000)])
def test_what_is_not_finite_stays_in_its_group(shape, bad, act):
    T, C, groups, B, S = shape
    n = Norm(*shape, "fp16", act, seed=7)
    n.fwd()
    n.bwd()
    good = n.outputs()
    n.x[B - 1, S // 2, 2] = bad
    n.fwd()
    n.bwd()
    now = n.outputs()
    w = C * T // groups
    hit = torch.zeros_like(now["y"], dtype=torch.bool)
    hit[B - 1, :, :w] = True
    for k in ("y", "dx"):
        assert bool(torch.isnan(now[k][hit]).all()) and torch.equal(now[k][~hit], good[k][~hit])


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(8, 96, 32, 2, 197), (16, 64, 1, 20, 1), (4, 24, 1, 1, 5000), (1, 320, 32, 2, 49), (4, 32, 4, 9, 2)])
def test_activations_far_from_zero(shape, dtype, act):
    """Arguments of hundreds on either side, where exponentials leave float and a pair of values holds both ends."""
    n = Norm(*shape, dtype, act, seed=12)
    n.gamma.mul_(150.0)
    n.step()


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of the 64-bit forward pass, in a few directions, next to the kernel's gradients."""
    shape, act = (4, 12, 3, 2, 29), "gelu"
    T, C, groups, B, S = shape
    n = Norm(*shape, "fp32", act, seed=8)
    n.step()
    host = {k: getattr(n, k).double().cpu().numpy() for k in ("x", "dy", "gamma", "beta", "dx", "dgamma", "dbeta")}
    rng = np.random.default_rng(9)

    def loss(x, gamma, beta):
        return (reference(x, gamma, beta, None, T, groups, act)["y"][0] * host["dy"]).sum()

    h = 1e-5
    for name, grad in (("x", "dx"), ("gamma", "dgamma"), ("beta", "dbeta")):
        for _ in range(3):
            v = rng.standard_normal(host[name].shape)
            up, down = ({**{k: host[k] for k in ("x", "gamma", "beta")}, name: host[name] + sign * h * v} for sign in (1, -1))
            numeric = (loss(**up) - loss(**down)) / (2 * h)
            given = (host[grad] * v).sum()
            # h^2 times a third derivative of order one summed over the entries, the loss's own roundings over h, and float's in the gradient
            size = np.abs(host[grad] * v).sum()
            assert abs(numeric - given) <= 1e-7 * size + 1e-4 * size * 1e-2 + 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 96, 32, 64, 197), (16, 64, 1, 3000, 1), (4, 24, 1, 2, 20000), (1, 320, 32, 8, 200)])
def test_the_same_bits_again_on_another_stream_and_replayed(shape):
    """Two norms that share one scratch, captured one after the other into a graph; replays give the bits of plain calls."""
    a, b = Norm(*shape, "bf16", "silu", seed=10), Norm(*shape, "bf16", "silu", seed=11)
    b.scratch = a.scratch
    for n in (a, b):
        n.fwd()
        n.bwd()
        torch.cuda.synchronize()
    first = a.outputs(), b.outputs()
    for n in (a, b):
        for k in ("y", "dx", "dgamma", "dbeta", "stats"):
            getattr(n, k).zero_()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        a.fwd(s)
        b.fwd(s)
        a.bwd(s)
        b.bwd(s)
    for _ in range(2):
        with torch.cuda.stream(side):
            graph.replay()
        for n, want in zip((a, b), first):
            got = n.outputs()
            assert all(torch.equal(got[k], want[k]) for k in want)
    a.guard.check()
    b.guard.check()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(8, 96, 32, 2, 197), (16, 64, 1, 20, 1), (4, 24, 8, 1, 20000), (1, 320, 32, 2, 49), (4, 32, 4, 9, 2)])
def test_arguments_beyond_any_exponential(shape, dtype, act):
    """Arguments of 1e25: the activations are 0 and z there, their slopes 0 and 1."""
    n = Norm(*shape, dtype, act, seed=13)
    n.gamma.fill_(1e25)
    n.fwd()
    n.bwd()
    n.guard.check()
    T, C, groups, B, S = shape
    x, dy = (t.double().view(B, S, groups, -1) for t in (n.x, n.dy))
    mean, rstd = (n.stats[..., k].double().view(B, 1, groups, 1) for k in (0, 1))
    z = float(n.gamma[0]) * (x - mean) * rstd
    y, up = n.y.double().view_as(z), z > 0
    assert float(z.abs().min()) > 1e6                                                 # (beta, 0.3, and the mean's rounding do not count)
    # below: |z| sigmoid(z) and its like fall from 1e-16 on past any z that the kernels may hold them at
    assert float(y[~up].abs().max()) < 1e-15
    # above: two roundings of float on either side of a subtraction, of values up to max |x|, and the output's own
    near = z.abs() + float(n.gamma[0]) * rstd * x.abs().amax()
    half = torch.finfo(n.y.dtype).eps / 2
    assert bool(((y - z)[up].abs() <= (2.0 ** -20 * near + half * z.abs() + 1)[up]).all())
    want = torch.where(up, dy, 0).view(B, S, C, T)
    size = want.abs().sum((0, 1, 3))
    assert bool(((n.dbeta.double() - want.sum((0, 1, 3))).abs() <= (B * S * T * 2.0 ** -24 + 2.0 ** -20) * size + 1e-12).all())
