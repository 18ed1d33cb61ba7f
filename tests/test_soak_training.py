"""Long opt-in checks of norm and optimiser: tensors beyond 4 GB and 2^31 elements, and random shapes."""

import numpy as np
import pytest
import torch

import paper_2607_21271_b200 as eq
from tests.test_groupnorm import ACTS, EPS, Norm, reference

pytestmark = pytest.mark.soak


@pytest.mark.parametrize("T,C,groups,B,S", [(8, 96, 1, 3_200_000, 1), (8, 96, 32, 16_300, 197), (16, 64, 1, 1, 2_200_000)])
def test_norms_of_tensors_beyond_four_gigabytes(T, C, groups, B, S):
    """Instances (of the one map: rows) around the 2^31 and 2^32 byte offsets and at the end, against the formulas."""
    D = C * T
    x, y, dy, dx = (torch.empty(B, S, D, dtype=torch.float16, device="cuda") for _ in range(4))
    assert x.numel() * 2 > 1 << 32
    for b in range(0, B, 4096):
        x[b:b + 4096].normal_()
        dy[b:b + 4096].normal_()
    gamma, beta = torch.randn(C, device="cuda").half(), torch.randn(C, device="cuda").half()
    stats = torch.empty(B, groups, 2, device="cuda")
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    desc = eq.eqlinear_groupnorm_desc(T, C, groups, eq.EQL_FP16, B, S, act=ACTS["silu"], eps=EPS)
    bytes_ = eq.eqlinear_groupnorm_scratch_bytes(desc)
    scratch = torch.empty(max(256, bytes_), dtype=torch.uint8, device="cuda")
    eq.eqlinear_groupnorm_fwd(desc, x, gamma, beta, None, y, stats, scratch, bytes_)
    eq.eqlinear_groupnorm_bwd(desc, x, dy, gamma, beta, None, stats, dx, dgamma, dbeta, scratch, bytes_)
    torch.cuda.synchronize()
    host = lambda t: t.double().cpu().numpy()                                         # noqa: E731
    half = 2.0 ** -11
    if B == 1:
        n, mean = 0, 0.0
        for r in range(0, S, 1 << 16):
            part = x[0, r:r + (1 << 16)].double()
            mean, n = mean + float(part.sum()), n + part.numel()
        mean /= n
        var = sum(float((x[0, r:r + (1 << 16)].double() - mean).square().sum()) for r in range(0, S, 1 << 16)) / n
        assert abs(float(stats[0, 0, 0]) - mean) <= 1e-5 and abs(float(stats[0, 0, 1]) * (var + EPS) ** 0.5 - 1) <= 1e-5
        for row in ((1 << 31) // (2 * D), (1 << 32) // (2 * D), S - 1):
            z = (host(x[0, row]) - mean) * (var + EPS) ** -0.5 * np.repeat(host(gamma), T) + np.repeat(host(beta), T)
            want = z / (1 + np.exp(-z))
            assert np.all(np.abs(host(y[0, row]) - want) <= 1e-4 + half * np.abs(want))
    else:
        for b in ((1 << 31) // (2 * S * D), (1 << 32) // (2 * S * D), B - 1):
            want = reference(host(x[b:b + 1]), host(gamma), host(beta), None, T, groups, "silu", host(dy[b:b + 1]))
            for k, got in (("y", y), ("dx", dx)):
                value, bound = want[k]
                assert np.all(np.abs(host(got[b:b + 1]) - value) <= bound + half * (np.abs(value) + bound) + 2.0 ** -25), (b, k)
    total = sum(float(dy[b:b + 4096].double().sum()) for b in range(0, B, 4096))
    assert bool(torch.isfinite(dx).all()) and np.isfinite(total) and bool(torch.isfinite(dgamma).all())


def test_a_step_over_more_than_two_to_the_31_elements():
    n = (1 << 31) + 5003
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    spots = torch.tensor([0, 255, 256, (1 << 30) + 1, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 1], device="cuda")
    g[spots] = torch.tensor([1.0, -1.0, 2.0, -3.0, 4.0, -5.0, 6.0, -7.0], dtype=torch.bfloat16, device="cuda")
    table = [eq.eqlinear_adamw_tensor(p, g, m, v, n, eq.EQL_BF16, eq.EQL_BF16, exp_avg_scale=ms, exp_avg_sq_scale=vs)]
    bytes_ = eq.eqlinear_adamw_workspace_bytes(table, 8)
    ws = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    h = eq.eqlinear_adamw(table, 8, ws, bytes_)
    norm = torch.zeros(1, device="cuda")
    try:
        eq.eqlinear_adamw_clip(h, 1e30, norm=norm)
        eq.eqlinear_adamw_step(h, 0.5)
        torch.cuda.synchronize()
        assert abs(float(norm) - 141.0 ** 0.5) <= 1e-5
        want = -0.5 * torch.sign(g[spots].float())
        assert torch.equal(p[spots].float(), want) and int((p != 0).sum()) == len(spots)
        assert int((m != 0).sum()) == len(spots) and int((v != 0).sum()) == len(spots)
    finally:
        torch.cuda.synchronize()
        eq.eqlinear_adamw_destroy(h)


@pytest.mark.parametrize("seed", range(60))
def test_random_norms(seed):
    rng = np.random.default_rng(1000 + seed)
    dtype = ("fp32", "fp16", "bf16")[seed % 3]
    size = 4 if dtype == "fp32" else 2
    T = int(rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 32]))
    step = next(k for k in range(1, 17) if k * T * size % 16 == 0)
    C = int(step * rng.integers(1, max(2, 1500 // (T * step))))
    groups = int(rng.choice([g for g in range(1, C + 1) if C % g == 0]))
    rows = int(np.exp(rng.uniform(0, np.log(400_000 / (C * T) + 2)))) + 1
    S = int(rng.choice([1, rng.integers(1, rows + 1), rows]))
    B = max(1, rows // S)
    lengths = rng.integers(0, S + 1, B) if rng.random() < 0.4 else None
    Norm(T, C, groups, B, S, dtype, ("none", "gelu", "silu")[int(rng.integers(3))], lengths=lengths, seed=seed).step()


@pytest.mark.parametrize("T,C,groups,B,S", [(8, 96, 1, 3_200_000, 1), (8, 96, 32, 16_300, 197), (16, 64, 1, 1, 2_200_000)])
def test_parameter_gradients_over_tensors_beyond_four_gigabytes(T, C, groups, B, S):
    """All of dgamma and dbeta, and dx at a few instances or rows, against the formulas in 64 bits from x, dy and the statistics given."""
    D = C * T
    gen = torch.Generator(device="cuda").manual_seed(7)
    x, dy, dx = (torch.empty(B * S, D, dtype=torch.float16, device="cuda") for _ in range(3))
    assert x.numel() * 2 > 1 << 32
    step = (1 << 16) // S * S or 1 << 16                      # whole instances, or rows of the one map
    for r in range(0, B * S, step):
        x[r:r + step].normal_(generator=gen)
        dy[r:r + step].normal_(generator=gen)
    gamma, beta = (torch.randn(C, device="cuda", generator=gen).half() for _ in range(2))
    stats = torch.stack([0.1 * torch.randn(B, groups, device="cuda", generator=gen), 1 + 0.1 * torch.rand(B, groups, device="cuda", generator=gen)], -1)
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    desc = eq.eqlinear_groupnorm_desc(T, C, groups, eq.EQL_FP16, B, S, act=ACTS["silu"], eps=EPS)
    bytes_ = eq.eqlinear_groupnorm_scratch_bytes(desc)
    scratch = torch.empty(max(256, bytes_), dtype=torch.uint8, device="cuda")
    eq.eqlinear_groupnorm_bwd(desc, x, dy, gamma, beta, None, stats, dx, dgamma, dbeta, scratch, bytes_)
    torch.cuda.synchronize()
    want = torch.zeros(2, C, dtype=torch.float64, device="cuda")
    squares = torch.zeros(2, C, dtype=torch.float64, device="cuda")
    ga, be = (p.double().view(1, groups, C // groups, 1) for p in (gamma, beta))

    def parts(r, end):
        """xh and dz of rows r to end, [rows, groups, channels, tuple]"""
        st = stats[r // S:-(-end // S)].double().repeat_interleave(min(S, end - r), 0).view(end - r, groups, 1, 1, 2)
        xh = (x[r:end].double().view(end - r, groups, C // groups, T) - st[..., 0]) * st[..., 1]
        z = xh * ga + be
        p = torch.sigmoid(z)
        return xh, dy[r:end].double().view_as(xh) * p * (1 + z * (1 - p)), st[..., 1]

    for r in range(0, B * S, step):
        xh, dz, _ = parts(r, min(B * S, r + step))
        for k, term in enumerate((dz * xh, dz)):
            want[k] += term.sum((0, 3)).view(C)
            squares[k] += term.square().sum((0, 3)).view(C)
    # n roundings, independent, of partial sums no larger than 6 standard deviations of the whole one: 6 rms sqrt(n) * U * sqrt(n)
    n = B * S * T
    for got, w, sq in zip((dgamma, dbeta), want, squares):
        assert bool(((got.double() - w).abs() <= 8 * 2.0 ** -24 * n * torch.sqrt(sq / n)).all())
        assert float(w.abs().max()) > 100 * 8 * 2.0 ** -24 * n * float(torch.sqrt(sq / n).max())       # what an instance more or less would show in
    if B == 1:
        s1, s2 = (ga.view(C) * want[1]).sum() / (S * D), (ga.view(C) * want[0]).sum() / (S * D)
        for row in ((1 << 31) // (2 * D), (1 << 32) // (2 * D), S - 1):
            xh, dz, rstd = parts(row, row + 1)
            value = (rstd * (ga * dz - s1 - xh * s2)).view(D)
            assert bool(((dx[row].double() - value).abs() <= 2.0 ** -11 * value.abs() + 1e-5).all())    # half's rounding, and float's of values below 100


@pytest.mark.parametrize("seed", range(90))
def test_random_norms_of_wide_rows(seed):
    """Rows of a thousand to ten thousand elements: all kernels' borders, with tuples and groups of every kind."""
    rng = np.random.default_rng(5000 + seed)
    dtype = ("fp32", "fp16", "bf16")[seed % 3]
    size = 4 if dtype == "fp32" else 2
    T = int(rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 20, 32]))
    step = next(k for k in range(1, 17) if k * T * size % 16 == 0)
    C = int(step * max(1, round(np.exp(rng.uniform(np.log(1000), np.log(10000))) / (T * step))))
    few = [g for g in range(1, 9) if C % g == 0]
    groups = int(rng.choice(few if rng.random() < 0.8 else [g for g in range(1, min(C, 64) + 1) if C % g == 0]))
    rows = int(np.exp(rng.uniform(0, np.log(600_000 / (C * T) + 2)))) + 1
    S = int(rng.choice([1, rng.integers(1, rows + 1), rows]))
    B = max(1, rows // S)
    lengths = rng.integers(0, S + 1, B) if rng.random() < 0.4 else None
    Norm(T, C, groups, B, S, dtype, ("none", "gelu", "silu")[int(rng.integers(3))], lengths=lengths, seed=seed).step()
