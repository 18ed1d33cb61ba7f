"""The resident norm kernels' plans, walked on the host: what the kernels put side by side in shared memory has room there.

The plan function is a symbol of the library; what a kernel of form N stores is restated here from its sources, where N pairs of a
vector of V elements (16 bytes) have values of their own."""

import ctypes

import pytest

import paper_2607_21271_b200 as eq

I, U, L = ctypes.c_int, ctypes.c_uint, ctypes.c_int64
SLOTS = 220 * 1024                               # dynamic shared memory that the kernels are allowed


class Divisor(ctypes.Structure):
    _fields_ = [("d", U), ("inverse", U)]


class WideDivisor(ctypes.Structure):
    _fields_ = [("d", U), ("inverse", ctypes.c_ulonglong)]


class NormShape(ctypes.Structure):               # csrc/groupnorm_common.cuh
    _fields_ = [(k, I) for k in ("T", "C", "groups", "act", "D", "width", "vectors")] + [("B", L), ("S", L), ("eps", ctypes.c_float)]


class ResidentNorm(ctypes.Structure):
    _fields_ = [("supported", ctypes.c_bool)] + [(k, I) for k in ("groups", "blocks", "cluster", "threads", "instances")] + [("rows", L)] + \
        [(k, I) for k in ("form", "run", "sums", "share", "slot_bytes", "side_offset", "shared_bytes")] + \
        [(k, Divisor) for k in ("tuple", "width", "entry", "runs", "columns", "lanes")] + [("by_cluster", WideDivisor), ("by_blocks", WideDivisor)]


def plan(T, C, groups, B, S, dtype, backward):
    f = getattr(eq.load_library(), "_ZN3eql18resident_norm_planERKNS_9NormShapeE11eql_dtype_tb")
    f.restype, f.argtypes = ResidentNorm, [ctypes.POINTER(NormShape), I, ctypes.c_bool]
    D = C * T
    return f(NormShape(T, C, groups, 0, D, D // groups, D * (4 if dtype == eq.EQL_FP32 else 2) // 16, B, S, 1e-5), dtype, backward)


def shapes(V, backward):
    """Blocks about every border of the rules (256, 512 and 1024 columns) and between, one, two, three and many groups to a row, tuples
    of every kind next to a vector."""
    for T in (1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 20, 24, 28, 32, 64):
        for columns in (5, 8, 31, 96, 100, 255, 256, 257, 258, 261, 300, 384, 510, 511, 512, 513, 515, 768, 1020, 1023, 1024, 1025):
            C = columns * V // T
            for c in {C, C + 1, C + 2} - {0}:
                for groups in {1, 2, 3, c} if c < 64 else {1, 2, 3}:
                    if c % groups == 0 and c * T % V == 0:
                        yield T, c, groups


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dtype,V", [(eq.EQL_FP32, 4), (eq.EQL_FP16, 8), (eq.EQL_BF16, 8)])
def test_what_threads_put_side_by_side_has_room(dtype, V, backward):
    P, wide, crossing = V // 2, 0, 0
    for T, C, groups in shapes(V, backward):
        for S in (1, 3, 49):
            r = plan(T, C, groups, 3, S, dtype, backward)
            if not r.supported:
                continue
            where, width = (T, C, groups, S), C // groups * T
            assert r.threads in ((256, 512) if backward else (256, 1024)), where
            assert r.columns.d * r.lanes.d <= r.threads and r.columns.d * V == r.groups * width, where
            # a run of N = `form` is of one channel, and only the general form has kernels of more than 256 threads
            N = r.form
            assert (N == 1 and T % V == 0) or (N == 2 and T % (V // 2) == 0) or N == P, where
            assert r.threads == 256 or N == P, where
            # entries of a vector: one where it lies in one group, else one a run, or (general form) one an element
            entries = 1 if width % V == 0 else N if N < P else V
            assert r.entry.d * V == width * entries, where
            channels = r.groups * (C // groups)
            side = r.threads * (r.sums + entries) + channels if backward else max(r.threads * entries, 2 * r.threads // 32)
            assert r.side_offset >= r.slot_bytes + 8 * r.groups + 24 * r.cluster * r.groups, where
            assert r.side_offset + 8 * side <= r.shared_bytes <= SLOTS, where
            if backward:
                # a thread stores one sum of dz and dz * xh where N is 1, else one a run of N or two (each half of a pair)
                assert r.sums in ((1,) if N == 1 else (N, 2 * N)) and r.sums * r.run == V, where
                assert T % r.run == 0 and r.runs.d * r.run == T, where      # a sum is of one channel, whose sums follow each other
            lanes = r.lanes.d
            assert -(-r.rows // lanes) * r.threads * 16 * (2 if backward else 1) <= r.slot_bytes and r.rows * r.cluster >= S, where
            wide += r.threads > 256
            crossing += r.threads > 256 and width % V != 0
    assert wide > 100 and crossing > 10          # the walk reaches what it is for
