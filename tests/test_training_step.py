"""The parts of a training step together: norm and activation, the equivariant layer, its gradients, the norm's, the clipped AdamW step and
the plan's new weight - through dp_training_step, eagerly and as one captured graph."""

import math
import os

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

import paper_2607_21271_b200 as eq
from paper_2607_21271_b200 import parallel
from tests.harness import eql_dtype, torch_dtype


def test_the_update_comes_last():
    seen = []
    flat = torch.zeros(3)
    order = parallel.dp_training_step(lambda: seen.append("f"), lambda: seen.append("w"), lambda: seen.append("d"), flat, update=lambda: seen.append("u"))
    assert seen == ["f", "w", "d", "u"] and order[-2:] == ["allreduce_done", "update"]
    assert "update" not in parallel.dp_training_step(lambda: 0, lambda: 0, lambda: 0, flat)


def _rank(rank, world, port, out):
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    flat, dw, db = parallel.grad_buffers(2, 3, 4, "cpu")
    p = torch.zeros_like(flat)

    def weight_grad():
        dw.fill_(rank + 1.0)
        db.fill_(10.0 * (rank + 1))

    parallel.dp_training_step(lambda: None, weight_grad, lambda: None, flat, update=lambda: p.sub_(flat))
    np.save(os.path.join(out, f"p{rank}.npy"), p.numpy())
    dist.barrier()
    dist.destroy_process_group()


def test_every_rank_updates_with_the_summed_gradient(tmp_path):
    mp.spawn(_rank, args=(2, 29771, str(tmp_path)), nprocs=2)
    a, b = (np.load(tmp_path / f"p{r}.npy") for r in range(2))
    assert np.array_equal(a, b) and a[0] == -3.0 and a[-1] == -30.0


class Block:
    """y = layer(act(norm(x))) with loss <dy, y>, its parameters in one optimiser."""

    def __init__(self, T, Ci, Co, B, S, groups, dtype, bits, act="silu", seed=0):
        self.T, self.Ci, self.Co, self.B, self.S, self.groups, self.act = T, Ci, Co, B, S, groups, act
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        td, code = torch_dtype(dtype), eql_dtype(dtype)
        new = lambda *s, std=1.0, to=td: (torch.randn(*s, generator=g, device="cuda") * std).to(to)      # noqa: E731
        empty = lambda *s, like=td: torch.empty(*s, dtype=like, device="cuda")                            # noqa: E731
        self.x, self.dy = new(B, S, Ci * T), new(B * S, Co * T)
        self.z, self.y, self.dz, self.dx = empty(B, S, Ci * T), empty(B * S, Co * T), empty(B, S, Ci * T), empty(B, S, Ci * T)
        self.stats = empty(B, groups, 2, like=torch.float32)
        # master parameters in float; what the kernels take in the layer's type
        shapes = {"w": (Co, Ci, T), "bias": (Co,), "gamma": (Ci,), "beta": (Ci,)}
        self.master = {k: new(*s, std=(Ci * T) ** -0.5 if k == "w" else 0.1, to=torch.float32) for k, s in shapes.items()}
        self.master["gamma"] += 1.0
        self.param = {k: v.to(td) for k, v in self.master.items()}
        for k in self.master:
            self.master[k] = self.param[k].float()
        self.flat, self.dw, self.db = parallel.grad_buffers(Co, Ci, T, "cuda")
        self.grad = {"w": self.dw, "bias": self.db, "gamma": empty(Ci, like=torch.float32), "beta": empty(Ci, like=torch.float32)}
        self.state, table = {}, []
        for k, p in self.param.items():
            n, blocks = p.numel(), -(-p.numel() // 256)
            kinds = (torch.float32, torch.float32) if bits == 32 else (torch.float8_e4m3fn, torch.float8_e5m2)
            self.state[k] = {"m": torch.zeros(n, dtype=kinds[0], device="cuda"), "v": torch.zeros(n, dtype=kinds[1], device="cuda")}
            if bits == 8:
                self.state[k] |= {"ms": torch.zeros(blocks, device="cuda"), "vs": torch.zeros(blocks, device="cuda")}
            st = self.state[k]
            table.append(eq.eqlinear_adamw_tensor(p, self.grad[k], st["m"], st["v"], n, code, eq.EQL_FP32, master=None if dtype == "fp32" else self.master[k],
                                                  exp_avg_scale=st.get("ms"), exp_avg_sq_scale=st.get("vs"), weight_decay=0.01 if k == "w" else 0.0))
        if dtype == "fp32":
            self.master = self.param
        s = torch.cuda.current_stream().cuda_stream
        self.ws_bytes = eq.eqlinear_workspace_bytes(T, Ci, Co, code)
        self.ws = empty(self.ws_bytes, like=torch.uint8)
        self.plan = eq.eqlinear_plan(T, Ci, Co, code, self.param["w"], self.param["bias"], self.ws, self.ws_bytes, stream=s)
        self.desc = eq.eqlinear_groupnorm_desc(T, Ci, groups, code, B, S, act={"silu": eq.EQL_ACT_SILU, "gelu": eq.EQL_ACT_GELU}[act])
        self.norm_bytes = eq.eqlinear_groupnorm_scratch_bytes(self.desc)
        self.bytes = max(256, self.norm_bytes, eq.eqlinear_bwd_weight_scratch_bytes(self.plan, B * S))
        self.scratch = empty(self.bytes, like=torch.uint8)
        opt_bytes = eq.eqlinear_adamw_workspace_bytes(table, bits)
        self.opt_ws = empty(opt_bytes, like=torch.uint8)
        self.opt = eq.eqlinear_adamw(table, bits, self.opt_ws, opt_bytes, s)
        self.norm = empty(1, like=torch.float32)
        torch.cuda.synchronize()

    def step(self):
        s, N = torch.cuda.current_stream().cuda_stream, self.B * self.S
        p = self.param

        def fwd():
            eq.eqlinear_groupnorm_fwd(self.desc, self.x, p["gamma"], p["beta"], None, self.z, self.stats, self.scratch, self.bytes, s)
            eq.eqlinear_fwd(self.plan, self.z, self.y, N, s)

        def data_grad():
            eq.eqlinear_bwd_data(self.plan, self.dy, self.dz, N, s)
            eq.eqlinear_groupnorm_bwd(self.desc, self.x, self.dz, p["gamma"], p["beta"], None, self.stats, self.dx, self.grad["gamma"], self.grad["beta"],
                                      self.scratch, self.bytes, s)

        def update():
            eq.eqlinear_adamw_clip(self.opt, 1.0, norm=self.norm, stream=s)
            eq.eqlinear_adamw_step(self.opt, 1e-2, 0.9, 0.99, 1e-8, stream=s)
            eq.eqlinear_plan_set_weight(self.plan, p["w"], p["bias"], s)

        return parallel.dp_training_step(fwd, lambda: eq.eqlinear_bwd_weight(self.plan, self.z, self.dy, self.dw, self.db, N, self.scratch, self.bytes, s),
                                         data_grad, self.flat, update=update)

    def expected(self):
        """Values and gradients in 64 bits by automatic differentiation, from the parameters as they are now."""
        x = self.x.double().requires_grad_()
        p = {k: v.double().requires_grad_() for k, v in self.param.items()}
        h = x.view(self.B, self.S, self.groups, -1)
        var, mean = torch.var_mean(h, dim=(1, 3), unbiased=False, keepdim=True)
        h = ((h - mean) / (var + 1e-5).sqrt()).view(self.B, self.S, self.Ci, self.T) * p["gamma"].view(-1, 1) + p["beta"].view(-1, 1)
        z = torch.nn.functional.silu(h) if self.act == "silu" else torch.nn.functional.gelu(h)
        t = torch.arange(self.T, device="cuda")
        dense = p["w"][:, :, (t[:, None] - t[None, :]) % self.T]                      # [o, i, t, s]
        y = torch.einsum("bnis,oits->bnot", z, dense) + p["bias"].view(-1, 1)
        (y.reshape(self.B * self.S, -1) * self.dy.double()).sum().backward()
        return {"y": y.detach().reshape(self.y.shape), "dx": x.grad, **{k: v.grad for k, v in p.items()}}

    def snapshot(self):
        torch.cuda.synchronize()
        out = {"norm": self.norm, "y": self.y, "dx": self.dx, **{"p" + k: v for k, v in self.param.items()}, **{"w" + k: v for k, v in self.master.items()}}
        out |= {k + n: v for k, st in self.state.items() for n, v in st.items()}
        return {k: v.clone() for k, v in out.items()}

    def close(self):
        torch.cuda.synchronize()
        eq.eqlinear_adamw_destroy(self.opt)
        eq.eqlinear_plan_destroy(self.plan)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits,shape", [("fp32", 32, (8, 16, 24, 4, 60, 4)), ("fp16", 32, (4, 32, 40, 3, 100, 8)), ("bf16", 8, (8, 16, 24, 300, 1, 1)),
                                              ("fp32", 8, (1, 40, 24, 2, 333, 5))])
def test_training_steps_against_automatic_differentiation(dtype, bits, shape):
    T, Ci, Co, B, S, groups = shape
    m = Block(T, Ci, Co, B, S, groups, dtype, bits, seed=1)
    # relative to the largest value: the layer's own bars (1e-5; 3e-3; 1.2e-2), for what passes through the layer and then the norm, or the
    # other way round, both parts of it: the norm's share is a few roundings of the type, below a second such bar
    bar = 2 * {"fp32": 1e-5, "fp16": 3e-3, "bf16": 1.2e-2}[dtype]
    try:
        for step in range(1, 4):
            want = m.expected()
            before = {k: v.double().clone() for k, v in m.master.items()}
            assert m.step()[-1] == "update"
            torch.cuda.synchronize()
            got = {"y": m.y, "dx": m.dx, **m.grad}
            for k, ref in want.items():
                err = (got[k].double().reshape(ref.shape) - ref).abs().max() / ref.abs().max()
                assert float(err) <= bar, f"step {step}, {k}: {float(err):.2e}"
            total = math.sqrt(sum(float(g.double().square().sum()) for g in m.grad.values()))
            assert abs(float(m.norm) - total) <= 2.0 ** -23 * total
            moved = {k: (m.master[k].double() - before[k]).abs().max().item() for k in before}
            # an AdamW step moves a parameter by about the learning rate: (1 - b1) / sqrt(1 - b2) of it at most, over the bias corrections
            most = 1e-2 * (1 - 0.9) / math.sqrt(1 - 0.99) * math.sqrt(1 - 0.99 ** step) / (1 - 0.9 ** step) * step
            for k, far in moved.items():
                size = before[k].abs().max().item()
                # (the moments of the steps before may be off by the codes' half steps: 2^-4 of m, and 2^-3 of v, so 2^-3 of its root at most)
                assert 0 < far <= most * (1 if bits == 32 else 1.25) + 1e-2 * 0.01 * size + 1e-6, f"step {step}, {k}: {far} of {most}"
            assert eq.eqlinear_adamw_info(m.opt, 0).step == step
        assert eq.eqlinear_plan_device_status(m.plan) == 0
    finally:
        m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [("fp16", 32), ("bf16", 8)])
def test_a_captured_training_step_is_the_step(dtype, bits):
    """The whole step in one graph, replayed, next to the same calls made one by one."""
    args = (4, 32, 40, 5, 77, 8, dtype, bits)
    a, b = Block(*args, act="gelu", seed=2), Block(*args, act="gelu", seed=2)
    try:
        a.step(); b.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.step()
        for _ in range(3):
            graph.replay()
            b.step()
            x, y = a.snapshot(), b.snapshot()
            assert all(torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)) for k in x)
    finally:
        a.close()
        b.close()
