"""Performance cases of what a training program calls around the equivariant linear layer.

Two kinds of case:

  "norm"   group norm with an activation over features [B, S, C*T] (group index fastest, statistics over positions, the
           channels of a norm group and the group axis; one gamma and beta per channel), "fwd" for inference or "step" for
           forward and backward;
  "adamw"  one optimiser step over all tensors of a network, with states in 32 or in 8 bits, optionally with the clipping
           of the global gradient norm (and the loss scale taken out) in front.

The plain forms say what is computed, in elementary torch operations; with `own` the package's entry points compute it.
Shapes are those of the package's workloads (ViT and Swin token shapes, the group-order sweep, the operator-benchmark
shapes) or generic.
"""

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
EPS_NORM = 1e-5
BLOCK = 256                     # elements that share one scale of an 8-bit state
E4M3_MAX, E5M2_MAX = 448.0, 57344.0
TINY = 2.0 ** -100              # blocks whose largest magnitude is below hold zeros
FIRST_STEP = 1000               # the optimiser is in mid-training
LR, EPS_ADAM, DECAY = 1e-3, 1e-8, 0.05


# ------------------------------------------------------------------------------------------------ cases

def _norm(name, T, C, groups, B, S, dtype, mode, act, ragged=False):
    c = {"op": "norm", "T": T, "C": C, "groups": groups, "B": B, "S": S, "dtype": dtype, "mode": mode, "act": act, "ragged": ragged}
    return {"name": name, **c} if name else c


def _adamw(name, net, T, width, layers, state_bits, dtype, grad, clip, loss_scale=0.0, beta2=0.999):
    c = {"op": "adamw", "net": net, "T": T, "width": width, "layers": layers, "state_bits": state_bits, "dtype": dtype,
         "grad": grad, "clip": clip, "loss_scale": loss_scale, "beta2": beta2}
    return {"name": name, **c} if name else c


def listed():
    return [
        # The smallest configuration of the package: nothing but the latency of a call.
        _norm("norm_tiny_fp32_fwd", 4, 8, 2, 1, 64, "fp32", "fwd", "none"),
        # The norm in front of a ViT-B MLP, every token by itself (one group), batch 128: inference.
        _norm("norm_vit_b_tokens_fp16_fwd", 8, 96, 1, 128 * 197, 1, "fp16", "fwd", "none"),
        # First stage of Swin-T, batch 128: norm and GELU over 56 x 56 maps, inference.
        _norm("norm_swin_t_s1_fp16_fwd", 4, 24, 8, 128, 56 * 56, "fp16", "fwd", "gelu"),
        # Training between two layers of ViT-B width, batch 128, many small groups.
        _norm("norm_vit_b_bf16_step", 8, 96, 32, 128, 197, "bf16", "step", "silu"),
        # Training in single precision, batch 64 of ViT-S width, images of different lengths in one padded batch.
        _norm("norm_vit_s_fp32_step", 8, 48, 8, 64, 197, "fp32", "step", "gelu", ragged=True),
        # Training the per-token norm of the group-order sweep's layers (total width 1024).
        _norm("norm_sweep_T16_tokens_fp16_step", 16, 64, 1, 65536, 1, "fp16", "step", "none"),
        # Training on 56 x 56 maps at a total width of 384: the largest, memory traffic alone.
        _norm("norm_maps_bf16_step", 4, 96, 24, 128, 56 * 56, "bf16", "step", "gelu"),
        # One very large map normalised as a whole: a single group of 67 million elements.
        _norm("norm_one_map_fp16_step", 16, 64, 1, 1, 65536, "fp16", "step", "silu"),
        # One layer's weight and bias: the latency of an optimiser step.
        _adamw("adamw_one_layer_fp32", "layer", 8, 48, 1, 32, "fp32", "fp32", 0.0),
        # A network of 12 ViT-B blocks of order 8 in half precision: clipping, loss scale, float master weights.
        _adamw("adamw_vit_b_fp16", "blocks", 8, 96, 12, 32, "fp16", "fp32", 1.0, loss_scale=4096.0),
        # The same network in bfloat16 with states in 8 bits.
        _adamw("adamw8_vit_b_bf16", "blocks", 8, 96, 12, 8, "bf16", "fp32", 1.0),
        # Eight of the operator benchmark's widest layers (134 million weights), 16-bit gradients as an exchange leaves them.
        _adamw("adamw8_op_c2048_bf16", "layer", 4, 2048, 8, 8, "bf16", "bf16", 0.0, beta2=0.95),
    ]


def _spread(rng, low, high):
    """A whole number from low to high, spread evenly over its logarithm."""
    return max(low, min(high, round(low * (high / low) ** rng.random())))


def draw(rng):
    if rng.random() < 0.65:
        dtype = rng.choice(["fp16", "bf16", "fp16", "bf16", "fp32"])
        size = TYPES[dtype].itemsize
        T = rng.choice([1, 2, 3, 4, 4, 5, 6, 8, 8, 12, 16, 32])
        step = 1
        while (step * T * size) % 16:                     # rows are whole 16-byte pieces, as the layer's
            step += 1
        C = max(step, _spread(rng, 8, 1024 // T if T < 128 else 8) // step * step)
        most = 240_000_000 // size // (C * T)             # rows: bytes and work below the largest listed case's
        rows = _spread(rng, 1, most)
        S = rng.choice([1, _spread(rng, 2, max(2, min(rows, 70000))), 197, 49, 56 * 56])
        B = max(1, rows // S) if S > 1 else rows
        if B * S > most:
            B, S = 1, max(1, most)
        divisors = [g for g in range(1, C + 1) if C % g == 0 and g <= 64 and (g == 1 or S * (C // g) * T >= 16)]
        groups = rng.choice([1, rng.choice(divisors), divisors[-1]])        # a norm is over sixteen values at least
        return _norm(None, T, C, groups, B, S, dtype, rng.choice(["fwd", "step", "step"]), rng.choice(["none", "gelu", "silu"]),
                     ragged=S > 1 and rng.random() < 0.3)
    dtype = rng.choice(["fp16", "bf16", "fp32"])
    T = rng.choice([1, 3, 4, 8, 8, 16])
    net = rng.choice(["layer", "blocks"])
    width = _spread(rng, 5, 1200 // T)
    layers = _spread(rng, 1, 24)
    bits, grad = rng.choice([8, 32]), rng.choice(["fp32", "fp32", "bf16" if dtype == "fp32" else dtype])
    clip, loss_scale, beta2 = rng.choice([0.0, 1.0, 0.3]), rng.choice([0.0, 1024.0]), rng.choice([0.95, 0.999])
    while True:                 # no more than the largest listed case costs
        case = _adamw(None, net, T, width, layers, bits, dtype, grad, clip, loss_scale, beta2)
        if layers == 1 or work(case)["bytes"] <= 2e9:
            return case
        layers -= 1


def _tensors(case):
    """(elements, decayed) of each tensor of the network."""
    T, w = case["T"], case["width"]
    if case["net"] == "layer":
        one = [(w * w * T, True), (w, False)]
    else:                       # norm, q/k/v, projection, norm, fc1, fc2, each layer with its bias
        one = [(w, False), (w, False), (3 * w * w * T, True), (3 * w, False), (w * w * T, True), (w, False),
               (w, False), (w, False), (4 * w * w * T, True), (4 * w, False), (4 * w * w * T, True), (w, False)]
    return one * case["layers"]


# ------------------------------------------------------------------------------------------------ inputs

class _Norm:
    """Features, parameters and the buffers of one norm."""

    def __init__(self, case, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        td = TYPES[case["dtype"]]
        T, C, B, S = case["T"], case["C"], case["B"], case["S"]

        def normal(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        # activations: channels with offsets and scales of their own, some tokens far larger than the rest
        scale, offset = (normal(C, 1) * 0.3).exp(), normal(C, 1)
        token = 1.0 + 15.0 * (torch.rand(B, S, 1, 1, generator=g, device="cuda") < 0.002)
        self.x = ((normal(B, S, C, T) * scale + offset) * token).to(td).view(B, S, C * T)
        self.gamma = (1.0 + 0.2 * normal(C)).to(td)
        self.beta = (0.2 * normal(C)).to(td)
        self.lengths = None
        if case["ragged"]:
            n = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            n[0] = S                                      # one full image, and one empty where there are two
            n[1:2] = 0
            self.lengths = n
        self.y = torch.full_like(self.x, 0.5)             # rows of the padding stay what they are
        self.step = case["mode"] == "step"
        self.stats = None
        if self.step:
            self.dy = normal(B, S, C * T).to(td)
            self.dx = torch.full_like(self.x, 0.25)
            self.dgamma, self.dbeta = (torch.empty(C, device="cuda") for _ in range(2))
            self.stats = torch.empty(B, case["groups"], 2, device="cuda")
        self.case = case
        if own:                                           # the descriptor and scratch that a program keeps
            import paper_2607_21271_b200 as eq

            self.desc = eq.eqlinear_groupnorm_desc(
                T, C, case["groups"], {"fp32": eq.EQL_FP32, "fp16": eq.EQL_FP16, "bf16": eq.EQL_BF16}[case["dtype"]], B, S,
                act={"none": eq.EQL_ACT_NONE, "gelu": eq.EQL_ACT_GELU, "silu": eq.EQL_ACT_SILU}[case["act"]], eps=EPS_NORM)
            self.scratch_bytes = eq.eqlinear_groupnorm_scratch_bytes(self.desc)
            self.scratch = torch.empty(max(256, self.scratch_bytes), dtype=torch.uint8, device="cuda")
            self.stream = torch.cuda.current_stream().cuda_stream


class _AdamW:
    """Parameters, gradients and states of a network, each kind in one buffer in which every tensor starts at a multiple of
    256 elements; what lies between two tensors is zero and stays so."""

    def __init__(self, case, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        td, gd = TYPES[case["dtype"]], TYPES[case["grad"]]
        sizes = _tensors(case)
        starts, total = [], 0
        for n, _ in sizes:
            starts.append(total)
            total += -(-n // BLOCK) * BLOCK
        real = torch.zeros(total, device="cuda")
        self.decay = torch.zeros(total, device="cuda")
        rate = torch.zeros(total, device="cuda")          # gradients of different layers differ in size
        rates = (torch.randn(len(sizes), generator=g, device="cuda") - 6.0).exp().tolist()
        for (n, decayed), at, r in zip(sizes, starts, rates):
            real[at:at + n] = 1.0
            rate[at:at + n] = r
            if decayed:
                self.decay[at:at + n] = DECAY

        def normal():
            return torch.randn(total, generator=g, device="cuda")

        spread = (normal() * 1.5).exp() * rate            # each weight's own typical gradient
        weight = 0.05 * normal() * real
        self.loss_scale = torch.full((1,), case["loss_scale"], device="cuda") if case["loss_scale"] else None
        # gradients: about one hundredth of all entries are zero
        grad = normal() * spread * (torch.rand(total, generator=g, device="cuda") > 0.01)
        self.grad = (grad * (case["loss_scale"] or 1.0)).to(gd)
        m, v = 0.3 * normal() * spread, spread.square() * (0.5 + torch.rand(total, generator=g, device="cuda"))
        self.param = weight.to(td)
        self.master = self.param.float() if td != torch.float32 else None
        self.bits = case["state_bits"]
        if self.bits == 8:
            self.m, self.m_scale = _to_8_bits(m, E4M3_MAX, torch.float8_e4m3fn, False)
            self.v, self.v_scale = _to_8_bits(v, E5M2_MAX, torch.float8_e5m2, True)
        else:
            self.m, self.v = m, v
        self.norm = torch.zeros(1, device="cuda")
        self.t = FIRST_STEP
        self.clip, self.beta2 = case["clip"], case["beta2"]
        if own:                                           # the handle that a program keeps
            import paper_2607_21271_b200 as eq

            code = {torch.float32: eq.EQL_FP32, torch.float16: eq.EQL_FP16, torch.bfloat16: eq.EQL_BF16}
            tensors = []
            for (n, decayed), at in zip(sizes, starts):
                part, block = slice(at, at + n), slice(at // BLOCK, at // BLOCK + -(-n // BLOCK))
                tensors.append(eq.eqlinear_adamw_tensor(
                    self.param[part], self.grad[part], self.m[part], self.v[part], n, code[td], code[gd],
                    master=None if self.master is None else self.master[part],
                    exp_avg_scale=self.m_scale[block] if self.bits == 8 else None,
                    exp_avg_sq_scale=self.v_scale[block] if self.bits == 8 else None,
                    weight_decay=DECAY if decayed else 0.0))
            self.stream = torch.cuda.current_stream().cuda_stream
            bytes_ = eq.eqlinear_adamw_workspace_bytes(tensors, self.bits)
            self.workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
            self.opt = eq.eqlinear_adamw(tensors, self.bits, self.workspace, bytes_, stream=self.stream)
            eq.eqlinear_adamw_set_step(self.opt, FIRST_STEP, stream=self.stream)

    def __del__(self):
        if getattr(self, "opt", None):
            import paper_2607_21271_b200 as eq

            eq.eqlinear_adamw_destroy(self.opt)


def prepare(case, seed):
    return _Norm(case, seed) if case["op"] == "norm" else _AdamW(case, seed)


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if isinstance(s, _Norm):
        return _norm_own(s) if own else _norm_plain(s)
    return _adamw_own(s) if own else _adamw_plain(s)


def _norm_own(s):
    import paper_2607_21271_b200 as eq

    eq.eqlinear_groupnorm_fwd(s.desc, s.x, s.gamma, s.beta, s.lengths, s.y, s.stats, s.scratch, s.scratch_bytes, stream=s.stream)
    if not s.step:
        return s.y
    eq.eqlinear_groupnorm_bwd(s.desc, s.x, s.dy, s.gamma, s.beta, s.lengths, s.stats, s.dx, s.dgamma, s.dbeta,
                              s.scratch, s.scratch_bytes, stream=s.stream)
    return {"y": s.y, "stats": s.stats, "dx": s.dx, "dgamma": s.dgamma, "dbeta": s.dbeta}


def _adamw_own(s):
    import paper_2607_21271_b200 as eq

    if s.clip or s.loss_scale is not None:
        eq.eqlinear_adamw_clip(s.opt, s.clip or math.inf, loss_scale=s.loss_scale, norm=s.norm, stream=s.stream)
    eq.eqlinear_adamw_step(s.opt, LR, 0.9, s.beta2, EPS_ADAM, stream=s.stream)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    out = {"param": s.param, "exp_avg": s.m, "exp_avg_sq": s.v, "norm": s.norm}
    if s.master is not None:
        out["master"] = s.master
    if s.bits == 8:
        out["exp_avg_scale"], out["exp_avg_sq_scale"] = s.m_scale, s.v_scale
    return out


def _cdf(z):
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))


def _act(z, act):
    return z if act == "none" else z * _cdf(z) if act == "gelu" else z / (1.0 + torch.exp(-z))


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "gelu":
        return _cdf(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _norm_plain(s):
    c = s.case
    B, S, G, K, T = c["B"], c["S"], c["groups"], c["C"] // c["groups"], c["T"]
    shape, over = (B, S, G, K, T), (1, 3, 4)
    x = s.x.float().view(shape)
    lengths = s.lengths if s.lengths is not None else torch.full((B,), S, dtype=torch.int32, device=x.device)
    valid = (torch.arange(S, device=x.device)[None, :] < lengths[:, None]).view(B, S, 1, 1, 1)
    count = (lengths.clamp(min=1).double() * K * T).view(B, 1, 1, 1, 1)
    mean = (torch.where(valid, x, 0.0).sum(over, keepdim=True, dtype=torch.float64) / count).float()
    centred = torch.where(valid, x - mean, 0.0)
    var = (centred.square().sum(over, keepdim=True, dtype=torch.float64) / count).float()
    rstd = 1.0 / (var + EPS_NORM).sqrt()
    xh = centred * rstd
    gamma, beta = s.gamma.float().view(G, K, 1), s.beta.float().view(G, K, 1)
    z = xh * gamma + beta
    y = torch.where(valid, _act(z, c["act"]).to(s.y.dtype), s.y.view(shape)).view(s.y.shape)
    if not s.step:
        return y
    dz = torch.where(valid, s.dy.float().view(shape) * _act_slope(z, c["act"]), 0.0)
    dgamma, dbeta = ((dz * xh).sum((0, 1, 4), dtype=torch.float64).float().view(-1), dz.sum((0, 1, 4), dtype=torch.float64).float().view(-1))
    scaled = dz * gamma
    first = (scaled.sum(over, keepdim=True, dtype=torch.float64) / count).float()
    second = ((scaled * xh).sum(over, keepdim=True, dtype=torch.float64) / count).float()
    dx = torch.where(valid, (rstd * (scaled - first - xh * second)).to(s.dx.dtype), s.dx.view(shape)).view(s.dx.shape)
    return {"y": y, "stats": torch.cat([mean.view(B, G, 1), rstd.view(B, G, 1)], 2), "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _to_8_bits(values, top, kind, positive):
    """(codes, scales) of blocks of 256.  Each step is one rounded float operation: what lies next to a border between two
    codes goes where these operations put it."""
    v = values.view(-1, BLOCK)
    most = v.abs().amax(1)
    fine = most >= TINY
    limit = torch.full_like(most, top)
    scale = torch.where(fine, most / limit, 0.0)
    inverse = torch.where(fine, limit / torch.where(fine, most, 1.0), 0.0)
    q = v * inverse[:, None]
    if positive:                # a second moment that is not zero is never held as zero: the least code stands for it
        q = torch.where((v > 0) & fine[:, None], q.clamp(min=2.0 ** -16), q)
    return q.clamp(-top, top).to(kind).view(-1), scale


def _from_8_bits(codes, scale):
    return (codes.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _adamw_plain(s):
    """The states are updated by separately rounded float operations, in this order: states in 8 bits depend on their bits."""
    s.t += 1
    g = s.grad.float()
    if s.clip or s.loss_scale is not None:
        scale = s.loss_scale if s.loss_scale is not None else torch.ones_like(s.norm)
        s.norm = (g.double().square().sum().sqrt() / scale.double()).float()
        limit = torch.full_like(s.norm, s.clip or math.inf)
        g = g * ((limit / (s.norm + 1e-6)).clamp(max=1.0) / scale)
    m, v = (s.m, s.v) if s.bits == 32 else (_from_8_bits(s.m, s.m_scale), _from_8_bits(s.v, s.v_scale))
    m = m * 0.9 + g * (1.0 - 0.9)
    v = v * s.beta2 + (g * g) * (1.0 - s.beta2)
    if s.bits == 32:
        s.m, s.v = m, v
    else:
        s.m, s.m_scale = _to_8_bits(m, E4M3_MAX, torch.float8_e4m3fn, False)
        s.v, s.v_scale = _to_8_bits(v, E5M2_MAX, torch.float8_e5m2, True)
    first, second = 1.0 - 0.9 ** s.t, 1.0 - s.beta2 ** s.t
    p = s.master if s.master is not None else s.param
    p = p * (1.0 - LR * s.decay) - LR * (m / first) / ((v / second).sqrt() + EPS_ADAM)
    if s.master is not None:
        s.master, s.param = p, p.to(s.param.dtype)
    else:
        s.param = p
    return _adamw_outputs(s)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Each input read once and each output written once; operations of the formulas, counted per element."""
    if case["op"] == "norm":
        n, size = float(case["B"] * case["S"] * case["C"] * case["T"]), TYPES[case["dtype"]].itemsize
        if case["ragged"]:
            n /= 2                                        # lengths are spread evenly
        act = {"none": 0, "silu": 4, "gelu": 8}[case["act"]]
        params = 2.0 * case["C"] * size
        if case["mode"] == "fwd":
            return {"bytes": 2 * n * size + params, "flops": n * (6 + act)}
        more = case["B"] * case["groups"] * 8.0 + 2 * case["C"] * 4.0
        return {"bytes": 5 * n * size + 2 * params + more, "flops": n * (18 + 3 * act)}
    n = float(sum(k for k, _ in _tensors(case)))
    state = 4 if case["state_bits"] == 32 else 1 + 4.0 / BLOCK
    param = 8 if case["dtype"] == "fp32" else 10          # read and written as float, and once more in 16 bits
    return {"bytes": n * (TYPES[case["grad"]].itemsize + 4 * state + param), "flops": n * (16 + (3 if case["clip"] or case["loss_scale"] else 0))}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    if case["op"] == "norm":
        return _norm_exact(case, _Norm(case, seed))
    return _adamw_exact(case, _AdamW(case, seed))


def _norm_exact(case, s):
    """Instance by instance, with the padding cut off instead of masked."""
    B, S, C, T, G = (case[k] for k in ("B", "S", "C", "T", "groups"))
    x = s.x.double().view(B, S, G, -1)
    wide = [p.double().repeat_interleave(T).view(1, G, -1) for p in (s.gamma, s.beta)]
    length = [S] * B if s.lengths is None else s.lengths.tolist()
    # instances of the same length together
    order = {}
    for b, n in enumerate(length):
        order.setdefault(n, []).append(b)
    y = s.y.double().view(B, S, G, -1).clone()
    if s.step:
        dx = s.dx.double().view(B, S, G, -1).clone()
        dgamma, dbeta = torch.zeros(C, dtype=torch.float64, device=x.device), torch.zeros(C, dtype=torch.float64, device=x.device)
        stats = torch.zeros(B, G, 2, dtype=torch.float64, device=x.device)
    for n, who in order.items():
        if n == 0:
            if s.step:
                stats[who, :, 1] = EPS_NORM ** -0.5
            continue
        all_of_them = len(who) == B and n == S
        part = x if all_of_them else x[who, :n]
        var, mean = torch.var_mean(part, dim=(1, 3), unbiased=False, keepdim=True)
        rstd = torch.rsqrt(var + EPS_NORM)
        xh = (part - mean) * rstd
        z = torch.addcmul(wide[1], xh, wide[0])
        if case["act"] == "gelu":
            cdf = torch.special.ndtr(z)
            out, slope = z * cdf, cdf + z * torch.exp(z * z / -2) * (2 * math.pi) ** -0.5
        elif case["act"] == "silu":
            p = torch.sigmoid(z)
            out, slope = z * p, p + z * p * (1 - p)
        else:
            out, slope = z, None
        if all_of_them:
            y = out
        else:
            y[who, :n] = out
        if s.step:
            dy = s.dy.double().view(B, S, G, -1)
            dz = dy if all_of_them else dy[who, :n]
            dz = dz if slope is None else dz * slope
            dbeta += dz.sum((0, 1)).view(C, T).sum(1)
            dgamma += (dz * xh).sum((0, 1)).view(C, T).sum(1)
            dxh = dz * wide[0]
            grad = (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True)) * rstd
            if all_of_them:
                dx = grad
            else:
                dx[who, :n] = grad
            stats[who] = torch.cat([mean.view(len(who), G, 1), rstd.view(len(who), G, 1)], 2)
    y = y.reshape(B, S, C * T)
    return {"y": y, "stats": stats, "dx": dx.reshape(B, S, C * T), "dgamma": dgamma, "dbeta": dbeta} if s.step else y


def _adamw_exact(case, s):
    """States in 8 bits have a border between two codes wherever one is near: their codes have no value here."""
    t = FIRST_STEP + 1
    unscale = 1.0 / (case["loss_scale"] or 1.0)
    g = s.grad.double() * unscale
    norm = torch.zeros(1, dtype=torch.float64, device=g.device)
    if case["clip"] or case["loss_scale"]:
        norm = torch.linalg.vector_norm(g).view(1)
        g = g * min(1.0, (case["clip"] or math.inf) / (float(norm) + 1e-6))
    if case["state_bits"] == 8:
        m = s.m.double() * s.m_scale.double().repeat_interleave(BLOCK)
        v = s.v.double() * s.v_scale.double().repeat_interleave(BLOCK)
    else:
        m, v = s.m.double(), s.v.double()
    m = torch.lerp(g, m, 0.9)
    v = torch.lerp(g.square(), v, case["beta2"])
    p = (s.master if s.master is not None else s.param).double()
    p = p - p * (LR * s.decay.double()) - (LR / (1 - 0.9 ** t)) * m / (torch.sqrt(v / (1 - case["beta2"] ** t)) + EPS_ADAM)
    out = {"param": p, "exp_avg": m, "exp_avg_sq": v, "norm": norm}
    if s.master is not None:
        out["master"] = p
    if case["state_bits"] == 8:
        out |= {"exp_avg": None, "exp_avg_sq": None, "exp_avg_scale": m.abs().view(-1, BLOCK).amax(1) / E4M3_MAX,
                "exp_avg_sq_scale": v.view(-1, BLOCK).amax(1) / E5M2_MAX}
    return out
