"""What the operators around the loss pass are measured on: the cases, their inputs, their plain form and their
definition in 64 bits.

The operators are the last norm before the fused LM head and what follows its gradients:

  norm_fwd   h = x + residual, y = h / sqrt(mean(h^2) + eps) * (weight + offset); y in the row's type and / or as e4m3
             codes with one float32 scale per row or per group of columns
  norm_bwd   gradients of that: dx (for x and residual alike) and the weight's, summed over the rows
  grad_norm  2-norm over many gradient tensors and the factor that clips it
  adamw      one AdamW step over many tensors, states in float32 or as e4m3 codes with a float32 scale per 256 elements,
             nearest or seeded rounding

Plain forms are elementary torch operations in 32 bits; `own` makes the calls of the framework instead.
"""
import math
import random

import torch

own = False

EPS_NORM = 1e-6
LR, BETA1, BETA2, EPS_ADAM, DECAY, STEP0, SEED = 1e-6, 0.9, 0.999, 1e-8, 0.01, 10, 1234
MAX_NORM = 1.0
BLOCK = 256                 # elements that share the scale of an 8-bit state
E4M3_MAX = 448.0
E4M3_TINY = 2.0 ** -9       # the smallest e4m3 value above zero
SCALE_MIN = 2.0 ** -126

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # one generated token's hidden row in front of the output layer: latency
        {"name": "norm_fwd_one_token", "op": "norm_fwd", "n": 1, "h": 4096, "dtype": "bf16", "wdtype": "bf16", "residual": True, "out": "same", "group": 0, "pad": 0, "offset": 0.0},
        # the hidden rows of one fused LM-head step (64 prompts x 16 rollouts x 64 tokens)
        {"name": "norm_fwd_lmhead_step", "op": "norm_fwd", "n": 65536, "h": 4096, "dtype": "bf16", "wdtype": "bf16", "residual": True, "out": "same", "group": 0, "pad": 0, "offset": 0.0},
        # a packed batch of 64 rollouts whose next product takes 8-bit rows scaled per 128 columns
        {"name": "norm_fwd_e4m3_groups", "op": "norm_fwd", "n": 33880, "h": 4096, "dtype": "bf16", "wdtype": "f32", "residual": True, "out": "both", "group": 128, "pad": 0, "offset": 0.0},
        # float32 rows of an odd width inside a wider buffer, 8-bit rows with one scale each
        {"name": "norm_fwd_odd_rows", "op": "norm_fwd", "n": 4099, "h": 2501, "dtype": "f32", "wdtype": "f32", "residual": False, "out": "e4m3", "group": 0, "pad": 6, "offset": 1.0},
        # backward of the fused LM-head step: dHidden comes in, the residual stream's gradient joins
        {"name": "norm_bwd_lmhead_step", "op": "norm_bwd", "n": 65536, "h": 4096, "dtype": "bf16", "wdtype": "bf16", "through": True, "pad": 0, "offset": 0.0},
        # one short response, odd width
        {"name": "norm_bwd_one_response", "op": "norm_bwd", "n": 131, "h": 1027, "dtype": "f32", "wdtype": "f32", "through": False, "pad": 0, "offset": 0.0},
        # the output layer's gradient and its norm's, before clipping at 1
        {"name": "grad_norm_output_layer", "op": "grad_norm", "rows": 151936, "h": 4096, "gains": 1, "ragged": 0, "ragged_max": 1, "layout": 0, "grad": "bf16"},
        # many small tensors of odd sizes, as adapters and gains are
        {"name": "grad_norm_many_small", "op": "grad_norm", "rows": 64, "h": 1024, "gains": 33, "ragged": 120, "ragged_max": 40000, "layout": 1, "grad": "f32"},
        # the output layer's update: bf16 weights with float32 master weights and states
        {"name": "adamw_output_layer", "op": "adamw", "rows": 151936, "h": 4096, "gains": 1, "ragged": 0, "ragged_max": 1, "layout": 0, "param": "bf16", "master": True, "grad": "bf16", "state": "f32", "seeded": False},
        # the same on the smallest memory: bf16 weights alone, 8-bit states, seeded rounding
        {"name": "adamw_8bit_output_layer", "op": "adamw", "rows": 128256, "h": 4096, "gains": 1, "ragged": 0, "ragged_max": 1, "layout": 0, "param": "bf16", "master": False, "grad": "bf16", "state": "e4m3", "seeded": True},
        # many small float32 tensors of odd sizes with 8-bit states
        {"name": "adamw_8bit_many_small", "op": "adamw", "rows": 64, "h": 1024, "gains": 33, "ragged": 120, "ragged_max": 40000, "layout": 2, "param": "f32", "master": False, "grad": "f32", "state": "e4m3", "seeded": False},
        # the smallest update there is: a gain vector
        {"name": "adamw_one_gain", "op": "adamw", "rows": 0, "h": 4096, "gains": 1, "ragged": 0, "ragged_max": 1, "layout": 0, "param": "f32", "master": False, "grad": "f32", "state": "f32", "seeded": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "grad_norm", "adamw", "adamw"])
    if op in ("norm_fwd", "norm_bwd"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        h = _spread(rng, 64, 16384)
        h = h if rng.random() < 0.4 else max(64, h // 64 * 64)          # odd widths among multiples of 64
        n = _spread(rng, 1, max(1, min(65536, 65536 * 4096 * 2 // (_BYTES[dtype] * h))))
        case = {"op": op, "n": n, "h": h, "dtype": dtype, "wdtype": rng.choice(["f32", dtype]),
                "pad": rng.choice([0, 0, 0, 8, 64, 5]), "offset": rng.choice([0.0, 0.0, 1.0])}
        if op == "norm_bwd":
            return case | {"through": rng.random() < 0.6}
        return case | {"residual": rng.random() < 0.7, "out": rng.choice(["same", "same", "e4m3", "both"]),
                       "group": rng.choice([0, 32, 64, 128, 256])}
    case = {"op": op, "rows": rng.choice([0, _spread(rng, 16, 65536)]), "h": _spread(rng, 64, 8192), "gains": rng.randint(1, 70),
            "ragged": rng.choice([0, 0, rng.randint(1, 200)]), "ragged_max": _spread(rng, 16, 200000), "layout": rng.randint(0, 1 << 30),
            "grad": rng.choice(["bf16", "f32"])}
    if op == "grad_norm":
        return case
    param = rng.choice(["bf16", "f32"])
    return case | {"param": param, "master": param == "bf16" and rng.random() < 0.5, "state": rng.choice(["f32", "e4m3"]),
                   "seeded": rng.random() < 0.5}


# ---- shapes of the tensor lists ----------------------------------------------------------------------------------

def _sizes(case):
    rng = random.Random(case["layout"])
    ragged = [_spread(rng, 1, case["ragged_max"]) for _ in range(case["ragged"])]
    return ([case["rows"] * case["h"]] if case["rows"] else []) + [case["h"]] * case["gains"] + ragged


def _decays(case):
    sizes = _sizes(case)
    gains = range(1 if case["rows"] else 0, (1 if case["rows"] else 0) + case["gains"])
    return [0.0 if k in gains else DECAY for k in range(len(sizes))]


def _blocks(case):
    return [-(-n // BLOCK) for n in _sizes(case)]


# ---- inputs -----------------------------------------------------------------------------------------------------

def _rows(g, n, h, pad, dtype, scale=None):
    """[n, h] rows of N(0, 1), by `scale` per column, in a buffer whose rows are h + pad apart."""
    wide = torch.empty(n, h + pad, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // (h + pad))
    for a in range(0, n, step):
        z = torch.randn(min(step, n - a), h + pad, generator=g, device="cuda")
        if scale is not None:
            z[:, :h] *= scale
        wide[a:a + step] = z
    return wide[:, :h]


def _flat(g, case, dtype, fill):
    """One buffer that holds the tensors one after the other, each from a multiple of BLOCK, zeros between them."""
    sizes, blocks = _sizes(case), _blocks(case)
    flat = torch.zeros(sum(blocks) * BLOCK, dtype=dtype, device="cuda")
    at = 0
    for n, b in zip(sizes, blocks):
        for a in range(0, n, 1 << 28):
            c = min(1 << 28, n - a)
            flat[at + a:at + a + c] = fill(torch.randn(c, generator=g, device="cuda"))
        at += b * BLOCK
    return flat


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op in ("norm_fwd", "norm_bwd"):
        n, h, pad, dtype = case["n"], case["h"], case["pad"], _TYPES[case["dtype"]]
        # a residual stream: channels of different size, a few of them far larger than the rest
        scale = torch.exp(0.5 * torch.randn(h, generator=g, device="cuda"))
        scale[torch.randint(0, h, (max(1, h // 512),), generator=g, device="cuda")] *= 30.0
        s["w"] = (1.0 - case["offset"] + 0.2 * torch.randn(h, generator=g, device="cuda")).to(_TYPES[case["wdtype"]])
        if op == "norm_fwd":
            s["x"] = _rows(g, n, h, pad, dtype)
            s["res"] = _rows(g, n, h, pad, dtype, scale) if case["residual"] else None
            s["h_out"] = torch.empty(n, h, dtype=dtype, device="cuda") if case["residual"] else None
            s["y"] = torch.empty(n, h, dtype=dtype, device="cuda") if case["out"] != "e4m3" else None
            s["q"] = torch.empty(n, h, dtype=torch.float8_e4m3fn, device="cuda") if case["out"] != "same" else None
            groups = -(-h // case["group"]) if case["group"] else 1
            s["scales"] = torch.empty(n, groups, device="cuda") if case["out"] != "same" else None
            s["rstd"] = torch.empty(n, device="cuda")
        else:
            s["dy"] = _rows(g, n, h, pad, dtype, torch.full((h,), 1e-3, device="cuda"))
            s["h"] = _rows(g, n, h, pad, dtype, scale)
            s["dh"] = _rows(g, n, h, pad, dtype, torch.full((h,), 1e-3, device="cuda")) if case["through"] else None
            s["rstd"] = torch.empty(n, device="cuda")
            step = max(1, (1 << 28) // h)
            for a in range(0, n, step):
                s["rstd"][a:a + step] = torch.rsqrt(s["h"][a:a + step].float().square().mean(1) + EPS_NORM)
            s["dx"] = torch.empty(n, h, dtype=dtype, device="cuda")
            s["dw"] = torch.empty(h, device="cuda")
        return s
    size = 1e-4 * math.exp(random.Random(seed).uniform(-1, 1))
    s["grad"] = _flat(g, case, _TYPES[case["grad"]], lambda z: z * size)
    if op == "grad_norm":
        s["norm"], s["coef"] = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        return s
    first = _flat(g, case, torch.float32, lambda z: z * 0.02)
    s["param"] = first.to(_TYPES[case["param"]])
    s["master"] = first if case["master"] else None
    m = _flat(g, case, torch.float32, lambda z: z * (0.3 * size))
    v = _flat(g, case, torch.float32, lambda z: (z * size).square() + 0.01 * size * size)
    if case["state"] == "f32":
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
    else:
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _to_codes(m, None, False), _to_codes(v.sqrt(), None, True)
    s["coef"] = torch.full((1,), 0.37, device="cuda")
    s["blocks"] = torch.tensor(_blocks(case), device="cuda")
    s["decay"] = torch.tensor(_decays(case), device="cuda")
    s["step"] = STEP0
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _e4m3(y, dither, floor):
    """|y| <= 448 (about) as e4m3: to nearest, or down after the addition of dither / 65536 of a step.  floor: what is above
    zero stays above zero."""
    if dither is None:
        q = y.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    else:
        a = y.abs()
        small = a < 2.0 ** -6           # below the normal values the step stays 2^-9, as it is from 2^-6 to 2^-5
        z = torch.where(small, a + 2.0 ** -6, a)
        z = ((z.view(torch.int32) + (dither << 4)) & ~0xFFFFF).view(torch.float32)
        z = torch.where(small, z - 2.0 ** -6, z).clamp(max=E4M3_MAX)
        q = torch.copysign(z, y).to(torch.float8_e4m3fn)
    if floor:
        q = torch.where((y > 0) & (q.float() == 0), E4M3_TINY, q.float()).to(torch.float8_e4m3fn)
    return q


def _to_codes(t, dither, floor):
    """A flat float32 buffer as e4m3 codes with a float32 scale for each BLOCK of them."""
    t = t.view(-1, BLOCK)
    scale = (t.abs().amax(1) / E4M3_MAX).clamp(min=SCALE_MIN)
    q = _e4m3(t * (1.0 / scale)[:, None], None if dither is None else dither.view(-1, BLOCK), floor)
    return q.view(-1), scale


def _signed(x):
    return x - (1 << 64) if x >= 1 << 63 else x


def _splitmix64(x):
    """The published SplitMix64 output function on int64 tensors (64-bit words in two's complement)."""
    x = x + _signed(0x9E3779B97F4A7C15)
    z = (x ^ ((x >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _dithers(n, step):
    """16 bits for the first state, the second state and the parameter of n elements: two elements share a 64-bit word,
    the parameter's bits are the first state's in reverse order."""
    key = _splitmix64(_splitmix64(torch.tensor(SEED)) + step).item()
    word = _splitmix64(torch.arange(-(-n // 2), device="cuda") + key)
    pair = torch.stack([word, word >> 32], 1).view(-1)[:n]
    rm, rv = (pair & 0xFFFF).int(), ((pair >> 16) & 0xFFFF).int()
    rp = ((rm & 0x5555) << 1) | ((rm >> 1) & 0x5555)
    rp = ((rp & 0x3333) << 2) | ((rp >> 2) & 0x3333)
    rp = ((rp & 0x0F0F) << 4) | ((rp >> 4) & 0x0F0F)
    return rm, rv, ((rp & 0x00FF) << 8) | (rp >> 8)


def _norm_fwd_plain(s):
    case = s["case"]
    h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
    rstd = torch.rsqrt(h.square().mean(1) + EPS_NORM)
    y = h * rstd[:, None] * (s["w"].float() + case["offset"])
    out = {"rstd": rstd}
    if s["h_out"] is not None:
        out["h"] = h.to(_TYPES[case["dtype"]])
    if s["y"] is not None:
        out["y"] = y.to(_TYPES[case["dtype"]])
    if s["q"] is not None:
        n, cols, group = case["n"], case["h"], case["group"] or case["h"]
        wide = torch.nn.functional.pad(y, (0, -cols % group)).view(n, -1, group)
        scale = (wide.abs().amax(2) / E4M3_MAX).clamp(min=SCALE_MIN)
        q = (wide * (1.0 / scale)[:, :, None]).view(n, -1)[:, :cols]
        out["q"], out["scales"] = _e4m3(q, None, False), scale
    return out


def _norm_bwd_plain(s):
    xhat = s["h"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    dw = (dy * xhat).sum(0)
    wdy = dy * (s["w"].float() + s["case"]["offset"])
    dx = (wdy - xhat * (wdy * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(_TYPES[s["case"]["dtype"]]), "dw": dw}


def _grad_norm_plain(s):
    norm = s["grad"].float().square().sum(dtype=torch.float64).sqrt().float().view(1)     # a long sum
    return {"norm": norm, "coef": MAX_NORM / norm.clamp(min=MAX_NORM)}


def _adamw_plain(s):
    case = s["case"]
    s["step"] += 1
    c1, c2 = 1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]
    n = s["param"].numel()
    rm, rv, rp = _dithers(n, s["step"]) if case["seeded"] else (None, None, None)
    g = s["grad"].float() * s["coef"]
    m, v = s["m"], s["v"]
    if case["state"] == "e4m3":
        m = (m.float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["v_scale"][:, None]).square().view(-1)
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    p = s["param"].float() if s["master"] is None else s["master"]
    decay = torch.repeat_interleave(s["decay"], s["blocks"], output_size=n // BLOCK)
    p = (p.view(-1, BLOCK) * (1.0 - LR * decay)[:, None]).view(-1) - (LR / c1) * (m / ((v / c2).sqrt() + EPS_ADAM))
    out = {}
    if s["master"] is not None:
        s["master"].copy_(p)
        out["master"] = s["master"]
    if rp is not None and case["param"] == "bf16" and s["master"] is None:
        p = ((p.view(torch.int32) + rp) & ~0xFFFF).view(torch.float32)
    s["param"].copy_(p)
    if case["state"] == "e4m3":
        (q, scale), (qv, scale_v) = _to_codes(m, rm, False), _to_codes(v.sqrt(), rv, True)
        s["m"].copy_(q), s["v"].copy_(qv), s["m_scale"].copy_(scale), s["v_scale"].copy_(scale_v)
        out |= {"m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    return out | {"param": s["param"], "m": s["m"], "v": s["v"]}


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _tensors(B, s):
    """The table of tensors that a user's program builds once, over the views of its flat buffers."""
    case, at, table = s["case"], 0, []
    for n, b, decay in zip(_sizes(case), _blocks(case), _decays(case)):
        cut = lambda name, k=BLOCK: None if s.get(name) is None else s[name][at * k:at * k + (n if k > 1 else b)]  # noqa: E731
        table.append(B.TensorSlot(grad=cut("grad"), param=cut("param"), master=cut("master"), m=cut("m"), v=cut("v"),
                                  m_scale=cut("m_scale", 1), v_scale=cut("v_scale", 1), weight_decay=decay,
                                  rng_first=at * BLOCK // 2))
        at += b
    return B.TensorList(table)


def _run_own(s):
    from paper_2605_07244_b200 import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "norm_fwd":
        if "np" not in s:
            s["np"] = B.NormParams(EPS_NORM, case["offset"], case["group"], 0)
        B.mrl_rmsnorm_residual_fwd(s["x"], s["res"], s["w"], s["np"], s["h_out"], s["y"], s["q"], s["scales"], s["rstd"])
        return {"rstd": s["rstd"], "h": s["h_out"], "y": s["y"], "q": s["q"], "scales": s["scales"]}
    if op == "norm_bwd":
        if "np" not in s:
            s["np"] = B.NormParams(EPS_NORM, case["offset"], 0, 0)
            s["ws"] = torch.empty(B.workspace_bytes(B.WS_RMSNORM_BWD, case["n"], 0, case["h"]), dtype=torch.uint8, device="cuda")
        B.mrl_rmsnorm_residual_bwd(s["dy"], s["dh"], s["h"], s["w"], s["rstd"], s["np"], s["dx"], s["dw"], s["ws"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if "list" not in s:
        s["list"] = _tensors(B, s)
        s["ws"] = torch.empty(B.workspace_bytes(B.WS_GRAD_NORM, 0, 0), dtype=torch.uint8, device="cuda")
        s["ap"] = B.AdamwParams(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS_ADAM, seed=SEED,
                                rounding=B.ROUND_SEEDED if case.get("seeded") else B.ROUND_NEAREST)
    if op == "grad_norm":
        B.mrl_grad_norm(s["list"], MAX_NORM, s["norm"], s["coef"], s["ws"])
        return {"norm": s["norm"], "coef": s["coef"]}
    s["step"] += 1
    s["ap"].step = s["step"]
    B.mrl_adamw_step(s["list"], s["ap"], grad_scale=s["coef"])
    return {k: s[k] for k in ("master", "m_scale", "v_scale", "param", "m", "v")}


def run(state):
    if own:
        return _run_own(state)
    return {"norm_fwd": _norm_fwd_plain, "norm_bwd": _norm_bwd_plain, "grad_norm": _grad_norm_plain,
            "adamw": _adamw_plain}[state["case"]["op"]](state)


def work(case):
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd"):
        n, h, e, w = case["n"], case["h"], _BYTES[case["dtype"]], _BYTES[case["wdtype"]]
        if op == "norm_bwd":
            return {"bytes": n * h * e * (4 if case["through"] else 3) + 4 * n + h * (w + 4), "flops": 10 * n * h}
        rows = e * (1 + 2 * case["residual"] + (case["out"] != "e4m3")) + (case["out"] != "same")
        groups = (-(-h // case["group"]) if case["group"] else 1) if case["out"] != "same" else 0
        return {"bytes": n * h * rows + 4 * n * (1 + groups) + h * w, "flops": 6 * n * h}
    total, count = sum(_sizes(case)), len(_sizes(case))
    if op == "grad_norm":
        return {"bytes": total * _BYTES[case["grad"]] + 8, "flops": 2 * total}
    param = _BYTES[case["param"]] + (8 if case["master"] else _BYTES[case["param"]])
    state = 16 * total if case["state"] == "f32" else 4 * total + 16 * sum(_blocks(case))
    return {"bytes": total * (_BYTES[case["grad"]] + param) + state + 8 * count, "flops": 16 * total}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _grouped_peak(y, group):
    """The largest magnitude of each group of columns, and the same spread over the columns."""
    n, h = y.shape
    which = torch.arange(h, device=y.device) // group
    peak = torch.zeros(n, int(which[-1]) + 1, dtype=y.dtype, device=y.device).scatter_reduce(1, which.expand(n, h), y.abs(), "amax")
    return peak, peak[:, which]


def exact(case, seed):
    """Unrounded: 8-bit codes as value / scale."""
    s = prepare(case, seed)
    wide = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"] == "norm_fwd":
        h = wide(s["x"]) + (wide(s["res"]) if case["residual"] else 0.0)
        length = (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["h"] + EPS_NORM).sqrt()
        y = (h / length) * (wide(s["w"]) + case["offset"])
        out = {"rstd": 1.0 / length[:, 0]}
        if case["residual"]:
            out["h"] = h
        if case["out"] != "e4m3":
            out["y"] = y
        if case["out"] != "same":
            peak, each = _grouped_peak(y, case["group"] or case["h"])
            out["scales"] = peak / E4M3_MAX
            out["q"] = torch.where(each > 0, y * E4M3_MAX / each, 0.0)
        return out
    if case["op"] == "norm_bwd":
        # y = h r (w + o) with r as it was stored, r' = -r^3 h / H
        h, r, dy, w = wide(s["h"]), wide(s["rstd"])[:, None], wide(s["dy"]), wide(s["w"]) + case["offset"]
        dw = torch.einsum("nh,nh,n->h", dy, h, r[:, 0])
        along = torch.einsum("nh,nh,h->n", dy, h, w)[:, None]
        dx = r * dy * w - r ** 3 * h * along / case["h"]
        return {"dx": dx + (wide(s["dh"]) if case["through"] else 0.0), "dw": dw}
    if case["op"] == "grad_norm":
        norm = torch.linalg.vector_norm(wide(s["grad"])).view(1)
        return {"norm": norm, "coef": torch.minimum(torch.ones_like(norm), MAX_NORM / norm)}
    t = STEP0 + 1
    g = wide(s["grad"]) * wide(s["coef"])
    m, v = wide(s["m"]), wide(s["v"])
    if case["state"] == "e4m3":
        m = m * wide(s["m_scale"]).repeat_interleave(BLOCK)
        v = (v * wide(s["v_scale"]).repeat_interleave(BLOCK)) ** 2
    m, v = m.lerp_(g, 1.0 - BETA1), v.lerp_(g.square_(), 1.0 - BETA2)
    p = wide(s["param"] if s["master"] is None else s["master"])
    decay = wide(s["decay"].repeat_interleave(s["blocks"] * BLOCK))
    step = (m / (1.0 - BETA1 ** t)).div_((v / (1.0 - BETA2 ** t)).sqrt_().add_(EPS_ADAM))
    p = p - LR * (step + decay * p)
    out = {"param": p}
    if case["master"]:
        out["master"] = p
    if case["state"] == "f32":
        return out | {"m": m, "v": v}
    for name, value in (("m", m), ("v", v.sqrt_())):
        peak = value.view(-1, BLOCK).abs().amax(1)
        out[name + "_scale"] = peak / E4M3_MAX
        out[name] = (value.view(-1, BLOCK) / (peak / E4M3_MAX).clamp(min=1e-300)[:, None]).view(-1)
    return out
