"""What scoring a frozen model in 8 bits and learning from its top alternatives is measured on: the cases, their inputs,
their plain form and their definition in 64 bits.

  quantize   weights or rows as e4m3 codes with a float32 scale per 128 x 128 or 1 x 128 block
  product    rows times weights, both such codes: the logits of a frozen peer, reference or teacher
  top        log-probs of given tokens with the entropy and the top alternatives of each row of logits
  distill    KL between a teacher's top alternatives (the rest of the vocabulary one more event, or left out) and the
             learner's logits, with its gradient

Plain forms are elementary torch operations in 32 bits; `own` makes the calls of the framework instead.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
BLOCK = 128

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # the output layer's weights, laid out once when a frozen model is loaded
        {"name": "quantize_output_layer", "op": "quantize", "n": 151936, "h": 4096, "dtype": "bf16", "rows": 128, "pad": 0},
        # float32 rows of an odd width in a wider buffer, a scale for each 128 of a row
        {"name": "quantize_odd_rows", "op": "quantize", "n": 4099, "h": 2501, "dtype": "f32", "rows": 1, "pad": 6},
        # one generated token's logits
        {"name": "product_one_token", "op": "product", "n": 1, "h": 4096, "v": 151936, "out": "bf16"},
        # a slab of response tokens scored by a frozen model
        {"name": "product_slab", "op": "product", "n": 4096, "h": 4096, "v": 151936, "out": "bf16"},
        # odd sizes all round, float32 logits
        {"name": "product_odd", "op": "product", "n": 777, "h": 1003, "v": 5003, "out": "f32"},
        # one generated token's alternatives
        {"name": "top_one_token", "op": "top", "n": 1, "v": 151936, "dtype": "bf16", "top": 20, "temperature": 1.0, "pad": 0, "masked": False},
        # the alternatives a teacher keeps for a slab of tokens
        {"name": "top_slab", "op": "top", "n": 8192, "v": 151936, "dtype": "bf16", "top": 64, "temperature": 1.0, "pad": 0, "masked": True},
        # float32 rows of an odd vocabulary in a wider buffer, the longest lists
        {"name": "top_odd_rows", "op": "top", "n": 2051, "v": 50021, "dtype": "f32", "top": 128, "temperature": 0.7, "pad": 3, "masked": False},
        # one short response
        {"name": "distill_one_response", "op": "distill", "n": 131, "v": 32003, "dtype": "bf16", "top": 20, "temperature": 1.0, "reverse": False, "rest": True, "pad": 0, "weighted": False},
        # a slab of the learner's own rollouts against a teacher's lists: the largest
        {"name": "distill_slab", "op": "distill", "n": 8192, "v": 128256, "dtype": "bf16", "top": 64, "temperature": 1.0, "reverse": True, "rest": True, "pad": 0, "weighted": True},
        # teacher's text at a higher temperature, its lists renormalised
        {"name": "distill_renormalised", "op": "distill", "n": 4096, "v": 151936, "dtype": "bf16", "top": 128, "temperature": 2.0, "reverse": False, "rest": False, "pad": 0, "weighted": False},
        # float32 logits of an odd vocabulary in a wider buffer
        {"name": "distill_odd_rows", "op": "distill", "n": 1021, "v": 50021, "dtype": "f32", "top": 8, "temperature": 1.0, "reverse": False, "rest": True, "pad": 3, "weighted": True},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "top", "top", "distill", "distill", "distill"])
    if op == "quantize":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        h = _spread(rng, 64, 16384)
        n = _spread(rng, 1, min(151936, 151936 * 4096 * 2 // (_BYTES[dtype] * h)))
        return {"op": op, "n": n, "h": h, "dtype": dtype, "rows": rng.choice([1, 128]), "pad": rng.choice([0, 0, 8, 5])}
    if op == "product":
        h = _spread(rng, 128, 8192)
        h = h if rng.random() < 0.3 else h // 128 * 128
        v = _spread(rng, 500, 151936)
        n = _spread(rng, 1, max(1, min(8192, 4096 * 4096 * 151936 // (h * v))))
        return {"op": op, "n": n, "h": h, "v": v, "out": rng.choice(["bf16", "bf16", "f32"])}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    v = _spread(rng, 1000, 160000)
    v = v if rng.random() < 0.4 else v // 64 * 64
    n = _spread(rng, 1, max(1, min(8192, 8192 * 128256 * 2 // (_BYTES[dtype] * v))))
    case = {"op": op, "n": n, "v": v, "dtype": dtype, "top": _spread(rng, 1, 128), "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]),
            "pad": rng.choice([0, 0, 0, 8, 64, 5])}
    if op == "top":
        return case | {"masked": rng.random() < 0.5}
    rest = rng.random() < 0.7
    return case | {"reverse": rest and rng.random() < 0.5, "rest": rest, "weighted": rng.random() < 0.5}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _rows(g, n, h, pad, dtype, fill):
    """[n, h] rows in a buffer whose rows are h + pad apart."""
    wide = torch.zeros(n, h + pad, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // h)
    for a in range(0, n, step):
        wide[a:a + step, :h] = fill(torch.randn(min(step, n - a), h, generator=g, device="cuda"))
    return wide[:, :h]


def _codes(g, n, h, rows, size):
    """Codes and scales of N(0, size^2) values in blocks of rows x 128; rows of codes start on 16 bytes."""
    x = _rows(g, n, h, 0, torch.float32, lambda z: z * size)
    q, scale = _quantize(x, rows)
    wide = torch.zeros(n, -(-h // 16) * 16, dtype=torch.float8_e4m3fn, device="cuda")
    wide[:, :h] = q
    return wide[:, :h], scale


def _logits(g, case):
    """Rows of N(0, 2^2) with one token far above the rest, as a model's logits are."""
    n, v = case["n"], case["v"]
    z = _rows(g, n, v, case["pad"], _TYPES[case["dtype"]], lambda z: z * 2.0)
    spike = torch.randint(0, v, (n, 1), generator=g, device="cuda")
    z.scatter_(1, spike, 12.0 + torch.randn(n, 1, generator=g, device="cuda").to(z.dtype))
    return z


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, n = case["op"], case["n"]
    s = {"case": case}
    if op == "quantize":
        h = case["h"]
        size = torch.exp(0.5 * torch.randn(h, generator=g, device="cuda")) * 0.02      # channels of different size
        s["x"] = _rows(g, n, h, case["pad"], _TYPES[case["dtype"]], lambda z: z * size)
        s["codes"] = torch.zeros(n, -(-h // 16) * 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :h]
        s["scales"] = torch.empty(-(-n // case["rows"]), -(-h // BLOCK), device="cuda")
    elif op == "product":
        s["x8"], s["x_scales"] = _codes(g, n, case["h"], 1, 1.0)
        s["w8"], s["w_scales"] = _codes(g, case["v"], case["h"], 128, 1.3 * case["h"] ** -0.5)
        s["out"] = torch.empty(n, case["v"], dtype=_TYPES[case["out"]], device="cuda")
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        v, top = case["v"], case["top"]
        s["logits"] = _logits(g, case)
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if op == "top":
            s["ids"] = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
            s["mask"] = (torch.rand(n, generator=g, device="cuda") < 0.9).to(torch.uint8) if case["masked"] else None
            s["top_ids"] = torch.empty(n, top, dtype=torch.int32, device="cuda")
            s |= {k: torch.empty(n, device="cuda") for k in ("logp", "lse", "entropy")}
            s["top_logp"] = torch.empty(n, top, device="cuda")
        else:
            # the teacher: the learner's logits with noise, its log-probs at the temperature, some lists shorter than others
            noisy = lambda: s["logits"].float() + torch.randn(n, v, generator=g, device="cuda")  # noqa: E731
            val, ids = noisy().div_(case["temperature"]).topk(top, 1)
            norm = (val[:, :1] + torch.log(torch.exp(val - val[:, :1]).sum(1, keepdim=True) * 1.2))    # a sixth for the rest
            length = torch.randint((top + 1) // 2, top + 1, (n, 1), generator=g, device="cuda")
            unused = torch.arange(top, device="cuda") >= length
            s["top_ids"] = ids.int().masked_fill(unused, -1)
            s["top_logp"] = (val - norm).masked_fill(unused, 0.0)
            s["mask"] = (torch.rand(n, generator=g, device="cuda") < 0.9).to(torch.uint8)
            s["mask"][0] = 1
            s["weight"] = torch.rand(n, generator=g, device="cuda") + 0.5 if case["weighted"] else None
            s["dlogits"] = torch.empty(n, v, dtype=_TYPES[case["dtype"]], device="cuda")
            s["row_kl"], s["loss"] = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _quantize(x, rows):
    """e4m3 codes (to nearest) and the scales of blocks of rows x 128; the last blocks may be short."""
    n, h = x.shape
    wide = torch.nn.functional.pad(x, (0, -h % BLOCK, 0, -n % rows)).view(-(-n // rows), rows, -1, BLOCK)
    scale = (wide.abs().amax((1, 3)).float() / E4M3_MAX).clamp(min=SCALE_MIN)
    q = (wide.float() * (1.0 / scale)[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(wide.shape[0] * rows, -1)[:n, :h], scale


def _values(codes, scales, rows):
    n, h = codes.shape
    return codes.float() * scales.repeat_interleave(rows, 0)[:n].repeat_interleave(BLOCK, 1)[:, :h]


def _product_plain(s):
    out = _values(s["x8"], s["x_scales"], 1) @ _values(s["w8"], s["w_scales"], 128).T
    return {"out": out.to(_TYPES[s["case"]["out"]])}


def _top_plain(s):
    case = s["case"]
    z = s["logits"].float()
    n, v = z.shape
    # largest first, the lowest index first among equals: one ordered whole number per logit
    bits = (z + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + ((1 << 32) - 1 - torch.arange(v, device="cuda"))
    top_ids = ((1 << 32) - 1 - (key.topk(case["top"], 1).values & 0xFFFFFFFF)).int()
    del bits, key
    x = z / case["temperature"]
    high = x.amax(1, keepdim=True)
    t = x - high
    e = t.exp()
    total = e.sum(1, keepdim=True)
    lse = high + total.log()
    out = {"logp": (x.gather(1, s["ids"].long()[:, None]) - lse)[:, 0], "lse": lse[:, 0],
           "entropy": (total.log() - (e * t).sum(1, keepdim=True) / total)[:, 0],
           "top_ids": top_ids, "top_logp": x.gather(1, top_ids.long()) - lse}
    if s["mask"] is not None:
        off = s["mask"] == 0
        out = {k: o.masked_fill(off if o.dim() == 1 else off[:, None], -1 if k == "top_ids" else 0) for k, o in out.items()}
    return out


def _lse(x):
    high = x.amax(1, keepdim=True)
    return high + (x - high).exp().sum(1, keepdim=True).log()


def _distill_plain(s):
    case = s["case"]
    x = s["logits"].float() / case["temperature"]
    n, v = x.shape
    used = s["top_ids"] >= 0
    at = s["top_ids"].long().clamp(min=0)
    listed = torch.zeros(n, v + 1, dtype=torch.bool, device="cuda")
    listed.scatter_(1, torch.where(used, at, v), True)          # unused places go to a column of their own
    listed = listed[:, :v]
    lse, lse_rest = _lse(x), _lse(x.masked_fill(listed, -math.inf))
    ln_p, ln_q = x.gather(1, at) - lse, s["top_logp"]
    q = ln_q.exp().masked_fill(~used, 0.0)
    if case["rest"]:
        q_rest = (1.0 - ln_q.double().exp().masked_fill(~used, 0.0).sum(1, keepdim=True)).clamp(min=1e-6).float()
        ln_p_rest = lse_rest - lse
        p, p_rest = ln_p.exp().masked_fill(~used, 0.0), ln_p_rest.exp()
        if case["reverse"]:
            ratio, ratio_rest = (ln_p - ln_q).masked_fill(~used, 0.0), ln_p_rest - q_rest.log()
            kl = (p * ratio).sum(1, keepdim=True) + p_rest * ratio_rest
            at_listed, of_rest = p * (ratio - kl), p_rest * (ratio_rest - kl)
        else:
            mass = q.sum(1, keepdim=True) + q_rest
            kl = (q * (ln_q - ln_p)).sum(1, keepdim=True) + q_rest * (q_rest.log() - ln_p_rest)
            at_listed, of_rest = mass * p - q, mass * p_rest - q_rest
    else:
        norm = _lse(ln_q.masked_fill(~used, -math.inf))
        q = q * (-norm).exp()
        kl = (q * (ln_q - norm - ln_p)).sum(1, keepdim=True)
        p = ln_p.exp().masked_fill(~used, 0.0)
        at_listed, of_rest = p - q, (lse_rest - lse).exp()
    on = s["mask"][:, None] != 0
    c = on / on.sum()
    if s["weight"] is not None:
        c = c * s["weight"][:, None]
    d = torch.zeros(n, v + 1, device="cuda")
    torch.mul((x - lse_rest).exp(), of_rest * c / case["temperature"], out=d[:, :v])
    d.scatter_(1, torch.where(used, at, v), at_listed * c / case["temperature"])
    kl = kl.masked_fill(~on, 0.0)
    return {"loss": (c * kl).double().sum().float().view(1), "row_kl": kl[:, 0], "dlogits": d[:, :v].to(_TYPES[case["dtype"]])}


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2605_07244_b200 import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "quantize":
        B.mrl_e4m3_quantize(s["x"], s["codes"], s["scales"], case["rows"])
        return {"codes": s["codes"], "scales": s["scales"]}
    if op == "product":
        B.mrl_e4m3_product(s["x8"], s["x_scales"], s["w8"], s["w_scales"], s["out"], s["status"])
        return {"out": s["out"]}
    if op == "top":
        B.mrl_top_logprobs(s["logits"], s["ids"], s["mask"], case["temperature"], s["logp"], s["lse"], s["entropy"], s["top_ids"],
                           s["top_logp"], s["status"])
        return {k: s[k] for k in ("logp", "lse", "entropy", "top_ids", "top_logp")}
    if "dp" not in s:
        s["dp"] = B.DistillParams(temperature=case["temperature"], coeff=1.0, rest_floor=1e-6,
                                  direction=B.DISTILL_REVERSE if case["reverse"] else B.DISTILL_FORWARD,
                                  rest=B.REST_EVENT if case["rest"] else B.REST_NONE)
        s["ws"] = torch.empty(B.workspace_bytes(B.WS_DISTILL, case["n"], case["v"]), dtype=torch.uint8, device="cuda")
    B.mrl_distill_loss_fwd_bwd(s["logits"], s["top_ids"], s["top_logp"], s["mask"], s["weight"], s["dp"], s["dlogits"], s["row_kl"],
                               s["loss"], None, s["status"], s["ws"])
    return {k: s[k] for k in ("loss", "row_kl", "dlogits")}


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "quantize":
        codes, scales = _quantize(state["x"], case["rows"])
        return {"codes": codes, "scales": scales}
    return {"product": _product_plain, "top": _top_plain, "distill": _distill_plain}[case["op"]](state)


def work(case):
    op, n = case["op"], case["n"]
    if op == "quantize":
        scales = -(-n // case["rows"]) * -(-case["h"] // BLOCK)
        return {"bytes": n * case["h"] * (_BYTES[case["dtype"]] + 1) + 4 * scales, "flops": 3 * n * case["h"]}
    if op == "product":
        h, v = case["h"], case["v"]
        scales = (n + -(-v // 128)) * -(-h // BLOCK)
        return {"bytes": (n + v) * h + 4 * scales + n * v * _BYTES[case["out"]], "flops": 2 * n * h * v}
    v, e, top = case["v"], _BYTES[case["dtype"]], case["top"]
    if op == "top":
        return {"bytes": n * v * e + n * (16 + 8 * top + case["masked"]), "flops": 6 * n * v}
    return {"bytes": 2 * n * v * e + n * (5 + 8 * top + 4 * case["weighted"]), "flops": 8 * n * v}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _blocks(n, rows, device="cuda"):
    return torch.arange(n, device=device) // rows


def _exact_distill(case, s):
    """The loss in float64 as it is defined; the gradient by differentiating it."""
    z = s["logits"].to(torch.float64).requires_grad_()
    n, v = z.shape
    rows = torch.arange(n, device="cuda")[:, None].expand_as(s["top_ids"])
    used = s["top_ids"] >= 0
    outside = torch.zeros(n, v, dtype=torch.float64, device="cuda")
    outside[rows[used], s["top_ids"].long()[used]] = -math.inf
    ln_p = torch.log_softmax(z / case["temperature"], 1)
    mine = ln_p.gather(1, s["top_ids"].long().clamp(min=0)).where(used, 0.0)
    theirs = s["top_logp"].to(torch.float64)
    q = theirs.exp().where(used, 0.0)
    if case["rest"]:
        rest = (1.0 - q.sum(1)).clamp(min=float(torch.tensor(1e-6)))
        rest_mine = torch.logsumexp(ln_p + outside, 1)
        if case["reverse"]:
            kl = (mine.exp() * (mine - theirs)).where(used, 0.0).sum(1) + rest_mine.exp() * (rest_mine - rest.log())
        else:
            kl = (q * (theirs - mine)).sum(1) + rest * (rest.log() - rest_mine)
    else:
        share = q / q.sum(1, keepdim=True)
        kl = (torch.special.xlogy(share, share) - share * mine).sum(1)
    on = s["mask"] != 0
    kl = kl.where(on, 0.0)
    loss = (kl * (1.0 if s["weight"] is None else s["weight"].to(torch.float64))).sum() / on.sum()
    grad, = torch.autograd.grad(loss, z)
    return {"loss": loss.detach().view(1), "row_kl": kl.detach(), "dlogits": grad}


def exact(case, seed):
    """Unrounded: 8-bit codes as value / scale."""
    s = prepare(case, seed)
    wide = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"] == "quantize":
        x, (n, h) = wide(s["x"]), s["x"].shape
        down, across = _blocks(n, case["rows"]), _blocks(h, BLOCK)
        peak = torch.zeros(n, int(across[-1]) + 1, dtype=torch.float64, device="cuda").scatter_reduce_(1, across.expand(n, h), x.abs(), "amax")
        peak = torch.zeros(int(down[-1]) + 1, peak.shape[1], dtype=torch.float64, device="cuda").scatter_reduce_(
            0, down[:, None].expand_as(peak), peak, "amax")
        scale = (peak / E4M3_MAX).clamp(min=SCALE_MIN)
        return {"codes": x / scale[down][:, across], "scales": scale}
    if case["op"] == "product":
        across = _blocks(case["h"], BLOCK)
        x = wide(s["x8"].float()) * wide(s["x_scales"])[:, across]
        w = wide(s["w8"].float()) * wide(s["w_scales"])[_blocks(case["v"], 128)][:, across]
        return {"out": torch.einsum("nh,vh->nv", x, w)}
    if case["op"] == "distill":
        return _exact_distill(case, s)
    z = wide(s["logits"]) / case["temperature"]
    lse = torch.logsumexp(z, 1)
    out = {"logp": z.gather(1, s["ids"].long()[:, None])[:, 0] - lse, "lse": lse, "top_logp": z.topk(case["top"], 1).values - lse[:, None]}
    ln_p = z.sub_(lse[:, None])
    out["entropy"] = -torch.linalg.vecdot(ln_p.exp(), ln_p)
    if s["mask"] is not None:
        for o in out.values():
            o[s["mask"] == 0] = 0
    return out | {"top_ids": None}
