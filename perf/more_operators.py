"""The operators between the residual stream and the attention call, as a transformer block runs them: root-mean-square norm with the
residual's addition, 8-bit quantisation with a scale per block of 128, the product of two such matrices (projections and their
gradients), and the pack with rotary positions.

A case is a dict with an "op" and the sizes of that operator:

    rms_fwd   rows, D, groups (rows that share a weight), x and res types ("none": no residual), y type ("e4m3": 8 bits with scales)
    rms_bwd   rows, D, groups, dy and h types, dres (whether the residual stream has a gradient of its own)
    quant     rows, cols, x type, fp8 type, block (rows of a block: 1 or 128), order ("rows", "cols" or "both")
    matmul    M, N, K, a ("e4m3" or "e5m2"), block (rows of a block of b), bias; the result is bf16
    rope, rope_bwd   B, S, H, d, rot (columns that turn), layout, axes (1, or 3 with a gh x gw grid a frame), x type, fused (x is the first third
              of a fused projection), unit_rms, factor (of the context's extension), first (the first position)

Scales are powers of two, held as exponents in a byte: the block's largest value lands in the upper half of the type's range.  Rows of 8-bit
matrices are padded with zeros to whole blocks of 128.  Everything is made on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
SIZE = {"none": 0, "fp32": 4, "bf16": 2, "e4m3": 1, "e5m2": 1}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}          # the largest value of the type, 1.75 times a power of two

LARGEST_ROWS = 119056 * 1536                    # elements of the largest listed norm, quantisation and pack
LARGEST_FLOPS = 2.0 * 119056 * 4608 * 1536      # operations of the largest listed product


def listed():
    return [
        # one token: a conditioning vector on its way to an 8-bit projection; latency only
        {"name": "rms_fwd_one_token", "op": "rms_fwd", "rows": 1, "D": 1536, "groups": 1, "x": "bf16", "res": "fp32", "y": "e4m3"},
        # the fp32 residual stream of a 720p clip takes a branch's result and goes to an 8-bit projection
        {"name": "rms_fwd_720p", "op": "rms_fwd", "rows": 119056, "D": 1536, "groups": 1, "x": "bf16", "res": "fp32", "y": "e4m3"},
        # back into that stream, whose own gradient is added
        {"name": "rms_bwd_720p", "op": "rms_bwd", "rows": 119056, "D": 1536, "groups": 1, "dy": "bf16", "h": "fp32", "dres": True},
        # a fused projection's weight after an optimiser step: for the forward product and, in the other order, for the gradient's
        {"name": "quant_weight", "op": "quant", "rows": 4608, "cols": 1536, "x": "fp32", "fp8": "e4m3", "block": 128, "order": "both"},
        # the gradient of a projection's result: by rows for the gradient of its input, by columns for the gradient of its weight
        {"name": "quant_720p", "op": "quant", "rows": 119056, "cols": 1536, "x": "bf16", "fp8": "e5m2", "block": 1, "order": "both"},
        # one token through a fused projection: the weight's bytes
        {"name": "matmul_one_token", "op": "matmul", "M": 1, "N": 4608, "K": 1536, "a": "e4m3", "block": 128, "bias": True},
        # 256 text tokens from an encoder of another width
        {"name": "matmul_text", "op": "matmul", "M": 256, "N": 1536, "K": 4096, "a": "e4m3", "block": 128, "bias": True},
        # the fused projection of a 720p clip's tokens to queries, keys and values
        {"name": "matmul_720p", "op": "matmul", "M": 119056, "N": 4608, "K": 1536, "a": "e4m3", "block": 128, "bias": True},
        # the gradient of that projection's weight: a sum over all tokens
        {"name": "matmul_weight_grad", "op": "matmul", "M": 4608, "N": 1536, "K": 119056, "a": "e5m2", "block": 1, "bias": False},
        # single tokens of a batch at far positions, in a context extended four times
        {"name": "rope_token", "op": "rope", "B": 8, "S": 1, "H": 12, "d": 128, "rot": 64, "layout": "half", "axes": 1, "gh": 1, "gw": 1, "x": "bf16",
         "fused": True, "unit_rms": False, "factor": 4.0, "first": 119055},
        # the normalised queries of a 720p clip (33 x 45 x 80 grid and 256 text tokens), a part of the head for each axis
        {"name": "rope_720p", "op": "rope", "B": 1, "S": 119056, "H": 12, "d": 128, "rot": 128, "layout": "interleaved", "axes": 3, "gh": 45, "gw": 80,
         "x": "bf16", "fused": True, "unit_rms": True, "factor": 1.0, "first": 0},
        # the gradient of the same step for a ragged batch of two, half of a head of 64
        {"name": "rope_bwd_batch_d64", "op": "rope_bwd", "B": 2, "S": 4797, "H": 12, "d": 64, "rot": 32, "layout": "half", "axes": 1, "gh": 1, "gw": 1,
         "x": "fp32", "fused": False, "unit_rms": True, "factor": 1.0, "first": 7},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms_fwd", "rms_fwd", "rms_bwd", "quant", "quant", "matmul", "matmul", "matmul", "matmul", "rope", "rope", "rope_bwd"])
    while True:
        width = rng.choice([64 * rng.randint(2, 64), _log_int(rng, 30, 8192)])
        if op in ("rms_fwd", "rms_bwd"):
            groups = rng.choice([1, 1, 2, 4])
            case = {"op": op, "rows": groups * _log_int(rng, 1, 60000), "D": width, "groups": groups}
            if op == "rms_fwd":
                case.update(x=rng.choice(["fp32", "bf16", "bf16"]), res=rng.choice(["none", "fp32", "bf16"]), y=rng.choice(["fp32", "bf16", "e4m3", "e4m3"]))
            else:
                case.update(dy=rng.choice(["fp32", "bf16", "bf16"]), h=rng.choice(["fp32", "bf16"]), dres=rng.random() < 0.6)
            if case["rows"] * case["D"] <= LARGEST_ROWS:
                return case
        elif op == "quant":
            case = {"op": op, "rows": _log_int(rng, 1, 119056), "cols": width, "x": rng.choice(["fp32", "bf16"]), "fp8": rng.choice(["e4m3", "e4m3", "e5m2"]),
                    "block": rng.choice([1, 1, 128]), "order": rng.choice(["rows", "cols", "both", "both"])}
            if case["rows"] * case["cols"] <= LARGEST_ROWS:
                return case
        elif op == "matmul":
            long = rng.random() < 0.25
            tokens = _log_int(rng, 1, 119056)
            case = {"op": op, "M": width if long else tokens, "N": rng.choice([64 * rng.randint(2, 64), _log_int(rng, 30, 8192)]), "K": tokens if long else width,
                    "a": rng.choice(["e4m3", "e4m3", "e5m2"]), "block": 1 if long else rng.choice([1, 128, 128]), "bias": rng.random() < 0.5}
            if work(case)["flops"] <= LARGEST_FLOPS / 2:
                return case
        else:
            d = rng.choice([64, 128, 128])
            axes = rng.choice([1, 1, 3])
            case = {"op": op, "B": rng.choice([1, 1, 2, 5]), "S": _log_int(rng, 1, 119056), "H": rng.randint(1, 24), "d": d,
                    "rot": rng.choice([d, d, d // 2, 8 * rng.randint(2, d // 8)]), "layout": rng.choice(["interleaved", "half"]), "axes": axes,
                    "gh": rng.randint(8, 45) if axes == 3 else 1, "gw": rng.randint(8, 80) if axes == 3 else 1, "x": rng.choice(["fp32", "bf16"]),
                    "fused": rng.random() < 0.5, "unit_rms": rng.random() < 0.5, "factor": rng.choice([1.0, 1.0, 4.0, 16.0]),
                    "first": rng.choice([0, rng.randint(0, 1000000)]) if axes == 1 else 0}
            if case["B"] * case["S"] * case["H"] * d <= LARGEST_ROWS:
                return case


def _up(n, m):
    return (n + m - 1) // m * m


def _exponent(top, most):
    """The smallest e with top <= most * 2^e, as a 32-bit integer; 0 where there is nothing but zeros.  most = 1.75 * 2^p."""
    m, p = torch.frexp(top)
    e = p - 1 - int(math.log2(most)) + (m > 0.875).int()
    return torch.where(top == 0, torch.zeros_like(e), e.clamp(-127, 127))


def _power(e):
    """2^e in 32 bits, exactly: exponents as a float holds them."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x, kind, block):
    """x [rows, cols] -> 8-bit values [rows, cols padded to 128], scales [rows or blocks of 128 of them, blocks of columns padded to 4]."""
    rows, cols = x.shape
    r, c = _up(rows, block), _up(cols, 128)
    x = torch.nn.functional.pad(x.float(), (0, c - cols, 0, r - rows)).view(r // block, block, c // 128, 128)
    e = _exponent(x.abs().amax(dim=(1, 3)), TOP[kind])
    q = (x * _power(-e)[:, None, :, None]).view(r, c)[:rows].to(TYPES[kind])
    scales = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, _up(c // 128, 4) - c // 128), value=127)
    return q, scales.view(torch.float8_e8m0fnu)


def _values(q, scales, block):
    """What an 8-bit matrix stands for."""
    s = _power(scales.view(torch.uint8)[:, :q.shape[1] // 128].int() - 127)
    s = s.repeat_interleave(block, dim=0)[:q.shape[0]] if block > 1 else s
    return (q.float().view(q.shape[0], -1, 128) * s[:, :, None]).view(q.shape)


def _axis_pairs(case):
    """Pairs of columns that turn with each axis: an eighth with the frame, the rest with row and column."""
    n = case["rot"] // 2
    return [n] if case["axes"] == 1 else [n - 2 * ((n - n // 8) // 2), (n - n // 8) // 2, (n - n // 8) // 2]


def _frequencies(case):
    """Radians a position for every pair: base 10 000 on each axis; for a context extended by `factor` the slow pairs (under one turn in the original
    4 096 positions) are slowed by it, the fast ones (over 32 turns) kept, those between in proportion to their turns."""
    out = []
    for n in _axis_pairs(case):
        for i in range(n):
            f = 10000.0 ** (-i / n)
            keep = min(1.0, max(0.0, (4096 * f / (2 * math.pi) - 1) / (32 - 1)))
            out.append(f if case["factor"] == 1.0 else f * keep + f / case["factor"] * (1 - keep))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dev = case["op"], "cuda"
    st = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def uneven(rows, cols):                             # rows of different size, some columns larger than others
        x = normal(rows, cols) * torch.exp(0.5 * normal(rows, 1))
        return x.mul_(torch.exp(0.5 * normal(1, cols)))

    if op in ("rms_fwd", "rms_bwd"):
        rows, D, G = case["rows"], case["D"], case["groups"]
        st["weight"] = 1 + 0.2 * normal(G, D)
        if op == "rms_fwd":
            st["x"] = uneven(rows, D).to(TYPES[case["x"]])
            st["rstd"] = torch.empty(rows, device=dev)
            st["y"] = torch.empty(rows, _up(D, 128) if case["y"] == "e4m3" else D, device=dev, dtype=TYPES[case["y"]])
            if case["y"] == "e4m3":
                st["y_scales"] = torch.full((rows, _up(_up(D, 128) // 128, 4)), 127, device=dev, dtype=torch.uint8).view(torch.float8_e8m0fnu)
            if case["res"] != "none":
                st["res"] = (3 * uneven(rows, D)).to(TYPES[case["res"]])
                st["h"] = torch.empty_like(st["res"])
        else:
            h = (3 * uneven(rows, D)).to(TYPES[case["h"]])
            st.update(h=h, rstd=(h.double().square().mean(dim=-1) + EPS).rsqrt().float(), dy=normal(rows, D).to(TYPES[case["dy"]]),
                      dh=torch.empty_like(h), dweight=torch.empty(G, D, device=dev))
            if case["dres"]:
                st["dres"] = normal(rows, D).to(TYPES[case["h"]])
    elif op == "quant":
        rows, cols, blk = case["rows"], case["cols"], case["block"]
        st["x"] = uneven(rows, cols).to(TYPES[case["x"]])
        for order, name, r, c in (("rows", "q", rows, cols), ("cols", "qt", cols, rows)):
            if case["order"] in (order, "both"):
                st[name] = torch.empty(r, _up(c, 128), device=dev, dtype=TYPES[case["fp8"]])
                st[name + "_scales"] = torch.full((_up(r, blk) // blk, _up(_up(c, 128) // 128, 4)), 127, device=dev, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    elif op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        st["a"], st["a_scales"] = _quantise(uneven(M, K), case["a"], 1)
        st["b"], st["b_scales"] = _quantise(normal(N, K) * K ** -0.5, "e4m3", case["block"])
        st["bias"] = normal(N) if case["bias"] else None
        st["out"] = torch.empty(M, N, device=dev, dtype=torch.bfloat16)
    else:
        B, S, H, d = case["B"], case["S"], case["H"], case["d"]
        def tokens():                                   # token-major heads, alone or beside two others as a fused projection leaves them
            n = 3 if case["fused"] else 1
            return normal(B, S, n, H, d).to(TYPES[case["x"]])[:, :, 0]
        st["freqs"] = _frequencies(case)
        if case["axes"] == 3:                           # frame, row and column of every token, shared by the batch
            s = torch.arange(S, device=dev)
            st["positions"] = torch.stack([s // (case["gh"] * case["gw"]), s // case["gw"] % case["gh"], s % case["gw"]], dim=-1).int()
        elif S == 1:                                    # single tokens: each sequence of the batch is somewhere else
            st["positions"] = (case["first"] - 977 * torch.arange(B, device=dev)).clamp(min=0).int().view(B, 1, 1)
        else:
            st["positions"] = None
        st["premul"] = 0.1 * math.log(case["factor"]) + 1.0
        st["x"] = tokens()
        if op == "rope":
            st["y"] = torch.empty(B, H, S, d, device=dev, dtype=torch.bfloat16)
        else:
            st["dy"] = normal(B, H, S, d).to(torch.bfloat16)
            st["dx"] = torch.empty(B, S, 3 if case["fused"] else 1, H, d, device=dev, dtype=TYPES[case["x"]])[:, :, 0]
    return st


def _own(st):
    import paper_2511_12056_amd as pda
    case, op = st["case"], st["case"]["op"]
    if op == "rms_fwd":
        pda.rms_norm_fwd(st["x"], st["weight"], st["y"], res=st.get("res"), h=st.get("h"), y_scales=st.get("y_scales"), rstd=st["rstd"], eps=EPS)
        return {n: st[n] for n in ("h", "y", "y_scales", "rstd") if n in st}
    if op == "rms_bwd":
        if "workspace" not in st:                       # kept with the activations' buffers, as a training loop does
            st["workspace"] = pda.rms_norm_bwd_workspace(case["rows"], case["D"], case["groups"])
        pda.rms_norm_bwd(st["dy"], st["h"], st["weight"], st["rstd"], st["dh"], st["dweight"], dres=st.get("dres"), workspace=st["workspace"])
        return {"dh": st["dh"], "dweight": st["dweight"]}
    if op == "quant":
        pda.fp8_quant(st["x"], st.get("q"), st.get("q_scales"), st.get("qt"), st.get("qt_scales"), block_rows=case["block"])
        return {n: st[n] for n in ("q", "q_scales", "qt", "qt_scales") if n in st}
    if op == "matmul":
        if "workspace" not in st:
            st["workspace"] = pda.fp8_matmul_workspace(case["M"], case["N"], case["K"])
        return pda.fp8_matmul(st["a"], st["a_scales"], st["b"], st["b_scales"], st["out"], bias=st["bias"], workspace=st["workspace"])
    if "rope" not in st:                                # the description of the rotation, which a model keeps
        st["rope"] = pda.Rope(st["freqs"], layout=case["layout"], axis_pairs=_axis_pairs(case))
    where = {"first": case["first"]} if st["positions"] is None else {"positions": st["positions"]}
    if op == "rope":
        return pda.pack_heads_rope(st["x"], st["y"], st["rope"], unit_rms=case["unit_rms"], premul=st["premul"], **where)
    return pda.pack_heads_rope_bwd(st["dy"], st["x"] if case["unit_rms"] else None, st["dx"], st["rope"], unit_rms=case["unit_rms"],
                                   premul=st["premul"], **where)


def _turns(st):
    """cos and sin of every token's angles [B or 1, S, 1, rot / 2], in 64 bits."""
    case = st["case"]
    f = torch.tensor(st["freqs"], device="cuda", dtype=torch.float64)
    pos = st["positions"]
    if pos is None:
        angle = torch.arange(case["first"], case["first"] + case["S"], device="cuda", dtype=torch.float64)[None, :, None] * f
    else:
        axis = torch.repeat_interleave(torch.arange(case["axes"]), torch.tensor(_axis_pairs(case))).cuda()
        angle = pos.double().view(-1, case["S"], case["axes"])[:, :, axis] * f
    return torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]


def _turn(x, cos, sin, case):
    """Turns the pairs of the first rot columns of x [..., d] by the angles; the other columns stay."""
    rot = case["rot"]
    part = x[..., :rot]
    if case["layout"] == "half":
        u, v = part[..., :rot // 2], part[..., rot // 2:]
        turned = torch.cat([u * cos - v * sin, u * sin + v * cos], dim=-1)
    else:
        u, v = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([u * cos - v * sin, u * sin + v * cos], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def run(st):
    if own:
        return _own(st)
    case, op = st["case"], st["case"]["op"]
    if op == "rms_fwd":
        G, D = case["groups"], case["D"]
        h = st["x"] if case["res"] == "none" else (st["x"].float() + st["res"].float()).to(TYPES[case["res"]])
        x = h.float().view(G, -1, D)
        rstd = (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
        y = (x * rstd * st["weight"].view(G, 1, D)).view(-1, D)
        out = {"rstd": rstd.view(-1)}
        if case["res"] != "none":
            out["h"] = h
        if case["y"] == "e4m3":
            out["y"], out["y_scales"] = _quantise(y, "e4m3", 1)
        else:
            out["y"] = y.to(TYPES[case["y"]])
        return out
    if op == "rms_bwd":
        G, D = case["groups"], case["D"]
        rstd, dy = st["rstd"].view(G, -1, 1), st["dy"].float().view(G, -1, D)
        hh = st["h"].float().view(G, -1, D) * rstd
        g = dy * st["weight"].view(G, 1, D)
        dh = ((g - hh * (g * hh).mean(dim=-1, keepdim=True)) * rstd).view(-1, D)
        if case["dres"]:
            dh = dh + st["dres"].float()
        return {"dh": dh.to(TYPES[case["h"]]), "dweight": (dy * hh).sum(dim=1)}
    if op == "quant":
        out = {}
        if "q" in st:
            out["q"], out["q_scales"] = _quantise(st["x"], case["fp8"], case["block"])
        if "qt" in st:
            out["qt"], out["qt_scales"] = _quantise(st["x"].t(), case["fp8"], case["block"])
        return out
    if op == "matmul":
        a, b = _values(st["a"], st["a_scales"], 1), _values(st["b"], st["b_scales"], case["block"])
        out = torch.matmul(a, b.t())
        return (out if st["bias"] is None else out + st["bias"]).to(torch.bfloat16)
    cos, sin = (t.float() for t in _turns(st))
    if op == "rope":
        x = st["x"].float()
        if case["unit_rms"]:
            x = x * x.square().mean(dim=-1, keepdim=True).rsqrt()
        return (_turn(x, cos, sin, case) * st["premul"]).transpose(1, 2).to(torch.bfloat16, memory_format=torch.contiguous_format)
    dy = _turn(st["dy"].float().transpose(1, 2), cos, -sin, case)
    if case["unit_rms"]:
        x = st["x"].float()
        r = x.square().mean(dim=-1, keepdim=True).rsqrt()
        xh = x * r
        dy = (dy - xh * (dy * xh).mean(dim=-1, keepdim=True)) * r
    return (dy * st["premul"]).to(TYPES[case["x"]])


def _blocks_exact(x, kind, block, rounded):
    """The block's values over their scale and the scales, in 64 bits.  rounded: to the type, ties to even."""
    rows, cols = x.shape
    r, c = _up(rows, block), _up(cols, 128)
    full = torch.zeros(r, c, device=x.device, dtype=torch.float64)
    full[:rows, :cols] = x.abs()
    top = full.view(r // block, block, c // 128, 128).permute(0, 2, 1, 3).flatten(2).amax(dim=-1)
    over, e = torch.frexp(top / TOP[kind])              # over * 2^e, 1/2 <= over < 1: a power of two itself is enough for 1/2
    e = torch.where(top > 0, e - (over == 0.5).int(), torch.zeros_like(e)).clamp(-127, 127)
    scale = ((e.long() + 1023) << 52).view(torch.float64)
    q = torch.zeros(rows, c, device=x.device, dtype=torch.float64)
    q[:, :cols] = x / scale.repeat_interleave(block, dim=0)[:rows].repeat_interleave(128, dim=1)[:, :cols]
    if rounded:                                         # a type of m bits behind the point: steps of 2^-m of the value's power of two, down to its smallest
        m, least = (3, -6) if kind == "e4m3" else (2, -14)
        step = ((torch.frexp(q)[1].sub(1).clamp(min=least) - m + 1023).long() << 52).view(torch.float64)
        q = torch.round(q / step) * step
    padded = torch.ones(r // block, _up(c // 128, 4), device=x.device, dtype=torch.float64)
    padded[:, :c // 128] = scale
    return q, padded


def exact(case, seed):
    """What `run` returns, in 64 bits from the definitions; the 8-bit values of a norm before their rounding, which hangs on its last bit."""
    st = prepare(case, seed)
    op = case["op"]
    if op == "rms_fwd":
        D = case["D"]
        w = st["weight"].double().repeat_interleave(case["rows"] // case["groups"], dim=0)
        out = {}
        if case["res"] == "none":
            h = st["x"].double()
        else:                                           # what is normalised is the stream as it is stored
            out["h"] = st["x"].double() + st["res"].double()
            h = out["h"].to(TYPES[case["res"]]).double()
        norm = torch.linalg.vector_norm(h, dim=-1)
        out["rstd"] = 1 / torch.sqrt(norm * norm / D + EPS)
        y = h * out["rstd"][:, None] * w
        if case["y"] == "e4m3":
            out["y"], out["y_scales"] = _blocks_exact(y, "e4m3", 1, False)
        else:
            out["y"] = y
        return out
    if op == "rms_bwd":
        D, per = case["D"], case["rows"] // case["groups"]
        h, dy, r = st["h"].double(), st["dy"].double(), st["rstd"].double()[:, None]
        g = dy * st["weight"].double().repeat_interleave(per, dim=0)
        dh = r * g - h * r ** 3 * torch.sum(g * h, dim=-1, keepdim=True) / D
        if case["dres"]:
            dh = dh + st["dres"].double()
        return {"dh": dh, "dweight": (dy * h * r).view(case["groups"], per, D).sum(dim=1)}
    if op == "quant":
        x, out = st["x"].double(), {}
        if "q" in st:
            out["q"], out["q_scales"] = _blocks_exact(x, case["fp8"], case["block"], True)
        if "qt" in st:
            out["qt"], out["qt_scales"] = _blocks_exact(x.t().contiguous(), case["fp8"], case["block"], True)
        return out
    if op == "matmul":
        a, b = st["a"].double(), st["b"].double()
        a *= st["a_scales"].double()[:, :a.shape[1] // 128].repeat_interleave(128, dim=1)
        b *= st["b_scales"].double()[:, :b.shape[1] // 128].repeat_interleave(128, dim=1).repeat_interleave(case["block"], dim=0)[:case["N"]]
        out = torch.mm(a, b.t().contiguous())
        return out if st["bias"] is None else out + st["bias"].double()
    B, S, H, d, rot = case["B"], case["S"], case["H"], case["d"], case["rot"]
    if st["positions"] is None:
        at = (case["first"] + torch.arange(S, device="cuda")).view(1, S, 1)
    else:
        at = st["positions"].view(-1, S, case["axes"])
    freqs = torch.tensor(st["freqs"], device="cuda", dtype=torch.float64).split(_axis_pairs(case))
    angle = torch.cat([at[:, :, i:i + 1].double() * f for i, f in enumerate(freqs)], dim=-1).unsqueeze(2)
    turn = torch.polar(torch.ones_like(angle), angle)   # a pair is a complex number

    def pairs(x):
        p = x[..., :rot]
        return torch.complex(p[..., :rot // 2].contiguous(), p[..., rot // 2:].contiguous()) if case["layout"] == "half" else torch.view_as_complex(p.reshape(*p.shape[:-1], -1, 2))

    def columns(z, x):
        out = x.clone()
        out[..., :rot] = torch.cat([z.real, z.imag], dim=-1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
        return out

    x = st["x"].double()
    length = torch.linalg.vector_norm(x, dim=-1, keepdim=True) / math.sqrt(d)
    if op == "rope":
        x = x / length if case["unit_rms"] else x.contiguous()
        return (columns(pairs(x) * turn, x) * st["premul"]).permute(0, 2, 1, 3)
    dy = st["dy"].double().permute(0, 2, 1, 3).contiguous()
    g = columns(pairs(dy) * turn.conj(), dy) * st["premul"]
    if case["unit_rms"]:
        u = x / length
        g = (g - u * torch.sum(u * g, dim=-1, keepdim=True) / d) / length
    return g


def work(case):
    """Each input read once, each output written once."""
    op = case["op"]
    if op in ("rms_fwd", "rms_bwd"):
        rows, D = case["rows"], case["D"]
        n, params = rows * D, case["groups"] * D * 4
        if op == "rms_fwd":
            y = rows * (_up(D, 128) + _up(D, 128) // 128) if case["y"] == "e4m3" else n * SIZE[case["y"]]
            return {"bytes": n * (SIZE[case["x"]] + 2 * SIZE[case["res"]]) + y + rows * 4 + params, "flops": 6 * n}
        return {"bytes": n * (SIZE[case["dy"]] + SIZE[case["h"]] * (3 if case["dres"] else 2)) + rows * 4 + 2 * params, "flops": 12 * n}
    if op == "quant":
        rows, cols = case["rows"], case["cols"]
        out = (rows * _up(cols, 128) if case["order"] != "cols" else 0) + (cols * _up(rows, 128) if case["order"] != "rows" else 0)
        return {"bytes": rows * cols * SIZE[case["x"]] + out + out // 128, "flops": 3 * rows * cols}
    if op == "matmul":
        M, N, K = case["M"], case["N"], _up(case["K"], 128)
        return {"bytes": (M + N) * K + M * K // 128 + N * K // 128 // case["block"] + M * N * 2 + (4 * N if case["bias"] else 0),
                "flops": 2.0 * M * N * case["K"]}
    n = case["B"] * case["S"] * case["H"] * case["d"]
    reads = SIZE[case["x"]] if op == "rope" or case["unit_rms"] else 0
    return {"bytes": n * (2 + reads + (SIZE[case["x"]] if op == "rope_bwd" else 0)) + case["S"] * case["axes"] * 4, "flops": n * (12 if case["unit_rms"] else 4)}
