"""The operators on 8-bit rows whose speed is followed: their calls, and the same in plain torch.

  rows    fp32 / bf16 rows -> 8-bit rows: e4m3 codes and a power of two for every 128 values of a row
  norm    the residual's addition and RMSNorm, the result as 8-bit rows (the input of q/k/v and gate/up)
  matmul  the product of 8-bit rows with 8-bit weights (q/k/v, o, down)
  gated   silu(x Wg^T) * (x Wu^T) of 8-bit rows and weights, the result as 8-bit rows (the input of down)

An 8-bit row of k values is kp codes, kp = k rounded up to 128s (zeros behind k), and one byte b per 128
codes, which stand for code * 2^(b - 127); the bytes are padded to a multiple of four with 127.  The power
is the smallest one for which no magnitude of the block passes 448, e4m3's largest.  Codes and bytes are
returned as float8_e4m3fn and float8_e8m0fnu, torch's types for such values.

Widths are those of the repository's two backbones and generic odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
EPS = 1e-6
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # batch of 32 speakers, one step: the attention output on its way into the o projection (latency)
        dict(name="rows_step_32", op="rows", m=32, k=3584, dtype="fp32"),
        # a long prompt's activations of a bf16 program, ragged
        dict(name="rows_bf16_8191", op="rows", m=8191, k=4096, dtype="bf16"),
        # one speaker, one step: the smallest call of all
        dict(name="norm_step_1", op="norm", m=1, k=3584, dtype="fp32", ytype="fp32"),
        # one pass of a prompt on the other backbone
        dict(name="norm_glm_1023", op="norm", m=1023, k=4096, dtype="fp32", ytype="fp32"),
        # a bf16 residual stream of odd width, a long batch of prompts
        dict(name="norm_bf16_odd_4099", op="norm", m=4099, k=2500, dtype="bf16", ytype="bf16"),
        # q/k/v of one speaker: weights once through the chip
        dict(name="matmul_step_qkv_1", op="matmul", m=1, n=4608, k=3584, out="fp32"),
        # down of a batch of 32: few outputs, long sums
        dict(name="matmul_step_down_32", op="matmul", m=32, n=3584, k=18944, out="fp32"),
        # odd everything
        dict(name="matmul_odd_77", op="matmul", m=77, n=1001, k=1000, out="bf16"),
        # down of one prompt pass
        dict(name="matmul_glm_down_1023", op="matmul", m=1023, n=4096, k=13696, out="fp32"),
        # gate/up of one speaker: the largest stream of a decoding step
        dict(name="gated_step_1", op="gated", m=1, n=18944, k=3584),
        # gate/up of a batch of 24
        dict(name="gated_glm_24", op="gated", m=24, n=13696, k=4096),
        # gate/up of a long prompt: matrix instructions
        dict(name="gated_glm_2048", op="gated", m=2048, n=13696, k=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rows", "norm", "matmul", "gated"])
    if op in ("rows", "norm"):
        k = rng.choice([3584, 4096, 13696, 18944, _log_int(rng, 64, 16000), 8 * _log_int(rng, 16, 2000)])
        m = _log_int(rng, 1, 8191 * 4096 // max(k, 4096))
        case = dict(op=op, m=m, k=k, dtype=rng.choice(["fp32", "bf16"]))
        if op == "norm":
            case["ytype"] = rng.choice(["fp32", "bf16"])
        return case
    m = _log_int(rng, 1, 2048)
    if op == "matmul":
        n, k = rng.choice([(4608, 3584), (3584, 3584), (3584, 18944), (4608, 4096), (4096, 4096), (4096, 13696),
                           (_log_int(rng, 16, 8192), _log_int(rng, 64, 8192))])
        return dict(op=op, m=m, n=n, k=k, out=rng.choice(["fp32", "bf16"]))
    n, k = rng.choice([(18944, 3584), (13696, 4096), (_log_int(rng, 64, 12000), _log_int(rng, 64, 4096))])
    return dict(op=op, m=min(m, 2048 * 13696 * 4096 // (n * k)), n=n, k=k)


# ---------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    """the operator's inputs as numbers, before anything is held in 8 bits"""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * std

    op, m, k = case["op"], case["m"], case["k"]
    out = {}
    if op in ("rows", "norm"):
        # activations: a few channels are many times the others, rows differ in size
        x = normal(m, k) * torch.exp(normal(m, 1)) * (1 + 30 * (torch.rand(k, generator=gen, device="cuda") < 0.004))
        out["x"] = x.to(DTYPES[case["dtype"]])
        if op == "norm":
            out["y"] = normal(m, k).to(DTYPES[case["ytype"]])
            out["gain"] = 1 + 0.1 * normal(k)
        return out
    out["x"] = normal(m, k) * (1 + 10 * (torch.rand(k, generator=gen, device="cuda") < 0.004))
    out["w"] = normal(case["n"], k, std=0.02).bfloat16()
    if op == "gated":
        out["up"] = normal(case["n"], k, std=0.02).bfloat16()
    return out


def prepare(case, seed):
    op, m, k = case["op"], case["m"], case["k"]
    v = _inputs(case, seed)
    state = {"op": op, "m": m, "k": k, "n": case.get("n")}
    if op in ("rows", "norm"):
        state.update(v)
        if op == "norm":
            state["h_out"] = torch.empty_like(v["x"])
        if own:
            from paper_2603_09215_amd import scaled
            state["rows"] = scaled.ScaledRows.empty(m, k, device="cuda")
        return state
    state["out_dtype"] = DTYPES[case["out"]] if op == "matmul" else None
    if own:   # the rows come from the operators above, the weights are laid out once
        from paper_2603_09215_amd import scaled
        state["rows"] = scaled.scaled_rows(v["x"])
        state["weights"] = scaled.ScaledWeights(v["w"], v.get("up"))
        if op == "matmul":
            state["out"] = torch.empty(m, case["n"], dtype=state["out_dtype"], device="cuda")
        else:
            state["out"] = scaled.ScaledRows.empty(m, case["n"], device="cuda")
    else:
        state["x8"] = _quantised(v["x"].double())
        state["w8"] = [_quantised(v[name].double()) for name in ("w", "up") if name in v]
    return state


# ---------------------------------------------------------------------------------- one pass

def run(state):
    op = state["op"]
    if own:
        from paper_2603_09215_amd import scaled
        if op == "rows":
            r = scaled.scaled_rows(state["x"], out=state["rows"])
            return {"codes": r.codes, "scales": r.scales}
        if op == "norm":
            r = scaled.scaled_norm(state["x"], state["gain"], EPS, y=state["y"], h_out=state["h_out"], out=state["rows"])
            return {"codes": r.codes, "scales": r.scales, "h": state["h_out"]}
        if op == "matmul":
            return {"out": scaled.scaled_matmul(state["rows"], state["weights"], out=state["out"])}
        r = scaled.scaled_gated(state["rows"], state["weights"], out=state["out"])
        return {"codes": r.codes, "scales": r.scales}
    if op == "rows":
        codes, scales = _quantised(state["x"].double())
        return {"codes": codes, "scales": scales}
    if op == "norm":
        # in 64 bits: a value next to a border between two codes falls on the side the definition says
        h = _to_type(state["x"].double() + state["y"].double(), state["x"].dtype)
        state["h_out"].copy_(h)
        v = h.double()
        v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * state["gain"].double()
        codes, scales = _quantised(v)
        return {"codes": codes, "scales": scales, "h": state["h_out"]}
    x = _values(*state["x8"])
    if op == "matmul":
        return {"out": (x @ _values(*state["w8"][0]).T).to(state["out_dtype"])}
    g, u = x @ _values(*state["w8"][0]).T, x @ _values(*state["w8"][1]).T
    codes, scales = _quantised((g / (1 + torch.exp(-g)) * u).double())
    return {"codes": codes, "scales": scales}


def _power(e, dtype=torch.float64):
    """2^e of whole numbers, from the format's exponent field: exact"""
    if dtype == torch.float32:
        return ((e + 127).to(torch.int32) << 23).view(torch.float32)
    return ((e + 1023).to(torch.int64) << 52).view(torch.float64)


def _to_grid(v, bits, lowest):
    """64-bit values to `bits` significant ones, half to even; below 2^lowest in steps of its last bit"""
    _, e = torch.frexp(v)
    last = torch.clamp(e - 1, min=lowest) - (bits - 1)
    return torch.round(v * _power(-last)) * _power(last)


def _to_type(v, dtype):
    return (_to_grid(v, 8, -126) if dtype == torch.bfloat16 else v).to(dtype)


def _quantised(v):
    """(codes [m][kp], scales [m][pitch]) of 64-bit values"""
    m, k = v.shape
    blocks = (k + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(v, (0, blocks * BLOCK - k)).view(m, blocks, BLOCK)
    f, x = torch.frexp(v.abs().amax(-1))   # largest = f 2^x, f in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(f > 0, torch.clamp(x - 9 + (f > 0.875).int(), min=-126), torch.zeros_like(x))
    codes = _to_grid(v * _power(-e).unsqueeze(-1), 4, -6)
    codes = codes.float().view(m, blocks * BLOCK).to(torch.float8_e4m3fn)
    scales = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -blocks % 4), value=127)
    return codes, scales.view(torch.float8_e8m0fnu)


def _values(codes, scales):
    m, kp = codes.shape
    e = scales.view(torch.uint8)[:, :kp // BLOCK].int() - 127
    return (codes.float().view(m, kp // BLOCK, BLOCK) * _power(e, torch.float32).unsqueeze(-1)).view(m, kp)


# ---------------------------------------------------------------------------------- what a pass needs

def work(case):
    op, m, k = case["op"], case["m"], case["k"]
    size = {"fp32": 4, "bf16": 2}
    rows = lambda count, width: count * width * (1 + 1 / BLOCK)   # noqa: E731
    if op == "rows":
        return {"bytes": m * k * size[case["dtype"]] + rows(m, k), "flops": 3.0 * m * k}
    if op == "norm":
        return {"bytes": m * k * (2 * size[case["dtype"]] + size[case["ytype"]]) + 4 * k + rows(m, k), "flops": 7.0 * m * k}
    n = case["n"]
    if op == "matmul":
        return {"bytes": rows(m, k) + rows(n, k) + m * n * size[case["out"]], "flops": 2.0 * m * n * k}
    return {"bytes": rows(m, k) + rows(2 * n, k) + rows(m, n), "flops": 4.0 * m * n * k}


# ---------------------------------------------------------------------------------- the definition in 64 bits

def _e4m3_table():
    """the magnitudes of codes 0 .. 126, in order"""
    return torch.tensor([(c % 8) * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)],
                        dtype=torch.float64, device="cuda")


def _powers():
    return torch.tensor([2.0 ** e for e in range(-126, 128)], dtype=torch.float64, device="cuda")


def _nearest(v):
    """each magnitude to the nearest code, the even one at the middle of two"""
    table = _e4m3_table()
    hi = torch.searchsorted(table, v.abs().contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    above, below = table[hi] - v.abs(), v.abs() - table[lo]
    pick = torch.where(above < below, hi, torch.where(below < above, lo, torch.where(hi % 2 == 0, hi, lo)))
    return torch.copysign(table[pick], v)


def _eight_bits(v, rounded=True):
    """64-bit values -> (codes as the numbers they are, padded; scales as powers of two, padded).  Not `rounded`:
    the numbers before they take the codes' type, as for an output in bf16"""
    m, k = v.shape
    codes, scales = [], []
    for c0 in range(0, k, BLOCK):
        part = v[:, c0:c0 + BLOCK]
        top = part.abs().max(dim=1, keepdim=True).values
        s = _powers()[torch.searchsorted(448 * _powers(), top)]   # the first that is large enough
        s = torch.where(top > 0, s, torch.ones_like(s))
        full = torch.zeros(m, BLOCK, dtype=torch.float64, device=v.device)
        full[:, :part.shape[1]] = _nearest(part / s) if rounded else part / s
        codes.append(full)
        scales.append(s)
    scales += [torch.ones_like(scales[0])] * (-len(scales) % 4)
    return torch.cat(codes, 1), torch.cat(scales, 1)


def exact(case, seed):
    op, k = case["op"], case["k"]
    v = _inputs(case, seed)
    if op == "rows":
        codes, scales = _eight_bits(v["x"].double())
        return {"codes": codes, "scales": scales}
    if op == "norm":
        total = v["x"].double() + v["y"].double()
        h = total.float().double()
        if case["dtype"] == "bf16":   # the stream holds 8 bits: the nearer of the two neighbours, the even one at the middle
            a = total.abs()
            unit = _powers()[torch.searchsorted(_powers(), a.clamp(min=2.0 ** -119), right=True) - 8]
            down = torch.floor(a / unit)
            rest = a / unit - down
            up = (rest > 0.5) | ((rest == 0.5) & (down % 2 == 1))
            h = torch.copysign((down + up) * unit, total)
        norm = h / torch.sqrt(h.square().sum(1, keepdim=True) / k + EPS) * v["gain"].double()
        codes, scales = _eight_bits(norm)
        return {"codes": codes, "scales": scales, "h": total}

    def held(t):
        c, s = _eight_bits(t.double())
        return (c.view(t.shape[0], -1, BLOCK) * s[:, :c.shape[1] // BLOCK, None]).view(t.shape[0], -1)

    x = held(v["x"])
    if op == "matmul":
        return {"out": torch.mm(x, held(v["w"]).t().contiguous())}
    g = torch.mm(x, held(v["w"]).t().contiguous())
    u = torch.mm(x, held(v["up"]).t().contiguous())
    # (sums in 32 bits decide which of two codes a value next to a border takes: any order of them is right)
    codes, scales = _eight_bits(g * torch.sigmoid(g) * u, rounded=False)
    return {"codes": codes, "scales": scales}
