"""Timed cases of the operators that serving a pruned encoder in 8 bits adds to the
library: quantising rows to 8-bit codes with a scale for each (alone, or behind the
residual's addition and a root-mean-square or layer norm), and the linear layer over
8-bit codes with a scale for each token and each output, dense or over the kept blocks.

``run`` computes a case in plain torch operations, or, with ``own`` set, through the
library's entry points; ``exact`` from the definitions in 64 bits.  Inputs are
synthetic, drawn on the GPU from the seed alone.  Codes are returned as the values
that they stand for.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
TOKENS = 197  # 224 x 224 image, 16 x 16 patches, plus the class token


# ---------------------------------------------------------------- the cases

def _rows(name, norm, M, D, dtype, residual):
    """norm: "rms", "layer" or "none" (the rows as they are); residual: x + y, whose sum is
    written too."""
    return {"name": name, "kind": "rows", "norm": norm, "M": M, "D": D, "dtype": dtype,
            "residual": residual}


def _linear(name, M, N, K, dtype, gelu=False, block=0, tall=0, sparsity=0):
    """block: 0 for a dense weight, else the width of the blocks of which `sparsity` percent
    are dropped, `tall` their height."""
    return {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "gelu": gelu,
            "b_r": tall or block, "b_c": block, "sparsity": sparsity}


def listed():
    return [
        # one token's residual stream into a wide layer: the smallest call, all latency
        _rows("norm_one", "rms", 1, 4096, "bf16", True),
        # the layer norm between two linear layers of the encoder, batch 64, fp16
        _rows("norm_encoder", "layer", 64 * TOKENS, 768, "f16", True),
        # long prompts of a wide model
        _rows("norm_wide", "rms", 8192, 4096, "bf16", True),
        # activations in fp32 before the second linear layer of an MLP, an odd number of rows
        _rows("rows_odd", "none", 1777, 5120, "f32", False),
        # single-token serving through a dense layer: the weight's bytes
        _linear("dense_one", 1, 4096, 4096, "bf16"),
        # the qkv layer of the encoder at batch 8
        _linear("dense_image", 8 * TOKENS, 2304, 768, "bf16"),
        # an odd number of tokens into fp32 outputs with the GELU
        _linear("dense_odd", 777, 5136, 1296, "f32", True),
        # long prompts of a wide model: the matrix cores
        _linear("dense_large", 16384, 8192, 4096, "bf16"),
        # one image through the pruned qkv layer: latency
        _linear("pruned_image", TOKENS, 2304, 768, "bf16", False, 32, 32, 50),
        # the smaller encoder's first MLP layer at batch 64 with the finest blocks
        _linear("pruned_gelu", 64 * TOKENS, 1536, 384, "f16", True, 16, 16, 75),
        # the qkv layer at batch 256, half of the blocks kept: the throughput workload
        _linear("pruned_batch", 256 * TOKENS, 2304, 768, "bf16", False, 32, 32, 50),
        # a long reduction over large blocks, few of them kept
        _linear("pruned_long", 8192, 4096, 4096, "f16", False, 64, 64, 80),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if rng.random() < 0.4:
        D = _spread(rng, 16, 16384)
        if rng.random() < 0.7:
            D = (D + 15) // 16 * 16
        return _rows(None, rng.choice(["rms", "rms", "layer", "none"]),
                     _spread(rng, 1, min(60000, 64000000 // (SIZE[dtype] * D))), D, dtype, rng.random() < 0.6)
    block = rng.choice([0, 0, 16, 32, 64])
    unit = block or 16
    tall = rng.choice([16, 32, 64]) if block else 0
    K = max(1, _spread(rng, 64, 8192) // unit) * unit
    N = max(1, _spread(rng, 64, 8192) // (tall or 16)) * (tall or 16)
    sparsity = rng.randint(30, 95) if block else 0
    # products and outputs bounded by the largest listed case
    most = min(60000, 500000000000 * 100 // ((100 - sparsity) * N * K), 260000000 // (SIZE[dtype] * N),
               65000000 // K)
    return _linear(None, _spread(rng, 1, max(1, most)), N, K, dtype, rng.random() < 0.3, block, tall,
                   sparsity)


# ---------------------------------------------------------------- inputs

def _codes(x):
    """8-bit codes of the rows of x, and their scales."""
    m = x.abs().amax(1, keepdim=True).clamp(min=1e-20)
    return torch.round(x * (127 / m)).to(torch.int8), (m / 127)[:, 0].contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[c["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    if c["kind"] == "rows":
        M, D = c["M"], c["D"]
        # activations: some channels are much larger than the others, and so are some rows
        x = normal(M, D) * torch.exp(normal(D)) * torch.exp(0.5 * normal(M, 1))
        s = {"case": c, "x": x.to(dt), "y": normal(M, D).to(dt) if c["residual"] else None}
        if c["norm"] != "none":
            s["gamma"] = (1 + 0.2 * normal(D)).to(dt)
        if c["norm"] == "layer":
            s["beta"] = (0.2 * normal(D)).to(dt)
        return s
    M, N, K = c["M"], c["N"], c["K"]
    x, xs = _codes(normal(M, K) * torch.exp(0.5 * normal(K)))
    w = normal(N, K) * 0.02
    mask = None
    if c["b_c"]:
        mask = torch.rand((N // c["b_r"], K // c["b_c"]), generator=g, device="cuda")
        mask = (mask * 100 >= c["sparsity"]).to(torch.uint8)
        w = w * mask.repeat_interleave(c["b_r"], 0).repeat_interleave(c["b_c"], 1)
    w, ws = _codes(w)
    s = {"case": c, "x": x, "xs": xs, "w": w, "ws": ws, "bias": (0.02 * normal(N)).to(dt)}
    if own:
        from paper_2407_02068_amd import lpv
        if mask is None:
            s["h"] = lpv.quant_pack(w, ws)
        else:
            s["h"] = lpv.quant_pack(w, ws, mask, c["b_r"], c["b_c"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    if own:
        return _own_rows(state) if state["case"]["kind"] == "rows" else _own_linear(state)
    return _plain_rows(state) if state["case"]["kind"] == "rows" else _plain_linear(state)


def _own_rows(s):
    from paper_2407_02068_amd import lpv
    norm, x, y = s["case"]["norm"], s["x"], s["y"]
    S = torch.empty_like(x) if y is not None else None
    if norm == "rms":
        q, scale = lpv.add_rmsnorm_quant(x, y, s["gamma"], EPS, S=S)
    elif norm == "layer":
        q, scale = lpv.add_layernorm_quant(x, y, s["gamma"], s["beta"], EPS, S=S)
    else:
        q, scale = lpv.quant_rows(x, y, S=S)
    return {"values": torch.mul(q, scale[:, None]), "scale": scale, "sum": S}


def _own_linear(s):
    from paper_2407_02068_amd import lpv
    return lpv.quant_linear(s["h"], s["x"], s["xs"], s["bias"], epi="gelu" if s["case"]["gelu"] else None)


def _plain_rows(s):
    # in 64 bits: a value next to the border of two codes takes one or the other
    norm, x, y = s["case"]["norm"], s["x"], s["y"]
    v = x.double()
    S = None
    if y is not None:
        v = v + y.double()
        S = v.to(x.dtype)
    r = 1.0
    if norm == "rms":  # (the norm's factor scales a row and leaves its codes)
        r = 1 / torch.sqrt((v * v).mean(1) + EPS)
        v = v * s["gamma"].double()
    elif norm == "layer":
        v = v - v.mean(1, keepdim=True)
        v = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
        v = v * s["gamma"].double() + s["beta"].double()
    m = v.abs().amax(1)
    q = torch.round(v * 127 / torch.where(m > 0, m, 1.0)[:, None])
    scale = (m * r / 127).float()
    return {"values": q.float() * scale[:, None], "scale": scale, "sum": S}


def _plain_linear(s):
    y = torch.matmul(s["x"].float(), s["w"].float().t())
    y = y * s["xs"][:, None] * s["ws"] + s["bias"].float()
    if s["case"]["gelu"]:
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["bias"].dtype)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rows(s) if case["kind"] == "rows" else _exact_linear(s)


def _exact_rows(s):
    norm, x = s["case"]["norm"], s["x"].to(torch.float64)
    total = x if s["y"] is None else torch.add(x, s["y"])
    out, factor = total, torch.ones(len(x), dtype=torch.float64, device=x.device)
    if norm == "rms":
        factor = torch.rsqrt(total.pow(2).sum(1) / total.shape[1] + EPS)
        out = total * s["gamma"]
    elif norm == "layer":
        var, mean = torch.var_mean(total, 1, correction=0, keepdim=True)
        out = torch.addcmul(s["beta"].double(), (total - mean) / (var + EPS).sqrt(), s["gamma"].double())
    top = torch.linalg.vector_norm(out, math.inf, dim=1)
    a = 127 * out.abs() / top.clamp(min=1e-300)[:, None]
    low = a.floor()
    up = (a - low > 0.5) | ((a - low == 0.5) & (low % 2 == 1))
    scale = top * factor / 127
    values = torch.copysign(low + up, out) * scale[:, None]
    return {"values": values, "scale": scale, "sum": None if s["y"] is None else total}


def _exact_linear(s):
    # each token and output in the units of its scale, some tokens at a time
    w = s["w"].double() * s["ws"].double()[:, None]
    w = w.t().contiguous()
    outs = []
    for i in range(0, len(s["x"]), 4096):
        v = torch.addmm(s["bias"].double(), s["x"][i:i + 4096].double() * s["xs"][i:i + 4096, None].double(), w)
        if s["case"]["gelu"]:
            v = v * torch.special.ndtr(v)
        outs.append(v)
    return torch.cat(outs)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    es = SIZE[c["dtype"]]
    if c["kind"] == "rows":
        n = c["M"] * c["D"]
        params = {"none": 0, "rms": 1, "layer": 2}[c["norm"]] * c["D"] * es
        return {"bytes": n * es * (3 if c["residual"] else 1) + n + 4 * c["M"] + params,
                "flops": n * (10 if c["norm"] != "none" else 4)}
    kept = c["N"] * c["K"] * (100 - c["sparsity"]) // 100
    return {"bytes": c["M"] * c["K"] + kept + c["M"] * c["N"] * es + 4 * c["M"] + (4 + es) * c["N"],
            "flops": 2 * c["M"] * kept}
