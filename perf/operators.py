"""Timed cases of the operators that finetuning a pruned student model adds to the
library: attention with a learned relative position bias (forward, and a training pass
with its gradients) and the distillation loss from a teacher's top logits.

``run`` computes a case in plain torch operations, or, with ``own`` set, through the
library's entry points; ``exact`` from the definitions in 64 bits.  Inputs are
synthetic, drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- the cases

def _attention(name, step, grid, side, n_seq, H, hd, dtype, region="none", images=1):
    """grid: "window" (side x side tokens, one bucket per offset), "class" (the same plus
    a class token with three buckets of its own) or "line" (side tokens in a row, 32
    buckets of signed distance, exact near, logarithmic far).  region: "none", "shift"
    (the four cases of a window cut by a cyclic shift, `images` windows apart) or "pad"
    (the last tokens of a sequence are padding)."""
    return {"name": name, "kind": "attention", "step": step, "grid": grid, "side": side,
            "n_seq": n_seq, "H": H, "hd": hd, "dtype": dtype, "region": region,
            "n_region": images}


def _distill(name, step, M, V, k, dtype, temperature, ragged=False):
    return {"name": name, "kind": "distill", "step": step, "M": M, "V": V, "k": k,
            "dtype": dtype, "temperature": temperature, "ragged": ragged}


def listed():
    return [
        # the last stage of a windowed encoder on one image: one window of 7 x 7 tokens,
        # the smallest call, all latency
        _attention("window_one", False, "window", 7, 1, 24, 32, "f16"),
        # the first stage at batch 64: 56 x 56 tokens in 64 windows each, shifted
        _attention("window_shift", False, "window", 7, 4096, 3, 32, "bf16", "shift", 64),
        # a whole 224 x 224 image as one sequence (14 x 14 patches and a class token),
        # batch 64
        _attention("image", False, "class", 14, 64, 12, 64, "bf16"),
        # long sequences: 512 x 512 images, padded to a common length, batch 8
        _attention("image_long", False, "class", 32, 8, 12, 64, "f16", "pad", 8),
        # training, the first stage of the windowed encoder
        _attention("window_step", True, "window", 7, 4096, 3, 32, "bf16", "shift", 64),
        # training with larger windows in fp16: 16 images of 48 x 48 tokens, 16 windows each
        _attention("window12_step", True, "window", 12, 256, 6, 32, "f16", "shift", 16),
        # training on whole images, batch 64
        _attention("image_step", True, "class", 14, 64, 12, 64, "bf16"),
        # training on long rows of tokens of an odd length, distances in 32 buckets
        _attention("line_step", True, "line", 777, 4, 8, 64, "bf16"),
        # the loss of a micro-batch over 1000 classes in fp32, the smallest step
        _distill("classes_step", True, 64, 1000, 16, "f32", 2.0),
        # scoring a validation set: the loss alone, rows with fewer teacher logits
        _distill("classes_loss", False, 16384, 1000, 8, "f16", 1.0, True),
        # training over a large odd number of classes
        _distill("many_classes_step", True, 2048, 21841, 64, "bf16", 2.0, True),
        # few rows over a very wide vocabulary: the row has to be shared
        _distill("wide_few_step", True, 4, 131072, 128, "f32", 1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.35:
        step = rng.random() < 0.7
        V = _spread(rng, 10, 131072)
        M = _spread(rng, 1, min(30000, (44000000 if step else 88000000) // V))
        return _distill(None, step, M, V, _spread(rng, 1, min(256, V)),
                        rng.choice(["f32", "f16", "bf16"]), rng.choice([1.0, 2.0, 4.0]),
                        rng.random() < 0.5)
    step = rng.random() < 0.6
    grid = rng.choice(["window", "window", "class", "line"])
    side = _spread(rng, 1, 1000 if step else 1200) if grid == "line" else rng.randint(2, 28)
    T = _tokens({"grid": grid, "side": side})
    H, hd = rng.randint(1, 16), rng.choice([32, 64])
    # pairs and elements bounded by the largest listed cases
    pairs, elements = (19000000, 9000000) if step else (90000000, 18000000)
    most = max(1, min(pairs // (H * T * T), elements // (H * hd * T)))
    n_seq = _spread(rng, 1, most)
    region = rng.choice(["none", "none", "shift" if grid == "window" else "pad", "pad"])
    return _attention(None, step, grid, side, n_seq, H, hd, rng.choice(["f16", "bf16"]), region,
                      rng.randint(1, min(64, n_seq)))


def _tokens(c):
    return c["side"] if c["grid"] == "line" else c["side"] ** 2 + (c["grid"] == "class")


# ---------------------------------------------------------------- inputs

def _index(c):
    """The T x T bucket index (int64, on the CPU) and the number of buckets."""
    s = c["side"]
    i = torch.arange(s)
    if c["grid"] == "line":
        d = i[None, :] - i[:, None]
        a = d.abs()
        far = 8 + (torch.log(a.clamp(min=1).double() / 8) / math.log(128 / 8) * 8).long()
        return torch.where(a < 8, a, far.clamp(max=15)) + 16 * (d > 0), 32
    y, x = i.repeat_interleave(s), i.repeat(s)
    idx = (y[:, None] - y[None, :] + s - 1) * (2 * s - 1) + x[:, None] - x[None, :] + s - 1
    n = (2 * s - 1) ** 2
    if c["grid"] == "window":
        return idx, n
    full = torch.empty((s * s + 1, s * s + 1), dtype=torch.int64)
    full[1:, 1:] = idx
    full[0, :], full[:, 0], full[0, 0] = n, n + 1, n + 2
    return full, n + 3


def _region(c, T, g):
    """None, or n_region x T labels: tokens attend within their label, -1 is padding."""
    n = c["n_region"]
    if c["region"] == "none":
        return None
    r = torch.zeros((n, T), dtype=torch.int32, device="cuda")
    if c["region"] == "pad":
        used = torch.randint(max(1, T // 2), T + 1, (n, 1), generator=g, device="cuda")
        r[torch.arange(T, device="cuda")[None, :] >= used] = -1
        return r
    # windows of an image in rows of w: the last row and column of them hold two parts
    s, w = c["side"], max(1, math.isqrt(n))
    i = torch.arange(T, device="cuda")
    low, right = (i // s >= s - s // 2).int(), (i % s >= s - s // 2).int()
    k = torch.arange(n, device="cuda")[:, None]
    r += 2 * low[None, :] * (k >= n - w).int() + right[None, :] * (k % w == w - 1).int()
    return r


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[c["dtype"]]
    normal = lambda shape, std=1.0: torch.randn(shape, generator=g, device="cuda") * std
    if c["kind"] == "attention":
        T, H, hd = _tokens(c), c["H"], c["hd"]
        idx, n_buckets = _index(c)
        M = c["n_seq"] * T
        s = {"case": c, "T": T, "index": idx.to(torch.int32).cuda(),
             "table": normal((n_buckets, H), 0.5).to(dt),
             "qkv": normal((M, 3 * H * hd)).to(dt), "region": _region(c, T, g)}
        if c["step"]:
            s["dout"] = normal((M, H * hd)).to(dt)
        if own:
            from paper_2407_02068_amd import lpv
            s["relpos"] = lpv.relpos(s["index"], n_buckets)
        return s
    M, V, k = c["M"], c["V"], c["k"]
    # logits as a linear layer of the library writes them: rows padded to 16 outputs
    z = torch.zeros((M, (V + 15) // 16 * 16), dtype=dt, device="cuda")
    z[:, :V] = normal((M, V), 2.0)
    # distinct ids: one of each k-th of the classes, in random order
    at = torch.arange(k, device="cuda")
    lo, hi = at * V // k, (at + 1) * V // k
    ids = lo + (torch.rand((M, k), generator=g, device="cuda") * (hi - lo)).long().clamp(max=V)
    ids = torch.minimum(ids, hi - 1)
    ids = ids.gather(1, torch.rand((M, k), generator=g, device="cuda").argsort(1))
    t = torch.rand((M, k), generator=g, device="cuda").clamp(min=1e-6)
    t = 8 + (t.log() * 0.5).cumsum(1)  # falling from about 8
    if c["ragged"]:  # some rows have fewer, a few none
        n = torch.randint(0, k + 1, (M, 1), generator=g, device="cuda")
        ids = torch.where(torch.arange(k, device="cuda") < torch.maximum(n, n % 16), ids, -1)
    s = {"case": c, "logits": z[:, :V], "ids": ids.to(torch.int32), "teacher": t}
    if c["step"]:  # the mean over the rows, some of them weighted; fp16 with a loss scale
        w = torch.rand(M, generator=g, device="cuda") + 0.5
        s["dloss"] = w / M * (1024 if c["dtype"] == "f16" else 1)
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    if own:
        return _own_attention(state) if c["kind"] == "attention" else _own_distill(state)
    return _plain_attention(state) if c["kind"] == "attention" else _plain_distill(state)


def _own_attention(s):
    from paper_2407_02068_amd import lpv
    c = s["case"]
    n, H, hd = c["n_seq"], c["H"], c["hd"]
    if not c["step"]:
        return lpv.relpos_attention(s["relpos"], s["table"], s["qkv"], n, H, region=s["region"], hd=hd)
    lse = torch.empty((n, H, s["T"]), dtype=torch.float32, device="cuda")
    out = lpv.relpos_attention(s["relpos"], s["table"], s["qkv"], n, H, region=s["region"], lse=lse,
                               hd=hd)
    dqkv, dtable = lpv.relpos_attention_grad(s["relpos"], s["table"], s["qkv"], out, lse, s["dout"],
                                             n, H, region=s["region"], hd=hd)
    return {"out": out, "dqkv": dqkv, "dtable": dtable}


def _own_distill(s):
    from paper_2407_02068_amd import lpv
    c = s["case"]
    if not c["step"]:
        return lpv.distill_loss(s["logits"], s["ids"], s["teacher"], c["temperature"])
    loss, dlogits = lpv.distill_grad(s["logits"], s["ids"], s["teacher"], c["temperature"], s["dloss"])
    return {"loss": loss, "dlogits": dlogits}


def _allowed(region, n_seq):
    """n_seq x 1 x T x T truth values, or None."""
    if region is None:
        return None
    r = region[torch.arange(n_seq, device=region.device) % region.shape[0]]
    return ((r[:, :, None] == r[:, None, :]) & (r[:, :, None] >= 0))[:, None]


def _plain_attention(s):
    c = s["case"]
    n, T, H, hd, dt = c["n_seq"], s["T"], c["H"], c["hd"], s["qkv"].dtype
    q, k, v = s["qkv"].float().view(n, T, 3, H, hd).permute(2, 0, 3, 1, 4).contiguous()
    bias = s["table"].float()[s["index"].long()].permute(2, 0, 1)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd) + bias
    ok = _allowed(s["region"], n)
    if ok is not None:
        p = torch.where(ok, p, -math.inf)
    m = p.amax(3, keepdim=True)
    p = torch.exp(p - torch.where(m == -math.inf, 0.0, m))
    p = p / p.sum(3, keepdim=True).clamp(min=1e-30)
    rows = lambda x: x.permute(0, 2, 1, 3).reshape(n * T, H * hd)
    o = torch.matmul(p, v)
    out = rows(o).to(dt)
    if not c["step"]:
        return out
    do = s["dout"].float().view(n, T, H, hd).permute(0, 2, 1, 3).contiguous()
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (ds - (do * o).sum(3, keepdim=True))
    dq = torch.matmul(ds, k) / math.sqrt(hd)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) / math.sqrt(hd)
    # (many tables, summed at the end: a few buckets would otherwise take every addition)
    pairs = ds.sum(0, dtype=torch.float64).permute(1, 2, 0).reshape(T * T, H)
    n_buckets = s["table"].shape[0]
    tables = max(64, 131072 // n_buckets)
    at = s["index"].long().view(-1) + torch.arange(T * T, device="cuda") % tables * n_buckets
    dtable = torch.zeros((tables * n_buckets, H), dtype=torch.float64, device="cuda")
    dtable.index_add_(0, at, pairs)
    dtable = dtable.view(tables, n_buckets, H).sum(0)
    return {"out": out, "dqkv": torch.cat([rows(dq), rows(dk), rows(dv)], 1).to(dt),
            "dtable": dtable.to(dt)}


def _plain_distill(s):
    c = s["case"]
    t, ids = c["temperature"], s["ids"].long()
    z = s["logits"].float() / t
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    valid = ids >= 0
    some = valid.any(1)
    at = ids.clamp(min=0)
    tl = torch.where(valid, s["teacher"] / t, -math.inf)
    top = torch.where(some, tl.amax(1), 0.0)[:, None]
    q = torch.exp(tl - top)
    mass = q.sum(1, keepdim=True).clamp(min=1e-30)
    q = q / mass
    log_q = tl - top - torch.log(mass)
    log_p = z.gather(1, at) - m - torch.log(total)
    loss = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1) * (t * t)
    if not c["step"]:
        return loss
    d = e / total
    d.scatter_add_(1, at, -q)
    d = d * (s["dloss"] * t)[:, None]
    return {"loss": loss, "dlogits": torch.where(some[:, None], d, 0.0).to(s["logits"].dtype)}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attention(s) if case["kind"] == "attention" else _exact_distill(s)


def _exact_attention(s):
    # a few sequences at a time; the gradients come from torch's differentiation of the
    # definition in 64 bits
    c = s["case"]
    n, T, H, hd = c["n_seq"], s["T"], c["H"], c["hd"]
    table = s["table"].double().requires_grad_(c["step"])
    dtable = torch.zeros_like(table) if c["step"] else None
    outs, grads = [], []
    batch = max(1, 20000000 // (H * T * T))
    for a in range(0, n, batch):
        b = min(n, a + batch)
        x = s["qkv"][a * T:b * T].double().requires_grad_(c["step"])
        q, k, v = (x.view(b - a, T, 3, H, hd)[:, :, i].transpose(1, 2) for i in range(3))
        logits = q @ k.transpose(-1, -2) * hd ** -0.5
        logits = logits + table[s["index"].long()].movedim(2, 0)
        dead = None
        if s["region"] is not None:
            r = s["region"][torch.arange(a, b, device="cuda") % s["region"].shape[0]]
            stop = (r[:, :, None] != r[:, None, :]) | (r[:, :, None] < 0)
            dead = stop.all(2)[:, None, :, None]
            logits = logits.masked_fill(stop[:, None] & ~dead, -math.inf)
        w = torch.softmax(logits, -1)
        if dead is not None:
            w = w.masked_fill(dead, 0.0)
        o = (w @ v).transpose(1, 2).reshape((b - a) * T, H * hd)
        outs.append(o.detach())
        if c["step"]:
            gx, gt = torch.autograd.grad(o, (x, table), s["dout"][a * T:b * T].double())
            grads.append(gx)
            dtable += gt
    out = torch.cat(outs)
    return {"out": out, "dqkv": torch.cat(grads), "dtable": dtable} if c["step"] else out


def _exact_distill(s):
    c = s["case"]
    t, M = c["temperature"], c["M"]
    z = s["logits"].double().requires_grad_(c["step"])
    tl = s["teacher"].double() / t
    tl = tl.masked_fill(s["ids"] < 0, -1e300)
    some = (s["ids"] >= 0).any(1)
    q = torch.softmax(tl, 1).masked_fill(s["ids"] < 0, 0.0)
    log_p = torch.log_softmax(z / t, 1).gather(1, s["ids"].long().clamp(min=0))
    kl = (torch.special.xlogy(q, q) - q * log_p).sum(1) * t ** 2
    loss = torch.where(some, kl, torch.zeros(M, dtype=torch.float64, device="cuda"))
    if not c["step"]:
        return loss
    return {"loss": loss.detach(),
            "dlogits": torch.autograd.grad(loss, z, s["dloss"].double())[0]}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    es = SIZE[c["dtype"]]
    if c["kind"] == "attention":
        T, H, hd, n = _tokens(c), c["H"], c["hd"], c["n_seq"]
        unit = n * T * H * hd * es
        products = n * H * T * T * hd * 2
        buckets = _index({**c, "side": 1})[1] if c["grid"] == "line" else (2 * c["side"] - 1) ** 2
        small = T * T * 2 + buckets * H * es + (0 if c["region"] == "none" else 4 * c["n_region"] * T)
        if not c["step"]:
            return {"bytes": 4 * unit + small, "flops": 2 * products}
        # forward, then q, k, v and dout in, dqkv out; the scores again and four products
        return {"bytes": (4 + 7) * unit + 8 * n * H * T + 2 * small, "flops": (2 + 5) * products}
    rows = c["M"] * c["V"] * es
    return {"bytes": rows * (2 if c["step"] else 1) + 8 * c["M"] * c["k"] + 8 * c["M"],
            "flops": 5 * c["M"] * c["V"]}
