"""Cases of the operators for a model's matrices: 8-bit products with block scales, and losses over a large vocabulary.

A model's weight matrix is what the randomized SVD compresses; these operators are what stands next to the factors: the
remainder kept in 8 bits and multiplied, and the losses that say what a compressed output matrix costs and repair it.
The kinds:
  quant    a matrix cast into e4m3 with a power-of-two scale for each block, and back (brsvd_quantize_e4m3, _dequantize_e4m3)
  linear   activations times 8-bit weights: the activations cast by rows of 128, the product (brsvd_linear_e4m3)
  step     the three products of a linear layer's training step, every operand cast (brsvd_quantize_e4m3, brsvd_gemm_e4m3)
  xent     softmax cross entropy of H W^T over the vocabulary without keeping the logits; with train, the gradients too
  distill  Kullback-Leibler divergence from a teacher's top logits, tau^2 KL(q || p); with train, the gradients too
run() makes one call of a user's program where `own` is true, else the same in elementary torch operations in 32 bits.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # the square in-core matrix put away in 8 bits, blocks of 128 x 128, and the values that it then stands for
        dict(name="quant 20000x20000 f32", kind="quant", rows=20000, cols=20000, dtype="f32", block=128),
        # activations of odd sizes, a scale for each 128 of a row
        dict(name="quant 1999x2783 bf16", kind="quant", rows=1999, cols=2783, dtype="bf16", block=1),
        # serving: one token through a square layer, where latency and the read of the weights count
        dict(name="linear 1x4096x4096", kind="linear", m=1, n=4096, k=4096, dtype="bf16"),
        # serving: a small batch through a wide layer with a ragged last block of columns
        dict(name="linear 24x20000x5000", kind="linear", m=24, n=20000, k=5000, dtype="bf16"),
        # a prompt through a large layer: bound by the matrix cores
        dict(name="linear 8192x8192x8192", kind="linear", m=8192, n=8192, k=8192, dtype="bf16"),
        # a training step of one layer at odd sizes
        dict(name="step 4001x4096x6000", kind="step", m=4001, n=4096, k=6000, dtype="bf16"),
        # scoring a short answer with a small vocabulary
        dict(name="xent 7x32000x1000", kind="xent", t=7, v=32000, d=1000, dtype="bf16", train=False, mean=False),
        # scoring with a factored output matrix: dim is the sketch width of the tall in-core configuration
        dict(name="xent 4096x100000x272", kind="xent", t=4096, v=100000, d=272, dtype="f16", train=False, mean=False),
        # a small training step of odd sizes, a gradient for each token
        dict(name="xent train 999x50001x1000", kind="xent", t=999, v=50001, d=1000, dtype="f16", train=True, mean=False),
        # a training step at full width, the largest call
        dict(name="xent train 8192x100000x4096", kind="xent", t=8192, v=100000, d=4096, dtype="bf16", train=True, mean=True),
        # a few tokens against stored top logits
        dict(name="distill 130x32000x2000 k20", kind="distill", t=130, v=32000, d=2000, top=20, tau=1.0, dtype="bf16", train=False, mean=False),
        # distillation of a compressed model, with gradients
        dict(name="distill train 4096x65536x2048 k64", kind="distill", t=4096, v=65536, d=2048, top=64, tau=2.0, dtype="bf16", train=True, mean=True),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n if rng.random() < 0.5 else max(lo, n // 8 * 8)     # widths are multiples of eight in most models, lengths are not


def draw(rng):
    kind = rng.choice(["quant", "linear", "linear", "step", "xent", "xent", "distill"])
    while True:
        if kind == "quant":
            c = dict(kind=kind, rows=_log(rng, 1, 40000), cols=_log(rng, 64, 40000), dtype=rng.choice(["bf16", "f16", "f32"]), block=rng.choice([1, 128]))
            ok = 1e4 <= c["rows"] * c["cols"] <= 4e8
        elif kind == "linear":
            c = dict(kind=kind, m=_log(rng, 1, 8192), n=_log(rng, 64, 30000), k=_log(rng, 100, 16000), dtype=rng.choice(["bf16", "f16", "f32"]))
            ok = c["n"] * c["k"] <= 2e8
        elif kind == "step":
            c = dict(kind=kind, m=_log(rng, 64, 8192), n=_log(rng, 100, 16000), k=_log(rng, 100, 16000), dtype="bf16")
            ok = c["n"] * c["k"] <= 1e8
        else:
            c = dict(kind=kind, t=_log(rng, 1, 8192), v=_log(rng, 1000, 131072), d=_log(rng, 16, 4096), dtype=rng.choice(["bf16", "bf16", "f16"]),
                     train=rng.random() < 0.6, mean=rng.random() < 0.5)
            if kind == "distill":
                c["top"], c["tau"] = rng.choice([8, 20, 50, 64, 128]), rng.choice([1.0, 2.0, 4.0])
            ok = c["v"] * c["d"] <= 4.1e8
        if ok and 1e6 <= work(c)["flops"] + work(c)["bytes"] and work(c)["flops"] <= work(listed()[9])["flops"]:
            return c


def _gaussian(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV)


def _exponents(x, block):
    """Of each block of x (fp32): the least e >= -126 for which no finite number in it exceeds 448 times 2^e, 0 where all are zero."""
    r, c = x.shape
    padded = torch.zeros(-(-r // block) * block, -(-c // 128) * 128, device=x.device)
    padded[:r, :c] = torch.where(torch.isfinite(x), x.abs(), 0.0)
    top = padded.view(-1, block, padded.shape[1] // 128, 128).amax(dim=(1, 3))
    m, e = torch.frexp(top)                                   # top = m 2^e with m in [1/2, 1), 448 = 7/8 2^9
    return torch.where(top > 0, (e - 9 + (m > 0.875).int()).clamp(min=-126), 0)


def _powers(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _spread(s, block, r, c):
    """A number for each block as one for each entry."""
    return s.repeat_interleave(block, 0)[:r].repeat_interleave(128, 1)[:, :c]


def _cast(x, block):
    """x (fp32) as (e4m3 numbers in rows of whole 16 bytes, scales)."""
    r, c = x.shape
    e = _exponents(x, block)
    q = torch.zeros(r, -(-c // 16) * 16, dtype=torch.float8_e4m3fn, device=x.device)[:, :c]
    q.copy_((x * _spread(_powers(-e), block, r, c)).to(torch.float8_e4m3fn))
    return q, _powers(e)


def _value(q, s, block):
    return q.float() * _spread(s, block, *q.shape)


def _activations(seed, m, k, dtype):
    """Activations: a few channels are an order of magnitude above the others, as behind a model's norms."""
    x = _gaussian(seed, m, k)
    x[:, 7::211] *= 12.0
    return x.to(TYPES[dtype])


def _weights(seed, n, k):
    """A weight matrix with a spectrum that falls off and noise, entries around 1/sqrt(k)."""
    r = max(1, min(64, n, k))
    left, right = _gaussian(seed, n, r), _gaussian(seed + 1, r, k)
    decay = torch.arange(1, r + 1, device=DEV).float().pow(-0.5)
    return ((left * decay) @ right * 0.5 + _gaussian(seed + 2, n, k)) / math.sqrt(k)


def _head(c, seed):
    """Hidden states and an output matrix whose logits single out a few words, and each token's word."""
    w = _weights(seed, c["v"], c["d"])
    w = w / w.pow(2).mean().sqrt() / math.sqrt(c["d"]) * 1.5
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 5)
    y = torch.randint(0, c["v"], (c["t"],), generator=g, device=DEV)
    h = _gaussian(seed + 6, c["t"], c["d"]) + 1.5 * w[y]
    return h.to(TYPES[c["dtype"]]), w.to(TYPES[c["dtype"]]), y


def prepare(case, seed):
    c, seed = case, 100 * seed
    if c["kind"] == "quant":
        x = _weights(seed, c["rows"], c["cols"]) if c["block"] == 128 else _activations(seed, c["rows"], c["cols"], "f32")
        return dict(c=c, x=x.to(TYPES[c["dtype"]]))
    if c["kind"] == "linear":
        w, s = _cast(_weights(seed + 3, c["n"], c["k"]), 128)
        return dict(c=c, x=_activations(seed, c["m"], c["k"], c["dtype"]), w=w, s=s)
    if c["kind"] == "step":
        dy = _gaussian(seed + 9, c["m"], c["n"]) * 1e-3
        return dict(c=c, x=_activations(seed, c["m"], c["k"], c["dtype"]), w=_weights(seed + 3, c["n"], c["k"]).to(TYPES[c["dtype"]]), dy=dy.to(TYPES[c["dtype"]]))
    h, w, y = _head(c, seed)
    t = c["t"]
    # the gradient of a mean is one number for all tokens, else each token has a weight of its own; in fp16 the loss is scaled
    scale = (4096.0 if c["dtype"] == "f16" else 1.0) / t
    each = 0.5 + torch.rand(t, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed + 8))
    g = torch.full((1,), scale, device=DEV).expand(t) if c["mean"] else each * scale
    state = dict(c=c, h=h, w=w, g=g)
    if c["kind"] == "xent":
        y[3::29] = -1                                          # prompt and padding, which do not count
        state["y"] = y
    else:
        teacher = [((a.float() + 0.3 * _gaussian(seed + 20 + i, *a.shape)).to(h.dtype) @ w.t()).topk(c["top"]) for i, a in enumerate(h.split(1024))]
        state["logits"] = torch.cat([v.float() for v, _ in teacher])
        state["ids"] = torch.cat([i for _, i in teacher])
        state["logits"][5::31, c["top"] // 2:] = -math.inf      # fewer stored for some tokens
        state["ids"][6::37] = -1                               # and none for others
    return state


def run(state):
    c = state["c"]
    return _OWN[c["kind"]](state, c) if own else _PLAIN[c["kind"]](state, c)


# ---- the framework's entry points ---------------------------------------------------------------------------------


def _own_quant(s, c):
    import paper_1706_07191_amd as B
    q, scales = B.brsvd_quantize_e4m3(s["x"], block_rows=c["block"])
    return B.brsvd_dequantize_e4m3(q, scales, block_rows=c["block"]), scales


def _own_linear(s, c):
    import paper_1706_07191_amd as B
    return B.brsvd_linear_e4m3(s["x"], s["w"], s["s"])


def _own_step(s, c):
    import paper_1706_07191_amd as B
    x, sx, xt, sxt = B.brsvd_quantize_e4m3(s["x"], transpose=True)
    g, sg, gt, sgt = B.brsvd_quantize_e4m3(s["dy"], transpose=True)
    w, sw, wt, swt = B.brsvd_quantize_e4m3(s["w"], block_rows=128, transpose=True)
    y = B.brsvd_gemm_e4m3(x, sx, w, sw, dtype=s["x"].dtype)
    dx = B.brsvd_gemm_e4m3(g, sg, wt, swt, dtype=s["x"].dtype)
    dw = B.brsvd_gemm_e4m3(gt, sgt, xt, sxt, block_rows=1, dtype=s["x"].dtype)
    return dict(y=y, dx=dx, dw=dw)


def _own_xent(s, c):
    import paper_1706_07191_amd as B
    loss, lse = B.brsvd_xent_forward(s["h"], s["w"], s["y"])
    if not c["train"]:
        return dict(loss=loss, lse=lse)
    dh, dw = B.brsvd_xent_backward(s["h"], s["w"], s["y"], lse, s["g"])
    return dict(loss=loss, lse=lse, dh=dh, dw=dw)


def _own_distill(s, c):
    import paper_1706_07191_amd as B
    loss, lse, z = B.brsvd_distill_forward(s["h"], s["w"], s["ids"], s["logits"], c["tau"])
    if not c["train"]:
        return dict(loss=loss, lse=lse)
    dh, dw = B.brsvd_distill_backward(s["h"], s["w"], s["ids"], s["logits"], c["tau"], lse, z, s["g"])
    return dict(loss=loss, lse=lse, dh=dh, dw=dw)


_OWN = dict(quant=_own_quant, linear=_own_linear, step=_own_step, xent=_own_xent, distill=_own_distill)


# ---- the plain form: elementary operations in 32 bits -------------------------------------------------------------


def _plain_quant(s, c):
    q, scales = _cast(s["x"].float(), c["block"])
    return _value(q, scales, c["block"]), scales


def _plain_linear(s, c):
    x = _value(*_cast(s["x"].float(), 1), 1)
    return (x @ _value(s["w"], s["s"], 128).t()).to(s["x"].dtype)


def _plain_step(s, c):
    x, xt = (_value(*_cast(a, 1), 1) for a in (s["x"].float(), s["x"].float().t()))
    g, gt = (_value(*_cast(a, 1), 1) for a in (s["dy"].float(), s["dy"].float().t()))
    w = _value(*_cast(s["w"].float(), 128), 128)
    dt = s["x"].dtype
    return dict(y=(x @ w.t()).to(dt), dx=(g @ w).to(dt), dw=(gt @ xt.t()).to(dt))


def _lse(z):
    top = z.amax(dim=1)
    return top + (z - top[:, None]).exp_().sum(dim=1).log()


def _gradients(s, g):
    """(dH, dW) for the gradient g with respect to the logits."""
    return (g @ s["w"].float()).to(s["h"].dtype), (g.t() @ s["h"].float()).to(s["w"].dtype)


def _plain_xent(s, c):
    y, h, w = s["y"], s["h"].float(), s["w"].float()
    z = h @ w.t()
    lse = _lse(z)
    counted = (y >= 0) & (y < c["v"])
    word = y.clamp(0, c["v"] - 1)[:, None]
    loss = torch.where(counted, lse - z.gather(1, word)[:, 0], 0.0)
    if not c["train"]:
        return dict(loss=loss, lse=lse)
    p = z.sub_(lse[:, None]).exp_()
    p.scatter_add_(1, word, torch.full_like(word, -1, dtype=torch.float32))
    p.mul_(torch.where(counted, s["g"], 0.0)[:, None])
    dh, dw = _gradients(s, p)
    return dict(loss=loss, lse=lse, dh=dh, dw=dw)


def _plain_distill(s, c):
    ids, tau, h, w = s["ids"], c["tau"], s["h"].float(), s["w"].float()
    z = (h @ w.t()).div_(tau)
    lse = _lse(z)
    listed_ = (ids >= 0) & (ids < c["v"]) & (s["logits"] > -math.inf)
    some = listed_.any(dim=1)
    a = torch.where(listed_, s["logits"], -math.inf) / tau
    a = torch.where(some[:, None], a, 0.0)
    logq = a - _lse(a)[:, None]
    q = torch.where(listed_, logq.exp(), 0.0)
    word = ids.clamp(0, c["v"] - 1)
    part = torch.where(listed_, q * (logq - z.gather(1, word) + lse[:, None]), 0.0)
    loss = part.sum(dim=1) * tau * tau
    if not c["train"]:
        return dict(loss=loss, lse=lse)
    p = z.sub_(lse[:, None]).exp_()
    p.scatter_add_(1, word, -q)
    p.mul_(torch.where(some, s["g"] * tau, 0.0)[:, None])
    dh, dw = _gradients(s, p)
    return dict(loss=loss, lse=lse, dh=dh, dw=dw)


_PLAIN = dict(quant=_plain_quant, linear=_plain_linear, step=_plain_step, xent=_plain_xent, distill=_plain_distill)


# ---- 64 bits, from the definitions --------------------------------------------------------------------------------


def _rounded(x, block):
    """What x (fp64) stands for in e4m3 with a power-of-two scale for each block: three bits behind the leading one, no
    step finer than 2^-9 times the scale, the scale the least power of two for which the block fits into +-448.  And the scales."""
    r, c = x.shape
    out, scales = torch.empty_like(x), torch.empty(-(-r // block), -(-c // 128), dtype=torch.float64, device=x.device)
    for j in range(scales.shape[1]):
        part = x[:, 128 * j:128 * (j + 1)]
        top = part.abs().amax(dim=1)
        if block > 1:
            top = torch.cat([top, top.new_zeros(scales.shape[0] * block - r)]).view(-1, block).amax(dim=1)
        scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-126)), 1.0)
        scale = torch.where(scale * 448 < top, 2 * scale, torch.where((scale * 224 >= top) & (top > 0) & (scale > 2.0 ** -126), scale / 2, scale))
        scales[:, j] = scale
        u = part / scale.repeat_interleave(block)[:r, None]
        exponent = torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
        step = torch.exp2(exponent - 3)
        out[:, 128 * j:128 * (j + 1)] = torch.round(u / step) * step * scale.repeat_interleave(block)[:r, None]
    return out, scales


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "quant":
        return _rounded(s["x"].double(), c["block"])
    if c["kind"] == "linear":
        x = _rounded(s["x"].double(), 1)[0]
        n, k = c["n"], c["k"]
        y = torch.empty(c["m"], n, dtype=torch.float64, device=DEV)
        for i in range(0, n, 128):
            factor = s["s"][i // 128].double().repeat_interleave(128)[:k]
            y[:, i:i + 128] = x @ (s["w"][i:i + 128].double() * factor).t()
        return y
    if c["kind"] == "step":
        x, xt = _rounded(s["x"].double(), 1)[0], _rounded(s["x"].double().t().contiguous(), 1)[0]
        g, gt = _rounded(s["dy"].double(), 1)[0], _rounded(s["dy"].double().t().contiguous(), 1)[0]
        w = _rounded(s["w"].double(), 128)[0]
        return dict(y=x @ w.t(), dx=g @ w, dw=gt @ xt.t())
    h, w, v, tau = s["h"].double(), s["w"].double(), c["v"], c.get("tau", 1.0)
    loss, lse, dh = [], [], []
    dw = torch.zeros_like(w) if c["train"] else None
    for i in range(0, c["t"], 1024):
        z = (h[i:i + 1024] @ w.t()) / tau
        norm = torch.logsumexp(z, dim=1)
        target, own_part = torch.zeros_like(z), torch.zeros_like(norm)
        if c["kind"] == "xent":
            rows = torch.nonzero((s["y"][i:i + 1024] >= 0) & (s["y"][i:i + 1024] < v))[:, 0]
            target[rows, s["y"][i:i + 1024][rows]] = 1.0
        else:
            ids, a = s["ids"][i:i + 1024], s["logits"][i:i + 1024].double() / tau
            a = a.masked_fill((ids < 0) | (ids >= v), -math.inf)
            q = torch.softmax(a, dim=1).nan_to_num(0.0)
            target.scatter_add_(1, ids.clamp(0, v - 1), q)
            own_part = torch.xlogy(q, q).sum(dim=1)
        mass = target.sum(dim=1)
        loss.append(tau * tau * (own_part + norm * mass - (target * z.nan_to_num(0.0)).sum(dim=1)))
        lse.append(norm)
        if c["train"]:
            grad = (torch.exp(z - norm[:, None]) * mass[:, None] - target) * (tau * s["g"][i:i + 1024].double())[:, None]
            dh.append(grad @ w)
            dw += grad.t().contiguous() @ h[i:i + 1024]
    got = dict(loss=torch.cat(loss), lse=torch.cat(lse))
    return dict(got, dh=torch.cat(dh), dw=dw) if c["train"] else got


def work(case):
    c = case
    size = {"f32": 4}.get(c["dtype"], 2)
    if c["kind"] == "quant":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (size + 1 + 1 + 4), "flops": 2 * n}         # read, 8 bits written and read again, the values
    if c["kind"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": size * m * (k + n) + n * k + n * k // 4096, "flops": 2 * m * n * k}
    if c["kind"] == "step":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": 2 * size * (m * k + n * k + m * n), "flops": 6 * m * n * k}
    t, v, d = c["t"], c["v"], c["d"]
    stored = 12 * t * c.get("top", 1) + 8 * t
    return {"bytes": size * (t + v) * d * (2 if c["train"] else 1) + stored, "flops": 2 * t * v * d * (3 if c["train"] else 1)}
