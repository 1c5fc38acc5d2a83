"""What the operators that answer for merged models, distil them and hold their layers in 4 bits
are measured on.

``log_probs`` reads answers off logits: log probability and rank of a given class, entropy and the
top alternatives (``Context.log_probs``). ``distill`` is the loss of a student against a teacher's
top logits and its gradient (``Context.distill_backward``). ``quantize`` brings a matrix into
blocks of 32 4-bit floating-point numbers with a shared power of two and back
(``Context.mx_quantize``, ``Context.mx_dequantize``), ``product`` is a projection with such weights
(``Context.mx_product``), its rows as they are or in 4 bits too. Sizes are those of the heads and FC
layers of the framework's own networks, and generic ones up to 200,000 classes.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
# magnitudes of the 4-bit codes 0..7; code 8 + c is the negative of c
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MOST_TOP = 64


# ---- cases -----------------------------------------------------------------

def _scores(name, op, dtype, rows, classes, top, temperature=1.0, masked=False):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "classes": classes, "top": top,
            "temperature": temperature, "masked": masked}


def _quantize(name, dtype, rows, cols):
    return {"name": name, "op": "quantize", "dtype": dtype, "rows": rows, "cols": cols}


def _product(name, dtype, acts, rows, n_in, n_out):
    return {"name": name, "op": "product", "dtype": dtype, "acts": acts, "rows": rows, "n_in": n_in, "n_out": n_out}


def listed():
    return [
        # the answer to one frame of an ImageNet head with its five best classes: latency alone counts
        _scores("log_probs one row", "log_probs", "f32", 1, 1000, 5),
        # scoring a stored backlog of frames of such a head, one class more than is even
        _scores("log_probs backlog", "log_probs", "bf16", 16384, 1001, 5),
        # a vocabulary-sized head, some of its classes never offered
        _scores("log_probs wide", "log_probs", "bf16", 2048, 100003, 20, masked=True),
        # a small joint retraining batch on the ImageNet head
        _scores("distill small head", "distill", "bf16", 131, 1000, 8, 2.0),
        # every cell and anchor of a detector's finest map, 80 classes each
        _scores("distill detector cells", "distill", "f32", 97344, 80, 10, 2.0),
        # retraining a vocabulary-sized head against many of its teacher's logits
        _scores("distill wide", "distill", "bf16", 4096, 65537, 64, 1.5, masked=True),
        # the features of a batch of frames on their way into a 4-bit product
        _quantize("quantize features", "bf16", 333, 2048),
        # VGG-16's first FC layer, the largest layer of the framework's networks
        _quantize("quantize vgg fc1", "f32", 4096, 25088),
        # one frame through VGG-16's second FC layer with 4-bit weights
        _product("product one row", "bf16", "float", 1, 4096, 4096),
        # odd frames of a few models through VGG-16's first FC layer, float32
        _product("product 37 rows f32", "f32", "float", 37, 25088, 4096),
        # frames of several models through a merged ResNet-50 head, both sides in 4 bits
        _product("product head", "bf16", "mx", 777, 2048, 1000),
        # a backlog through VGG-16's second FC layer, both sides in 4 bits
        _product("product backlog", "bf16", "mx", 16384, 4096, 4096),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["log_probs", "distill", "quantize", "product"])
    dtype = rng.choice(["bf16", "f32"])
    while True:
        if op in ("log_probs", "distill"):
            c = _scores("", op, dtype, _log(rng, 1, 100000), _log(rng, 2, 200000), _log(rng, 1, MOST_TOP),
                        rng.choice([1.0, 1.0, 0.7, 2.0, 4.0]), rng.random() < 0.3)
            c["top"] = min(c["top"], c["classes"])
            good = work(c)["bytes"] <= 4.2e8
        elif op == "quantize":
            c = _quantize("", dtype, _log(rng, 1, 65536), _log(rng, 16, 65536))
            good = work(c)["bytes"] <= 9.0e8
        else:
            c = _product("", dtype, rng.choice(["float", "mx"]), _log(rng, 1, 16384), _log(rng, 16, 25088),
                         _log(rng, 10, 4096))
            good = work(c)["flops"] <= (5.5e11 if c["acts"] == "mx" else 1.4e11)
        if good:
            del c["name"]
            return c


# ---- inputs ----------------------------------------------------------------

_contexts = {}


def _context(dtype):
    """One context per type, as a program keeps it."""
    if dtype not in _contexts:
        import paper_2201_07705_amd as P
        _contexts[dtype] = P.Context(0, dtype)
    return _contexts[dtype]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std

    s = dict(case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] in ("log_probs", "distill"):
        rows, classes, top = case["rows"], case["classes"], case["top"]
        # a broad floor with a few likely classes in every row
        z = normal(rows, classes, std=2.0)
        likely = torch.randint(classes, (rows, 4), device="cuda", generator=gen)
        z.scatter_add_(1, likely, 6.0 + normal(rows, 4, std=2.0))
        if case["op"] == "distill":
            # the teacher is of the student's mind, more or less; its last rows (padding) have no entry
            values, indices = torch.topk(z + normal(rows, classes, std=0.7), top, dim=1)
            if rows >= 16:
                indices[rows - rows // 16:] = -1
            s["indices"], s["values"] = indices.int(), values
            s["dloss"] = (0.5 + torch.rand(rows, device="cuda", generator=gen)) / rows
        else:
            s["labels"] = likely[:, 0].int()
            if rows >= 16:
                s["labels"][rows - rows // 16:] = -1
        if case["masked"]:
            # classes that are not offered, the teacher's choices aside
            z[:, torch.rand(classes, device="cuda", generator=gen) < 0.1] = -math.inf
            if case["op"] == "distill":
                keep = s["indices"].long().clamp_min(0)
                z.scatter_(1, keep, s["values"].float())
        s["logits"] = z.to(dtype)
    elif case["op"] == "quantize":
        # columns of different size, and a few large values, as in weights and features
        x = normal(case["rows"], case["cols"]) * torch.exp(normal(case["cols"]))
        s["x"] = (x * 0.02).to(dtype)
    else:
        m, k, n = case["rows"], case["n_in"], case["n_out"]
        s["x"] = torch.relu(normal(m, k) * torch.exp(normal(k, std=0.5))).to(dtype)
        s["bias"] = normal(n, std=0.1)
        w = normal(n, k, std=k ** -0.5).to(dtype)
        # the weights that a program keeps: 4-bit codes and a scale for each block
        if own:
            s["weight"] = _context(case["dtype"]).mx_quantize(w)
        else:
            s["codes"], s["scales"] = _encode(w.float())
    return s


# ---- one pass --------------------------------------------------------------

def _power(e):
    """2^e in float32 for whole e from -127 to 127, exactly (the pow of a device may be off in its last bit)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _encode(x):
    """[rows, cols] float32 as codes [rows, blocks, 32] and exponents [rows, blocks] (-128: not finite)."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    padded = torch.zeros(rows, blocks * BLOCK, device=x.device)
    padded[:, :cols] = x
    v = padded.view(rows, blocks, BLOCK)
    most = v.abs().amax(2)
    good = most < math.inf
    # the largest value comes into [4, 8)
    exponent = torch.frexp(torch.where(good, most, 0.0))[1] - 3
    exponent = torch.where(most > 0, exponent, -127).clamp(-127, 127)
    a = v * _power(-exponent)[:, :, None]
    code = torch.zeros(v.shape, dtype=torch.uint8, device=x.device)
    # to the nearest magnitude, from halfway between two to the even code
    size = a.abs()
    for i, (lo, hi) in enumerate(zip(MAGNITUDES, MAGNITUDES[1:])):
        half = (lo + hi) / 2
        code += size >= half if i % 2 else size > half
    code += (torch.signbit(a) * 8).to(torch.uint8)
    return code, torch.where(good, exponent, -128).to(torch.int8)


def _decode(codes, exponents, cols):
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    v = table[codes.int()]
    scale = torch.where(exponents == -128, math.nan, _power(exponents.int().clamp_min(-127)))
    return (v * scale[:, :, None]).view(codes.shape[0], -1)[:, :cols]


def _softmax_parts(z):
    """Largest value and logarithm of the sum of exponentials behind it, of each row."""
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    return m, e, e.sum(1, keepdim=True)


def _plain_log_probs(s):
    raw = s["logits"].float() + 0.0
    z = raw / s["temperature"]
    m, e, total = _softmax_parts(z)
    log_total = torch.log(total)
    d = torch.where(e > 0, z - m, 0.0)
    out = {"entropy": (log_total - (e * d).sum(1, keepdim=True) / total)[:, 0], "log_sum": (m + log_total)[:, 0]}
    # classes in the order of their logits, the lower index first among equals: as whole numbers
    classes = raw.shape[1]
    index = torch.arange(classes, device="cuda")
    bits = raw.view(torch.int32).long()
    bits = bits ^ ((bits >> 31) & 0x7fffffff)
    key = bits * (1 << 32) + (classes - 1 - index)
    best = torch.topk(key, s["top"], dim=1)[1]
    value = raw.gather(1, best)
    offered = value > -math.inf
    out["top_indices"] = torch.where(offered, best, -1).int()
    out["top_log_probs"] = (value / s["temperature"] - m) - log_total
    label = s["labels"].long()
    given = label >= 0
    at = label.clamp_min(0)[:, None]
    mine = raw.gather(1, at)
    before = (raw > mine).sum(1) + ((raw == mine) & (index < at)).sum(1)
    out["log_prob"] = torch.where(given, (mine / s["temperature"] - m - log_total)[:, 0], 0.0)
    out["rank"] = torch.where(given, before, -1).int()
    return out


def _plain_distill(s):
    t = s["temperature"]
    z = s["logits"].float() / t
    m, e, total = _softmax_parts(z)
    used = s["indices"] >= 0
    at = s["indices"].long().clamp_min(0)
    v = torch.where(used, s["values"].float() / t, -math.inf)
    most = v.amax(1, keepdim=True)
    some = most > -math.inf
    q = torch.where(used & some, torch.exp(v - torch.where(some, most, 0.0)), 0.0)
    mass = q.sum(1, keepdim=True).clamp_min(1e-30)
    q = q / mass
    log_q = v - most - torch.log(mass)
    log_p = z.gather(1, at) - m - torch.log(total)
    loss = t * t * torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1)
    grad = (e / total).scatter_add(1, at, -q)
    grad = torch.where(some, grad, 0.0) * (t * s["dloss"][:, None])
    return {"loss": loss, "dlogits": grad.to(DTYPES[s["dtype"]])}


def _plain(s):
    dtype = DTYPES[s["dtype"]]
    if s["op"] == "log_probs":
        return _plain_log_probs(s)
    if s["op"] == "distill":
        return _plain_distill(s)
    if s["op"] == "quantize":
        return _decode(*_encode(s["x"].float()), s["cols"]).to(dtype)
    x = s["x"].float()
    if s["acts"] == "mx":
        x = _decode(*_encode(x), s["n_in"])
    w = _decode(s["codes"], s["scales"], s["n_in"])
    return (x @ w.T + s["bias"]).to(dtype)


def run(s):
    if not own:
        return _plain(s)
    ctx = _context(s["dtype"])
    if s["op"] == "log_probs":
        return ctx.log_probs(s["logits"], labels=s["labels"], top=s["top"], temperature=s["temperature"])
    if s["op"] == "distill":
        loss = torch.empty(s["rows"], device="cuda")
        grad = ctx.distill_backward(s["dloss"], s["logits"], s["indices"], s["values"], temperature=s["temperature"],
                                    loss=loss)
        return {"loss": loss, "dlogits": grad}
    if s["op"] == "quantize":
        return ctx.mx_dequantize(ctx.mx_quantize(s["x"]))
    x = ctx.mx_quantize(s["x"]) if s["acts"] == "mx" else s["x"]
    return ctx.mx_product(x, s["weight"], bias=s["bias"])


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("log_probs", "distill"):
        rows, classes, top = case["rows"], case["classes"], case["top"]
        if case["op"] == "log_probs":
            return {"bytes": rows * (size * classes + 20 + 8 * top), "flops": 8.0 * rows * classes}
        return {"bytes": rows * (2 * size * classes + 8 + 8 * top), "flops": 8.0 * rows * classes}
    if case["op"] == "quantize":
        # the matrix in, its 4-bit form out and in again, its values out
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * size * n + 2 * (n / 2 + n / BLOCK), "flops": 4.0 * n}
    m, k, n = (case[q] for q in ("rows", "n_in", "n_out"))
    return {"bytes": size * (m * k + m * n) + n * k * (0.5 + 1 / BLOCK) + 4 * n, "flops": 2.0 * m * n * k}


# ---- the definitions in 64 bits ----------------------------------------------

def _power64(e):
    """2^e in float64 for whole numbers e of its normal range."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _blocks64(x):
    """The values that x [rows, cols] takes in 4 bits, by distance to every value there is."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    # in the order of their codes' parity, so that ties go to the even code
    grid = torch.tensor([MAGNITUDES[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64, device=x.device)
    step = max(BLOCK, (1 << 24) // max(rows, 1) // BLOCK * BLOCK)
    for at in range(0, cols, step):
        v = torch.nn.functional.pad(x[:, at:at + step].double(), (0, -(min(step, cols - at)) % BLOCK))
        v = v.reshape(rows, -1, BLOCK)
        most = v.abs().amax(2, keepdim=True)
        power = torch.floor(torch.log2(most.clamp_min(2.0 ** -126))) - 2
        # (logarithms next to a power of two)
        power = power + (most >= _power64(power + 3)).double() - (most < _power64(power + 2)).double()
        scale = _power64(power.clamp(-127, 127))
        a = (v / scale).abs()
        near, best = torch.full_like(a, math.inf), torch.zeros_like(a)
        for g in grid:
            off = (a - g).abs()
            best = torch.where(off < near, g, best)
            near = torch.minimum(near, off)
        out[:, at:at + step] = (torch.sign(v) * best * scale).reshape(rows, -1)[:, :min(step, cols - at)]
    return out


def _exact_log_probs(s):
    raw, t = s["logits"].double(), s["temperature"]
    parts = []
    for at in range(0, raw.shape[0], 512):
        z = raw[at:at + 512]
        lp = torch.log_softmax(z / t, 1)
        p = lp.exp()
        values, order = torch.sort(z, dim=1, descending=True, stable=True)
        values, order = values[:, :s["top"]], order[:, :s["top"]]
        label = s["labels"][at:at + 512].long()
        at_label = label.clamp_min(0)[:, None]
        mine = z.gather(1, at_label)
        index = torch.arange(z.shape[1], device=z.device)
        rank = ((z > mine) | ((z == mine) & (index < at_label))).sum(1)
        parts.append({
            "entropy": -torch.where(p > 0, p * lp, 0.0).sum(1), "log_sum": torch.logsumexp(z / t, 1),
            "top_indices": torch.where(values > -math.inf, order, -1).int(), "top_log_probs": lp.gather(1, order),
            "log_prob": torch.where(label >= 0, lp.gather(1, at_label)[:, 0], 0.0),
            "rank": torch.where(label >= 0, rank, -1).int()})
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_distill(s):
    t, losses, grads = s["temperature"], [], []
    for at in range(0, s["rows"], 512):
        z = s["logits"][at:at + 512].double() / t
        lp = torch.log_softmax(z, 1)
        index = s["indices"][at:at + 512].long()
        used = index >= 0
        v = (s["values"][at:at + 512].double() / t).masked_fill(~used, -math.inf)
        lq = torch.nan_to_num(torch.log_softmax(v, 1), nan=-math.inf)
        q = lq.exp()
        mine = lp.gather(1, index.clamp_min(0))
        losses.append(t * t * torch.where(q > 0, q * (lq - mine), 0.0).sum(1))
        g = lp.exp() * used.any(1, keepdim=True)
        g.scatter_add_(1, index.clamp_min(0), -q)
        grads.append(g * (t * s["dloss"][at:at + 512, None].double()))
    return {"loss": torch.cat(losses), "dlogits": torch.cat(grads)}


def exact(case, seed):
    global own
    # (the definition needs the plain codes of the weights, whichever side asks)
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "log_probs":
        return _exact_log_probs(s)
    if case["op"] == "distill":
        return _exact_distill(s)
    if case["op"] == "quantize":
        return _blocks64(s["x"])
    values = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    codes = s["codes"].long()
    w = values[codes % 8] * (1.0 - 2.0 * (codes // 8)) * _power64(s["scales"])[:, :, None]
    w = w.reshape(case["n_out"], -1)[:, :case["n_in"]]
    x = _blocks64(s["x"]) if case["acts"] == "mx" else s["x"].double()
    return torch.addmm(s["bias"].double(), x, w.T)
