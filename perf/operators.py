"""The policy's operators that are timed: their cases, inputs, plain forms and 64-bit results.

A case is one call that a program makes on the other side of the environments' loop: the norm in front of
a layer of the policy (forward, with an 8-bit output, or backward), a layer's 8-bit matrix product, the
verification of drafted actions or tokens, the update of the policy's weights.
"""
import math

import torch

own = False  # True: the framework's kernels; False: the plain forms

DEVICE = "cuda:0"
BLOCK = 128  # elements that share a scale
EPS = 1e-5
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16,
         "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
TINY = 2.0 ** -100  # the least maximum that a block's scale is made for
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP, SEED = 3e-4, 0.9, 0.999, 1e-8, 0.01, 100, 17


# ---- the cases -------------------------------------------------------------------------------------
def _norm(name, rows, width, dtype="bfloat16", direction="forward", residual=True, out="e4m3"):
    return {"name": name, "kind": "norm", "rows": rows, "width": width, "type": dtype, "direction": direction,
            "residual": residual, "out": out}


def _product(name, m, n, k, a="e4m3", scales="block", out="bfloat16"):
    return {"name": name, "kind": "product", "m": m, "n": n, "k": k, "a": a, "scales": scales, "out": out}


def _verify(name, batch, drafts, vocab, bonus, ragged, dtype="float32"):
    return {"name": name, "kind": "verify", "batch": batch, "drafts": drafts, "vocab": vocab, "bonus": bonus,
            "ragged": ragged, "type": dtype}


def _adamw(name, policies, inputs, width, layers, bits, dtype):
    return {"name": name, "kind": "adamw", "policies": policies, "inputs": inputs, "width": width, "layers": layers,
            "bits": bits, "type": dtype}


def listed():
    return [
        # one iteration of the smallest workload (10 envs x 5 agents) before a 256-wide layer: latency
        _norm("norm_50x256", 50, 256),
        # the headline workload (2000 envs x 1000 agents) before a 256-wide layer
        _norm("norm_2000000x256", 2000000, 256),
        # a training batch's way back through a layer of odd width, the residual's gradient added
        _norm("norm_backward_33333x999", 33333, 999, direction="backward", out="plain"),
        # one iteration of the smallest workload through a 256-wide layer: latency
        _product("product_50x256x256", 50, 256, 256),
        # a few rows against the weights of a wide layer: the weights' bytes
        _product("product_16x4096x4096", 16, 4096, 4096),
        # the headline workload through a 256-wide layer
        _product("product_2000000x256x256", 2000000, 256, 256),
        # a trainer's large batch through a wide layer: the matrix cores' rate
        _product("product_8192x8192x4096", 8192, 8192, 4096),
        # gradients against weights with a scale per row, odd sizes, as the way back has them
        _product("product_5000x333x1000_rows", 5000, 333, 1000, a="e5m2", scales="row", out="float32"),
        # the headline workload's drafted actions, one for each agent, five to choose from
        _verify("verify_2000000x1x5", 2000000, 1, 5, False, False),
        # sequences of up to four drafted tokens over a large vocabulary, and one more token from the last row
        _verify("verify_64x4x50000", 64, 4, 50000, True, True),
        # the two policies of Tag (taggers, runners), small layers: one step of the optimiser is all latency
        _adamw("adamw_2x64", 2, 21, 64, 2, 32, "float32"),
        # a large policy of odd widths, bfloat16 weights with 32-bit masters, states in 8 bits
        _adamw("adamw_2999_8bit", 1, 333, 2999, 7, 8, "bfloat16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm", "product", "verify", "adamw"])
    if kind == "norm":
        width = _log_uniform(rng, 5, 16384)
        rows = _log_uniform(rng, 1, max(1, min(2000000, 200000000 // width)))
        back = rng.random() < 0.35
        dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
        c = _norm("", rows, width, dtype, "backward" if back else "forward", rng.random() < 0.7,
                  "plain" if back else rng.choice(["e4m3", "e4m3", "plain", "e5m2"]))
    elif kind == "product":
        n, k = _log_uniform(rng, 5, 8192), _log_uniform(rng, 21, 8192)
        m = _log_uniform(rng, 1, min(2000000, 1200000000 // (2 * n + k), 270000000000 // (n * k)))
        c = _product("", m, n, k, rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"]), rng.choice(["block", "block", "row"]),
                     rng.choice(["bfloat16", "bfloat16", "float16", "float32"]))
    elif kind == "verify":
        vocab = 5 if rng.random() < 0.3 else _log_uniform(rng, 17, 150000)
        drafts = 1 if vocab == 5 else rng.randint(1, 8)
        batch = _log_uniform(rng, 1, min(2000000, 20000000 // ((drafts + 1) * vocab)))
        c = _verify("", batch, drafts, vocab, vocab != 5 and rng.random() < 0.7, drafts > 1 and rng.random() < 0.6,
                    rng.choice(["float32", "float32", "bfloat16", "float16"]))
    else:
        width, layers = _log_uniform(rng, 16, 3000), rng.randint(1, 6)
        c = _adamw("", rng.randint(1, 2) if width < 1500 else 1, _log_uniform(rng, 5, 1000), width, layers,
                   rng.choice([32, 32, 8]), rng.choice(["float32", "bfloat16"]))
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------------
def _blocks(n):
    return -(-n // BLOCK)


def _eight_bits(v, kind, rows):
    """Values -> (8-bit tensor whose rows are padded to 16 bytes, scales per `rows` rows x 128 elements)."""
    m, k = v.shape
    mb, kb = -(-m // rows), _blocks(k)
    padded = torch.zeros((mb * rows, kb * BLOCK), device=DEVICE)
    padded[:m, :k] = v
    cells = padded.view(mb, rows, kb, BLOCK)
    scale = cells.abs().amax(dim=(1, 3)).clamp_(min=TINY) / LARGEST[kind]
    cells = cells / scale[:, None, :, None]
    store = torch.zeros((m, -(-k // 16) * 16), device=DEVICE, dtype=TYPES[kind])
    store[:, :k] = cells.view(mb * rows, kb * BLOCK)[:m, :k].to(TYPES[kind])
    return store[:, :k], scale


def _shapes(case):
    """The tensors of the policies: input layer, hidden layers with a norm each, head of five actions."""
    w, one = case["width"], []
    one += [(w, case["inputs"]), (w,)]
    for _ in range(case["layers"]):
        one += [(w,), (w, w), (w,)]
    one += [(5, w), (5,)]
    return one * case["policies"]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=DEVICE, dtype=torch.float32)

    s = {"case": case}
    if case["kind"] == "norm":
        rows, width, t = case["rows"], case["width"], TYPES[case["type"]]
        s["weight"] = 1 + 0.1 * normal(width)
        if case["direction"] == "forward":
            s["x"] = normal(rows, width).to(t)
            s["residual"] = (2 * normal(rows, width)).to(t) if case["residual"] else None
        else:
            s["dy"], s["h"] = normal(rows, width).to(t), (2 * normal(rows, width)).to(t)
            s["dh"] = normal(rows, width).to(t) if case["residual"] else None
            s["rstd"] = torch.rsqrt(s["h"].double().square().mean(1) + EPS).float()
    elif case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], scale = _eight_bits(normal(m, k) * torch.exp(normal(m, 1)), case["a"], 1)
        s["a_scale"] = scale.t().contiguous().t()  # [m, blocks], the rows' scales of a block side by side
        s["b"], s["b_scale"] = _eight_bits(normal(n, k) / math.sqrt(k), "e4m3", 128 if case["scales"] == "block" else 1)
    elif case["kind"] == "verify":
        batch, drafts, vocab, t = case["batch"], case["drafts"], case["vocab"], TYPES[case["type"]]
        logits = 2 * normal(batch, drafts + int(case["bonus"]), vocab)
        s["target"] = torch.softmax(logits, -1).to(t)
        s["draft_probs"] = torch.softmax(logits[:, :drafts] + 0.7 * normal(batch, drafts, vocab), -1).to(t)
        del logits
        # the draft's own draws: the first action whose running sum passes a uniform number
        c = s["draft_probs"].float().cumsum(-1)
        s["drafts"] = torch.searchsorted(c, uniform(batch, drafts, 1) * c[..., -1:], right=True)[..., 0].clamp_(max=vocab - 1).to(torch.int32)
        s["u"] = uniform(batch, drafts + 1)
        s["lengths"] = torch.randint(0, drafts + 1, (batch,), generator=gen, device=DEVICE, dtype=torch.int32) if case["ragged"] else None
    else:
        # one store for each array, a tensor of the policy every 128 elements, as a program that updates in place keeps them
        starts, at = [], 0
        for shape in _shapes(case):
            starts.append(at)
            at += _blocks(math.prod(shape)) * BLOCK
        real = torch.zeros(at, device=DEVICE)
        for start, shape in zip(starts, _shapes(case)):
            real[start:start + math.prod(shape)] = 1
        t = TYPES[case["type"]]
        values = normal(at) * 0.06 * real
        s["param"] = values.to(t)
        s["master"] = values if t != torch.float32 else None
        s["grad"] = (normal(at) * 0.01 * real).to(t)
        m, r = normal(at) * 0.003 * real, (0.002 + 0.002 * uniform(at)) * real  # a hundred steps in: mean, root of the mean square
        if case["bits"] == 32:
            s["exp_avg"], s["exp_avg_sq"] = m, r * r
            s["avg_scale"] = s["sq_scale"] = None
        else:
            (q, a), (r8, b) = _eight_bits(m.view(-1, BLOCK), "e4m3", 1), _eight_bits(r.view(-1, BLOCK), "e4m3", 1)
            s["exp_avg"], s["avg_scale"], s["exp_avg_sq"], s["sq_scale"] = q.reshape(-1), a.reshape(-1), r8.reshape(-1), b.reshape(-1)
        if own:  # the optimiser that a program keeps: it holds which tensors there are
            import paper_2108_13976_amd as wd

            def views(store, per=1):
                return None if store is None else [store[a // per:a // per + (_blocks(math.prod(sh)) if per > 1 else math.prod(sh))]
                                                   for a, sh in zip(starts, _shapes(case))]

            s["optimiser"] = wd.AdamW(views(s["param"]), views(s["grad"]), lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS,
                                      weight_decay=DECAY, state_bits=case["bits"], seed=SEED, masters=views(s["master"]),
                                      exp_avg=views(s["exp_avg"]), exp_avg_sq=views(s["exp_avg_sq"]),
                                      avg_scale=views(s["avg_scale"], BLOCK), sq_scale=views(s["sq_scale"], BLOCK))
    return s


# ---- one pass -------------------------------------------------------------------------------------------
def _plain_norm(s):
    case = s["case"]
    if case["direction"] == "backward":
        dy, h, r = s["dy"].float(), s["h"].float(), s["rstd"][:, None]
        xhat, g = h * r, dy * s["weight"]
        dx = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["h"].dtype), "dw": (dy * xhat).double().sum(0).float()}
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    v = h.float()
    rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    y = v * rstd * s["weight"]
    got = {"rstd": rstd[:, 0]}
    if s["residual"] is not None:
        got["h"] = h
    if case["out"] == "plain":
        got["y"] = y.to(h.dtype)
        return got
    rows, width = y.shape
    cells = torch.nn.functional.pad(y, (0, _blocks(width) * BLOCK - width)).view(rows, -1, BLOCK)
    scale = cells.abs().amax(2).clamp(min=TINY) / LARGEST[case["out"]]
    got["q"] = (cells / scale[:, :, None]).view(rows, -1)[:, :width].to(TYPES[case["out"]])
    got["scale"] = scale
    return got


def _own_norm(s):
    import paper_2108_13976_amd as wd

    case = s["case"]
    if case["direction"] == "backward":
        dx, dw = wd.rms_norm_backward(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"])
        return {"dx": dx, "dw": dw}
    out = wd.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                      out8=None if case["out"] == "plain" else TYPES[case["out"]])
    got = {"rstd": out.rstd}
    if s["residual"] is not None:
        got["h"] = out.h
    if case["out"] == "plain":
        got["y"] = out.y
    else:
        got["q"], got["scale"] = out.q, out.scale
    return got


def _values(q, scale, rows):
    """What an 8-bit tensor stands for, in 32 bits."""
    m, k = q.shape
    each = scale.repeat_interleave(BLOCK, 1)[:, :k]
    return q.float() * (each if rows == 1 else each.repeat_interleave(rows, 0)[:m])


def _plain_product(s):
    a, b = _values(s["a"], s["a_scale"], 1), _values(s["b"], s["b_scale"], 128 if s["case"]["scales"] == "block" else 1)
    return (a @ b.t()).to(TYPES[s["case"]["out"]])


def _own_product(s):
    import paper_2108_13976_amd as wd

    return wd.product8(s["a"], s["a_scale"], s["b"], s["b_scale"], dtype=TYPES[s["case"]["out"]])


def _plain_verify(s):
    p, q, x, u = s["target"], s["draft_probs"], s["drafts"].long(), s["u"].double()
    batch, drafts = x.shape
    vocab, bonus = p.shape[2], s["case"]["bonus"]
    length = torch.full((batch,), drafts, device=DEVICE) if s["lengths"] is None else s["lengths"].long()
    px, qx = (t[:, :drafts].gather(2, x[:, :, None])[:, :, 0].double() for t in (p, q))
    place = torch.arange(drafts, device=DEVICE)
    ok = (u[:, :drafts] * qx < px) & (place < length[:, None])
    accepted = ok.int().cumprod(1).sum(1)
    whole = accepted == length
    each = torch.arange(batch, device=DEVICE)
    row = p[each, accepted.clamp(max=p.shape[1] - 1)].double()
    rest = row - torch.where(whole[:, None], torch.zeros_like(row), q[each, accepted.clamp(max=drafts - 1)].double())
    rest = rest.clamp_(min=0)
    rest = torch.where((rest > 0).any(1, keepdim=True), rest, row.clamp(min=0))
    c = rest.cumsum(1)
    past = (rest > 0) & (c > u[:, drafts:] * c[:, -1:])
    spots = torch.arange(vocab, device=DEVICE)
    first = torch.where(past, spots, vocab).amin(1)
    last = torch.where(rest > 0, spots, -1).amax(1)
    token = torch.where(first < vocab, first, last)
    slots = torch.arange(drafts + int(bonus), device=DEVICE)
    kept = torch.nn.functional.pad(x, (0, int(bonus)))
    drawn = (slots == accepted[:, None]) & (~whole[:, None] | bonus)
    tokens = torch.where(slots < accepted[:, None], kept, torch.where(drawn, token[:, None], -1))
    return {"accepted": accepted.int(), "tokens": tokens.int()}


def _own_verify(s):
    import paper_2108_13976_amd as wd

    accepted, tokens = wd.verify_drafts(s["target"], s["draft_probs"], s["drafts"], s["u"], lengths=s["lengths"])
    return {"accepted": accepted, "tokens": tokens}


def _words(elements):
    """One 32-bit random word for each element: Philox4x32-10 blocks of four, counter (element / 4, step), key SEED."""
    c0 = torch.arange(elements // 4, device=DEVICE, dtype=torch.int64)
    c1, c2, c3 = torch.zeros_like(c0), torch.full_like(c0, STEP), torch.full_like(c0, 4)
    k0, k1, low = SEED, 0, 0xFFFFFFFF

    def high(k, c):  # upper half of a 32 x 32 bit product
        return (k * (c >> 16) + ((k * (c & 0xFFFF)) >> 16)) >> 16

    for _ in range(10):
        hi_a, lo_a, hi_b, lo_b = high(0xD2511F53, c0), (0xD2511F53 * c0) & low, high(0xCD9E8D57, c2), (0xCD9E8D57 * c2) & low
        c0, c1, c2, c3 = hi_b ^ c1 ^ k0, lo_b, hi_a ^ c3 ^ k1, lo_a
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), 1).view(-1)


def _round_up_or_down(v, r):
    """v (e4m3's range) to a neighbour in e4m3, upwards with the probability of how near it is; r: 16 random bits."""
    size = v.abs()
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign((torch.floor(size / step + r.float() / 65536) * step).clamp(max=448.0), v)


def _plain_adamw(s):
    case = s["case"]
    p = (s["param"] if s["master"] is None else s["master"]).float()
    g = s["grad"].float()
    m, v = s["exp_avg"], s["exp_avg_sq"]
    if case["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["avg_scale"][:, None]).view(-1)
        r = (v.float().view(-1, BLOCK) * s["sq_scale"][:, None]).view(-1)
        v = r * r
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    c1, c2 = 1 - BETA1 ** STEP, 1 - BETA2 ** STEP
    p = p * (1 - LR * DECAY) - LR * (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS)
    s["param"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    if case["bits"] == 32:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
    else:
        # a tensor's elements are counted from its own start, in one run of numbers over the tensors' blocks
        word = _words(m.numel())
        for values, codes, scales, bits in ((m, s["exp_avg"], s["avg_scale"], word & 0xFFFF), (torch.sqrt(v), s["exp_avg_sq"], s["sq_scale"], word >> 16)):
            cells = values.view(-1, BLOCK)
            scale = cells.abs().amax(1).clamp(min=TINY) / 448
            new = _round_up_or_down((cells / scale[:, None]).view(-1), bits)
            if codes is s["exp_avg_sq"]:  # a root that is not zero stays above it
                new = torch.where(values > 0, new.clamp(min=2.0 ** -9), new)
            codes.copy_(new.to(torch.float8_e4m3fn))
            scales.copy_(scale)
    return {n: s[n] for n in ("param", "master", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale")}


def _own_adamw(s):
    s["optimiser"].step(step=STEP)
    return {n: s[n] for n in ("param", "master", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale")}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "product": _own_product, "verify": _own_verify, "adamw": _own_adamw}[kind](state)
    return {"norm": _plain_norm, "product": _plain_product, "verify": _plain_verify, "adamw": _plain_adamw}[kind](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------
def work(case):
    if case["kind"] == "norm":
        rows, width, b = case["rows"], case["width"], BYTES[case["type"]]
        each = rows * width
        if case["direction"] == "backward":
            moved = each * b * (4 if case["residual"] else 3) + 4 * rows + 8 * width
            return {"bytes": moved, "flops": 9 * each}
        moved = each * b * (3 if case["residual"] else 1) + 4 * rows + 4 * width
        moved += each * b if case["out"] == "plain" else each + 4 * rows * _blocks(width)
        return {"bytes": moved, "flops": 6 * each}
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        scales = m + (_blocks(n) if case["scales"] == "block" else n)
        return {"bytes": (m + n) * k + 4 * scales * _blocks(k) + m * n * BYTES[case["out"]], "flops": 2 * m * n * k}
    if case["kind"] == "verify":
        # an element of both rows for each draft, one row of both (the last row, the bonus, of one), randoms and tokens
        batch, drafts, vocab, b = case["batch"], case["drafts"], case["vocab"], BYTES[case["type"]]
        moved = batch * (2 * vocab * b + 2 * drafts * b + 4 * drafts + 4 * (drafts + 1) + 4 * (drafts + int(case["bonus"])) + 4)
        return {"bytes": moved + (4 * batch if case["ragged"] else 0), "flops": 4 * batch * vocab}
    n = sum(math.prod(shape) for shape in _shapes(case))
    b = BYTES[case["type"]]
    moved = n * (3 * b + (8 if case["type"] != "float32" else 0) - (b if case["type"] != "float32" else 0))
    moved += n * (16 if case["bits"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": moved, "flops": 16 * n}


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        w = s["weight"].double()
        if case["direction"] == "backward":
            rows, width = s["h"].shape
            h, dy, rstd = s["h"].double(), s["dy"].double(), s["rstd"].double()
            both = dy * h
            dot = (both * w).sum(1)  # sum of dy w h
            dx = dy * w * rstd[:, None] - h * (dot * rstd ** 3 / width)[:, None]
            return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dw": (both * rstd[:, None]).sum(0)}
        # the norm is that of the sum as it is stored
        h = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
        v = h.double()
        power = v.pow(2).sum(1) / case["width"] + EPS
        y = v / power.sqrt()[:, None] * w
        got = {"rstd": power.pow(-0.5)}
        if s["residual"] is not None:
            got["h"] = s["x"].double() + s["residual"].double()
        if case["out"] == "plain":
            return {**got, "y": y}
        scale = torch.stack([t.abs().amax(1) for t in y.split(BLOCK, 1)], 1).clamp(min=TINY) / LARGEST[case["out"]]
        return {**got, "scale": scale, "q": y / scale.repeat_interleave(BLOCK, 1)[:, :case["width"]]}
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        total = torch.zeros((m, n), dtype=torch.float64, device=DEVICE)
        for b in range(_blocks(k)):
            part = s["a"][:, b * BLOCK:(b + 1) * BLOCK].double() * s["a_scale"][:, b, None].double()
            scale = s["b_scale"][:, b].double()
            if case["scales"] == "block":
                scale = scale.repeat_interleave(BLOCK)[:n]
            total.addmm_(part, (s["b"][:, b * BLOCK:(b + 1) * BLOCK].double() * scale[:, None]).t())
        return total
    if case["kind"] == "verify":
        return None  # whole numbers: the plain form computes them in 64 bits
    b1, b2 = BETA1, BETA2
    p = (s["param"] if s["master"] is None else s["master"]).double()
    g = s["grad"].double()
    m, v = s["exp_avg"].double(), s["exp_avg_sq"].double()
    if case["bits"] == 8:
        m = m * s["avg_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["sq_scale"].double().repeat_interleave(BLOCK)) ** 2
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g ** 2 - v)
    move = m / (1 - math.pow(b1, STEP)) / ((v / (1 - math.pow(b2, STEP))).sqrt() + ADAM_EPS)
    p = p - LR * (DECAY * p + move)
    got = {"param": p, "master": None if s["master"] is None else p, "exp_avg": m, "exp_avg_sq": v, "avg_scale": None, "sq_scale": None}
    if case["bits"] == 8:
        v = v.sqrt()
        for values, codes, scales in ((m, "exp_avg", "avg_scale"), (v, "exp_avg_sq", "sq_scale")):
            got[scales] = values.view(-1, BLOCK).abs().amax(1).clamp(min=TINY) / 448
            got[codes] = values / got[scales].repeat_interleave(BLOCK)
    return got
