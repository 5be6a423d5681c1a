"""The measured operators around the decoder that learns and answers: token
embedding, final norm, next-token loss and optimizer step, each through the
package's public entry points and in a plain form of elementary tensor
operations.

Kinds of case:
  embed    svl_embed, and with a gradient svl_embed_backward: rows of a table by
           token, and the table's gradient as sums over each token's rows
  norm     svl_norm_forward, and with a gradient svl_norm_backward: RMS or layer
           norm of rows, and the gradients of the rows, the gain and the bias
  loss     svl_lm_loss: the language-model head's softmax cross entropy against
           each row's label, and the gradients of the rows and of the head; a row
           without a label (an image position) has neither loss nor gradient
  adamw    svl_adamw_step over a list of tensors, states in 32 bits or in 8, and
           for 8 bits svl_adamw_read_state: the moments that the codes stand for

Widths are those of workloads/configs.py (256, 3584, 4096, 5120) and the generic
1024; vocabularies are 32000 and generic odd sizes.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256                     # elements of an 8-bit state that share a scale
WORD = 0xFFFFFFFF


# ------------------------------------------------------------------ cases
def _case(kind, name, **more):
    case = dict(kind=kind, **more)
    if name:
        case["name"] = name
    return case


def _embed(name, rows, width, vocab, table, row, grad, accumulate=False, scale=1.0):
    return _case("embed", name, rows=rows, width=width, vocab=vocab, table=table, row=row, grad=grad,
                 accumulate=accumulate, scale=scale)


def _norm(name, rows, width, how, x, y, gain, grad, bias=False):
    return _case("norm", name, rows=rows, width=width, how=how, x=x, y=y, gain=gain, grad=grad, bias=bias)


def _loss(name, rows, width, vocab, compute, grad_x, grad_w, ignored, scale=1.0, accumulate=False):
    return _case("loss", name, rows=rows, width=width, vocab=vocab, compute=compute, grad_x=grad_x, grad_w=grad_w,
                 ignored=ignored, scale=scale, accumulate=accumulate)


def _adamw(name, sizes, param, grad, bits, master=False):
    return _case("adamw", name, sizes=",".join(str(int(n)) for n in sizes), param=param, grad=grad, bits=bits,
                 master=master)


def _decoder_layer(d, f):
    return [d] + [d * d] * 4 + [d] + [d * f] * 3


def listed():
    return [
        # serving: the hidden rows of eight requests' next tokens
        _embed("embed_step_b8", 8, 4096, 32000, "bf16", "bf16", False),
        # training: a batch's text, image positions without a token
        _embed("embed_train", 16384, 4096, 32000, "bf16", "f32", True),
        # serving: the rows of eight requests before the head
        _norm("norm_step_b8", 8, 4096, "rms", "f32", "bf16", "bf16", False),
        # training: the residual stream's norm before the head, forward and backward
        _norm("norm_train_rms", 8192, 4096, "rms", "f32", "bf16", "bf16", True),
        # training: a vision encoder's norm over the patches and class rows of five images
        _norm("norm_train_layer", 2885, 1024, "layer", "f16", "f16", "f32", True, bias=True),
        # serving: log-probabilities of given tokens, one row of each of eight requests
        _loss("score_step_b8", 8, 4096, 32000, "f16", False, False, 0.0),
        # a few questions, half of the positions without a label
        _loss("loss_prompt", 640, 4096, 32000, "bf16", True, True, 0.5),
        # the controllers learn through a frozen decoder: the rows' gradient only, odd sizes, a scaled loss
        _loss("loss_frozen_head", 3001, 3584, 65537, "f16", True, False, 0.25, 1024.0),
        # a training batch
        _loss("loss_train", 8192, 4096, 32000, "bf16", True, True, 0.1),
        # the compute controller's linears, biases and gates: small tensors of odd sizes
        _adamw("adamw_controller", [256 * 4096, 4096, 4096 * 4096, 4096] + [4097 + 130 * i for i in range(56)],
               "f32", "f32", 32),
        # a decoder layer in bf16 with 32-bit copies and states
        _adamw("adamw_layer", _decoder_layer(4096, 11008), "bf16", "bf16", 32, master=True),
        # a decoder layer of another width, its states in 8 bits, and their values read back
        _adamw("adamw_layer_8bit", _decoder_layer(3584, 9473), "bf16", "f32", 8, master=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["embed", "norm", "loss", "loss", "adamw"])
    width = rng.choice([256, 1024, 3584, 4096, 5120])
    any_type = lambda: rng.choice(["f32", "bf16", "f16"])  # noqa: E731
    if kind == "embed":
        grad = rng.random() < 0.7
        return _embed(None, log_int(1, 12000), width, log_int(500, 50000), any_type(), any_type(), grad,
                      grad and rng.random() < 0.4, rng.choice([1.0, 1.0, 16.0, 0.125]))
    if kind == "norm":
        how = rng.choice(["rms", "layer"])
        width = rng.choice([width, 8 * log_int(1, 700)])
        return _norm(None, log_int(1, 7000), width, how, any_type(), any_type(), any_type(), rng.random() < 0.7,
                     how == "layer" and rng.random() < 0.7)
    if kind == "loss":
        both = rng.choice(["none", "x", "w", "xw", "xw"])
        vocab = log_int(500, 140000)
        top = int(8192 * 4096 * 32000 * 0.6 / (width * vocab))
        compute = rng.choice(["bf16", "f16"])
        return _loss(None, log_int(1, min(top, 8000)), width, vocab, compute, "x" in both, "w" in both,
                     rng.choice([0.0, 0.1, 0.6, 0.9]), 1024.0 if compute == "f16" else 1.0,
                     "w" in both and rng.random() < 0.3)
    sizes = [log_int(1, 3000000) for _ in range(log_int(1, 90))]
    return _adamw(None, sizes, any_type(), any_type(), rng.choice([8, 32]), rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _randn(gen, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _tokens(gen, n, vocab, none=0.0):
    """Tokens of text: the i-th most frequent about 1 / i as often; -1 where there is none."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab)).long().clamp(1, vocab) - 1
    t = (rank * 7919 + 11) % vocab                       # frequent tokens lie anywhere in the table
    gone = torch.rand(n, generator=gen, device="cuda") < none
    return torch.where(gone, torch.full_like(t, -1), t).to(torch.int32)


def _sizes(case):
    return [int(n) for n in str(case["sizes"]).split(",")]


def _blocks(case):
    return [-(-n // BLOCK) for n in _sizes(case)]


def _prepare_adamw(case, gen):
    """Each kind of buffer is one allocation, the tensors at multiples of 256 elements in it."""
    sizes, blocks = _sizes(case), _blocks(case)
    total = sum(blocks) * BLOCK
    first = [0]
    for b in blocks:
        first.append(first[-1] + b * BLOCK)
    st = dict(first=first, step=17, seed=4242)
    # the space behind a tensor's end belongs to no tensor: zeros
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, n in zip(first, sizes):
        inside[a:a + n] = True

    def flat(std, dtype):
        return (torch.randn(total, generator=gen, device="cuda") * std * inside).to(dtype)

    master = flat(0.02, torch.float32)
    st["param"] = master.to(TYPES[case["param"]])
    if case["master"]:
        st["master"] = master
    # gradients of tensors whose sizes differ by decades, within each a spread of rows
    level = torch.exp(torch.randn(len(sizes), generator=gen, device="cuda") * 1.5 - 7.0)
    level = level.repeat_interleave(torch.tensor(blocks, device="cuda")).repeat_interleave(BLOCK)
    grad = torch.randn(total, generator=gen, device="cuda") * level * inside
    if case["bits"] == 32:
        st["m"] = torch.randn(total, generator=gen, device="cuda") * level * inside * 0.3
        st["v"] = (torch.rand(total, generator=gen, device="cuda") + 0.1) * level * level * inside
    else:
        coarse = level[::BLOCK]
        inside8 = inside.to(torch.uint8)
        for name in ("m", "v"):
            # codes of the top six binades and both signs (m) or none (v), scales near the gradients' size
            low, high = (64, 120) if name == "m" else (192, 248)
            c = torch.randint(low, high, (total,), generator=gen, device="cuda").to(torch.uint8)
            if name == "m":
                c += 128 * (torch.rand(total, generator=gen, device="cuda") < 0.5).to(torch.uint8)
            st[name] = c * inside8
            st[name + "_scale"] = _power(torch.frexp(coarse)[1])
    st["grad"] = grad.to(TYPES[case["grad"]])
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    st = dict(case=case)
    if kind == "embed":
        n, d, v = case["rows"], case["width"], case["vocab"]
        st["tokens"] = _tokens(gen, n, v, 0.1 if case["grad"] else 0.0)
        st["table"] = _randn(gen, (v, d), TYPES[case["table"]], 0.02)
        if case["grad"]:
            st["grad"] = _randn(gen, (n, d), TYPES[case["row"]], 0.01)
        if case["accumulate"]:
            st["held"] = _randn(gen, (v, d), TYPES[case["table"]], 0.01)
    elif kind == "norm":
        n, d = case["rows"], case["width"]
        # a residual stream: rows of different size, a few channels that stand out
        x = torch.randn((n, d), generator=gen, device="cuda")
        x *= torch.exp(torch.randn((n, 1), generator=gen, device="cuda") * 0.5)
        x[:, 5::97] *= 8.0
        st["x"] = (x + 0.1).to(TYPES[case["x"]])
        st["gain"] = (1 + _randn(gen, d, std=0.02)).to(TYPES[case["gain"]])
        st["bias"] = _randn(gen, d, TYPES[case["gain"]], 0.02) if case["bias"] else None
        if case["grad"]:
            st["grad"] = _randn(gen, (n, d), TYPES[case["y"]], 0.01)
    elif kind == "loss":
        n, d, v = case["rows"], case["width"], case["vocab"]
        dt = TYPES[case["compute"]]
        st["labels"] = _tokens(gen, n, v, case["ignored"])
        st["w"] = _randn(gen, (v, d), dt, 0.02)
        # normed rows that know their label more or less well
        sure = torch.rand((n, 1), generator=gen, device="cuda") * (16384.0 / d)
        st["x"] = (_randn(gen, (n, d)) + sure * st["w"][st["labels"].long().clamp(min=0)].float()).to(dt)
        valid = (st["labels"] >= 0).sum().clamp(min=1)
        st["row_weight"] = (torch.ones(n, device="cuda") * case["scale"] / valid).contiguous()   # the mean's gradient
        if case["accumulate"]:
            st["held"] = _randn(gen, (v, d), dt, 1e-4 * case["scale"])
    else:
        st.update(_prepare_adamw(case, gen))
    return st


# ------------------------------------------------------------------ plain forms
def _plain_embed(st):
    case = st["case"]
    there = (st["tokens"] >= 0) & (st["tokens"] < case["vocab"])
    at = torch.where(there, st["tokens"], torch.zeros_like(st["tokens"])).long()
    out = (st["table"][at].float() * case["scale"] * there[:, None]).to(TYPES[case["row"]])
    if not case["grad"]:
        return out
    total = torch.zeros((case["vocab"], case["width"]), device="cuda")
    total.index_add_(0, at, st["grad"].float() * there[:, None])
    total = total * case["scale"]
    if case["accumulate"]:
        st["held"].copy_(st["held"].float() + total)
        return out, st["held"]
    return out, total.to(TYPES[case["table"]])


EPS = 1e-6


def _plain_norm(st):
    case = st["case"]
    x, gain = st["x"].float(), st["gain"].float()
    mean = x.mean(-1, keepdim=True) if case["how"] == "layer" else torch.zeros_like(x[:, :1])
    c = x - mean
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    z = c * r
    y = z * gain
    if st["bias"] is not None:
        y = y + st["bias"].float()
    y = y.to(TYPES[case["y"]])
    if not case["grad"]:
        return y
    g = st["grad"].float()
    h = g * gain
    dx = h - z * (h * z).mean(-1, keepdim=True)
    if case["how"] == "layer":
        dx = dx - h.mean(-1, keepdim=True)
    out = (y, (dx * r).to(TYPES[case["x"]]), (g * z).sum(0))
    return out + (g.sum(0),) if st["bias"] is not None else out


def _plain_loss(st):
    case = st["case"]
    dt, w = TYPES[case["compute"]], st["w"].float()
    there = (st["labels"] >= 0) & (st["labels"] < case["vocab"])
    at = torch.where(there, st["labels"], torch.zeros_like(st["labels"])).long()[:, None]
    s = torch.matmul(st["x"].float(), w.t())
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    loss = torch.where(there, (lse - s.gather(1, at)).squeeze(1), torch.zeros_like(st["row_weight"]))
    out = [loss, torch.where(there, lse.squeeze(1), torch.zeros_like(loss))]
    if not (case["grad_x"] or case["grad_w"]):
        return tuple(out)
    del s
    p = e.div_(total)
    p.scatter_add_(1, at, torch.full_like(top, -1.0))
    p.mul_((st["row_weight"] * there)[:, None])
    if case["grad_x"]:
        out.append(torch.matmul(p, w).to(dt))
    if case["grad_w"]:
        dw = torch.matmul(p.t(), st["x"].float())
        if case["accumulate"]:
            st["held"].copy_(st["held"].float() + dw)
            out.append(st["held"])
        else:
            out.append(dw.to(dt))
    return tuple(out)


BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.95, 1e-8, 3e-4, 0.1


def _as_f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _power(e):
    """2 to whole numbers, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _values(code, scale, low, sign):
    """What 8-bit codes stand for: three digits after the point, exponents from `low` on, gradual below."""
    c = code.to(torch.int32).view(-1, BLOCK)
    s = 1.0 - 2.0 * (c >> 7).float() if sign else 1.0
    c = c & 127 if sign else c
    e, f = c >> 3, (c & 7).float()
    value = ((e > 0).float() + f / 8.0) * _power((e - 1).clamp(min=0) + low)
    return (s * value * scale[:, None]).flatten()


def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & WORD
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & WORD
    return x ^ (x >> 16)


def _random(case, seed):
    """32 random bits for each element: of the seed, the tensor's number and the element's place in it."""
    blocks = torch.tensor(_blocks(case), device="cuda")
    tensor = torch.arange(len(blocks), device="cuda").repeat_interleave(blocks)
    block = torch.arange(len(tensor), device="cuda") - (torch.cumsum(blocks, 0) - blocks).repeat_interleave(blocks)
    key = _mix((seed + 0x9E3779B9 * (tensor + 1)) & WORD)
    place = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    return _mix((place * 0x9E3779B9 + key[:, None]) & WORD)


def _codes(x, random16, low, sign):
    """Codes and scales of a block's values: a power of two for the block, then rounded up with the chance
    that the random bits give."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(-1)
    _, e = torch.frexp(top)
    scale = torch.where(top > 0, _power((e - 1).clamp(min=-90)), torch.zeros_like(top))
    y = torch.where(scale[:, None] > 0, x.abs() / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None],
                    torch.zeros_like(x))
    up = random16 << 4
    normal = ((y.view(torch.int32).long() + up) >> 20) - ((126 + low) << 3)
    small = ((y * 2.0 ** (23 - low)).long() + up) >> 20
    c = torch.where(y >= 2.0 ** low, normal, small)
    if sign:
        c = c | ((x < 0).long() << 7)
    return c.to(torch.uint8).flatten(), scale


# the lowest normal exponent of the codes: the first moment's, the second's root's
LOW_M, LOW_V = -13, -29


def _plain_adamw(st):
    case = st["case"]
    eight = case["bits"] == 8
    g = st["grad"].float()
    m = _values(st["m"], st["m_scale"], LOW_M, True) if eight else st["m"]
    v = _values(st["v"], st["v_scale"], LOW_V, False).square() if eight else st["v"]
    # the moments are float32, each product and each sum rounded once
    m = _as_f32(BETA1) * m + _as_f32(1 - BETA1) * g
    v = _as_f32(BETA2) * v + (_as_f32(1 - BETA2) * g) * g
    c1, c2 = 1 - BETA1 ** st["step"], 1 - BETA2 ** st["step"]
    p = st["master"] if case["master"] else st["param"].float()
    p = p * (1 - LR * DECAY) - LR * (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS)
    if case["master"]:
        st["master"].copy_(p)
    st["param"].copy_(p)
    out = [st["param"]] + ([st["master"]] if case["master"] else [])
    if not eight:
        st["m"].copy_(m)
        st["v"].copy_(v)
        return tuple(out + [st["m"], st["v"]])
    bits = _random(case, st["seed"])
    root = torch.sqrt(v.double()).float()                 # rounded once
    for name, x, r, low, sign in (("m", m, bits & 0xFFFF, LOW_M, True), ("v", root, bits >> 16, LOW_V, False)):
        c, s = _codes(x, r, low, sign)
        st[name].copy_(c)
        st[name + "_scale"].copy_(s)
    return tuple(out + [_values(st["m"], st["m_scale"], LOW_M, True),
                        _values(st["v"], st["v_scale"], LOW_V, False).square()])


# ------------------------------------------------------------------ the framework's calls
def _own(st):
    import paper_2607_20357_amd as svl
    case = st["case"]
    kind = case["kind"]
    if kind == "embed":
        if "emb" not in st:     # the description and the workspace that a program keeps
            st["emb"] = svl.make_embedding(case["width"], case["vocab"], table=case["table"], rows=case["row"],
                                           scale=case["scale"])
            if case["grad"]:
                st["ws"] = svl.alloc_embed_workspace(st["emb"], case["rows"])
        out = torch.empty((case["rows"], case["width"]), dtype=TYPES[case["row"]], device="cuda")
        svl.svl_embed(st["emb"], st["tokens"], st["table"], out)
        if not case["grad"]:
            return out
        grad = st["held"] if case["accumulate"] else torch.empty_like(st["table"])
        svl.svl_embed_backward(st["emb"], st["tokens"], st["grad"], grad, st["ws"], accumulate=case["accumulate"])
        return out, grad
    if kind == "norm":
        if "norm" not in st:
            st["norm"] = svl.make_norm(case["width"], kind=case["how"], x=case["x"], y=case["y"], gain=case["gain"],
                                       eps=EPS)
            if case["grad"]:
                st["ws"] = svl.alloc_norm_workspace(st["norm"], case["rows"])
        y = torch.empty(st["x"].shape, dtype=TYPES[case["y"]], device="cuda")
        if not case["grad"]:
            svl.svl_norm_forward(st["norm"], st["x"], st["gain"], y, bias=st["bias"])
            return y
        stats = torch.empty((case["rows"], 2), dtype=torch.float32, device="cuda")
        svl.svl_norm_forward(st["norm"], st["x"], st["gain"], y, bias=st["bias"], stats=stats)
        dx = torch.empty_like(st["x"])
        dgain = torch.empty(case["width"], dtype=torch.float32, device="cuda")
        dbias = torch.empty_like(dgain) if st["bias"] is not None else None
        svl.svl_norm_backward(st["norm"], st["x"], st["gain"], stats, st["grad"], dx, st["ws"], grad_gain=dgain,
                              grad_bias=dbias)
        return (y, dx, dgain) if dbias is None else (y, dx, dgain, dbias)
    if kind == "loss":
        if "head" not in st:
            st["head"] = svl.make_lm_head(case["width"], case["vocab"], compute=case["compute"])
            st["ws"] = svl.alloc_lm_loss_workspace(st["head"], case["rows"], grad_x=case["grad_x"],
                                                   grad_w=case["grad_w"])
        loss = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
        lse = torch.empty_like(loss)
        dx = torch.empty_like(st["x"]) if case["grad_x"] else None
        dw = None
        if case["grad_w"]:
            dw = st["held"] if case["accumulate"] else torch.empty_like(st["w"])
        svl.svl_lm_loss(st["head"], st["x"], st["w"], st["labels"], loss, st["ws"], lse=lse,
                        row_weight=st["row_weight"], grad_x=dx, grad_w=dw, accumulate=case["accumulate"])
        return tuple(t for t in (loss, lse, dx, dw) if t is not None)
    if "adam" not in st:
        st["adam"] = svl.make_adamw(lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                                    state_bits=case["bits"])
        tensors = []
        for a, n in zip(st["first"], _sizes(case)):
            t = {k: st[k][a:a + n] for k in ("param", "grad", "master", "m", "v") if k in st}
            if case["bits"] == 8:
                for k in ("m_scale", "v_scale"):
                    t[k] = st[k][a // BLOCK:a // BLOCK + -(-n // BLOCK)]
            tensors.append(t)
        st["tensors"] = svl.AdamwTensors(tensors)
    svl.svl_adamw_step(st["adam"], st["tensors"], step=st["step"], seed=st["seed"])
    out = [st["param"]] + ([st["master"]] if case["master"] else [])
    if case["bits"] == 32:
        return tuple(out + [st["m"], st["v"]])
    for k in ("m", "v"):
        value = torch.empty(st[k].shape, dtype=torch.float32, device="cuda")
        svl.svl_adamw_read_state(k, st[k], st[k + "_scale"], value)
        out.append(value)
    return tuple(out)


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"embed": _plain_embed, "norm": _plain_norm, "loss": _plain_loss, "adamw": _plain_adamw}[kind](state)


# ------------------------------------------------------------------ what a pass cannot do without
def _bytes(name):
    return TYPES[name].itemsize


def work(case):
    kind = case["kind"]
    if kind == "embed":
        n, d, v = case["rows"], case["width"], case["vocab"]
        t, r = _bytes(case["table"]), _bytes(case["row"])
        moved = n * 4 + min(n, v) * d * t + n * d * r
        if case["grad"]:
            # each gradient row in; every row of the table's gradient out, or the rows that change in and out
            moved += n * d * r + (2 * min(n, v) if case["accumulate"] else v) * d * t
        return {"bytes": moved, "flops": 0}
    if kind == "norm":
        n, d = case["rows"], case["width"]
        x, y, g = _bytes(case["x"]), _bytes(case["y"]), _bytes(case["gain"])
        vectors = d * g * (2 if case["bias"] else 1)
        moved = n * d * (x + y) + vectors
        if case["grad"]:
            moved += n * d * (x + y + x) + d * g + (8 if case["bias"] else 4) * d
        return {"bytes": moved, "flops": 0}
    if kind == "loss":
        d, v = case["width"], case["vocab"]
        n = case["rows"] * (1.0 - case["ignored"])      # rows with a label
        moved = 2 * (n * d + v * d) + 12 * case["rows"]
        products = 1 + case["grad_x"] + case["grad_w"]
        if case["grad_x"]:
            moved += 2 * case["rows"] * d
        if case["grad_w"]:
            moved += 2 * v * d * (2 if case["accumulate"] else 1)
        return {"bytes": moved, "flops": 2 * products * n * d * v}
    total = sum(_sizes(case))
    per = _bytes(case["grad"]) + _bytes(case["param"]) * (1 if case["master"] else 2) + (8 if case["master"] else 0)
    per += 16 if case["bits"] == 32 else 2 * 2 + 2 * (1 + 4)     # 8 bits: and the values read back
    return {"bytes": total * per, "flops": 0}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_embed(case, st):
    n, v = case["rows"], case["vocab"]
    token = st["tokens"].cpu().tolist()
    place = [[], []]
    for i, t in enumerate(token):
        if 0 <= t < v:
            place[0].append(i)
            place[1].append(t)
    where = torch.tensor(place, dtype=torch.int64, device="cuda").view(2, -1)
    out = torch.zeros((n, case["width"]), dtype=torch.float64, device="cuda")
    out[where[0]] = st["table"].double()[where[1]] * case["scale"]
    if not case["grad"]:
        return out
    # rows in the order of their tokens, then sums of the runs as differences of running sums
    order = torch.argsort(where[1], stable=True)
    run_sum = torch.cumsum(st["grad"].double()[where[0][order]], 0)
    run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum]) if len(token) else run_sum
    edge = torch.searchsorted(where[1][order].contiguous(), torch.arange(v + 1, device="cuda"))
    total = (run_sum[edge[1:]] - run_sum[edge[:-1]]) * case["scale"]
    return out, total + st["held"].double() if case["accumulate"] else total


def _exact_norm(case, st):
    x, gain = st["x"].double(), st["gain"].double()
    d = case["width"]
    centre = (torch.eye(d, dtype=torch.float64, device="cuda") - 1.0 / d) if d <= 1024 else None
    if case["how"] == "layer":
        c = x @ centre if centre is not None else x - x.sum(1, keepdim=True) / d
    else:
        c = x
    size = torch.sqrt(torch.linalg.vector_norm(c, dim=1, keepdim=True) ** 2 / d + EPS)
    y = c / size * gain
    if st["bias"] is not None:
        y = y + st["bias"].double()
    if not case["grad"]:
        return y
    g = st["grad"].double()
    h = g * gain
    # the derivative of c / size, then of the centring
    along = (h * c).sum(1, keepdim=True) / (d * size ** 3)
    dc = h / size - c * along
    dx = dc - dc.sum(1, keepdim=True) / d if case["how"] == "layer" else dc
    out = (y, dx, torch.einsum("nd,nd->d", g, c / size))
    return out + (torch.einsum("nd->d", g),) if st["bias"] is not None else out


def _exact_loss(case, st):
    n, v = case["rows"], case["vocab"]
    w, x = st["w"].double(), st["x"].double()
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for a in range(0, n, 1024):
        z = min(n, a + 1024)
        s = x[a:z] @ w.t().contiguous()
        lse[a:z] = torch.logsumexp(s, -1)
        label = st["labels"][a:z].long()
        ok = (label >= 0) & (label < v)
        at = torch.nonzero(ok).squeeze(1)
        loss[a + at] = lse[a + at] - s[at, label[at]]
        if case["grad_x"] or case["grad_w"]:
            p = torch.exp(s - lse[a:z, None])
            p[at, label[at]] -= 1.0
            p *= torch.where(ok, st["row_weight"][a:z].double(), torch.zeros_like(loss[a:z]))[:, None]
            if case["grad_x"]:
                dx[a:z] = p @ w
            if case["grad_w"]:
                dw += p.t().contiguous() @ x[a:z]
        del s
    has = (st["labels"] >= 0) & (st["labels"] < v)
    out = [loss, torch.where(has, lse, torch.zeros_like(lse))]
    if case["grad_x"]:
        out.append(dx)
    if case["grad_w"]:
        out.append(dw + st["held"].double() if case["accumulate"] else dw)
    return tuple(out)


def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _float32(x):
    return x.float().double()


def _exact_adamw(case, st):
    """Tensor by tensor in float64; a moment is rounded to float32 after each product and sum, as it is defined."""
    outs = {k: [] for k in ("param", "master", "m", "v")}
    step, seed = st["step"], st["seed"]
    for number, (a, n) in enumerate(zip(st["first"], _sizes(case))):
        z = a + -(-n // BLOCK) * BLOCK
        g = st["grad"][a:z].double()
        old = {}
        for k, bias, mask in (("m", 14, 127), ("v", 30, 255)):
            if case["bits"] == 32:
                old[k] = st[k][a:z].double()
                continue
            code = st[k][a:z].double()
            negative = code > mask
            code = torch.where(negative, code - 128, code)
            e = torch.floor(code / 8)
            f = code - 8 * e
            one = (e > 0).double()
            size = (one + f / 8) * _power64(torch.clamp(e, min=1) - bias)
            size = size * st[k + "_scale"][a // BLOCK:z // BLOCK].double().repeat_interleave(BLOCK)
            old[k] = torch.where(negative, -size, size) if k == "m" else _float32(size * size)
        b1, b2, r1, r2 = (_as_f32(t) for t in (BETA1, BETA2, 1 - BETA1, 1 - BETA2))
        m = _float32(_float32(b1 * old["m"]) + _float32(r1 * g))
        v = _float32(_float32(b2 * old["v"]) + _float32(_float32(r2 * g) * g))
        p = (st["master"] if case["master"] else st["param"])[a:z].double()
        rate = m / (1 - BETA1 ** step) / (torch.sqrt(v / (1 - BETA2 ** step)) + ADAM_EPS)
        p = p - LR * DECAY * p - LR * rate
        outs["param"].append(p)
        outs["master"].append(p)
        if case["bits"] == 8:
            def mixed(t):
                for shift, factor in ((16, 0x6A09E667), (15, 0xBB67AE85)):
                    t = torch.bitwise_xor(t, torch.div(t, 1 << shift, rounding_mode="floor"))
                    t = torch.remainder(t * factor, 1 << 32)
                return torch.bitwise_xor(t, torch.div(t, 1 << 16, rounding_mode="floor"))

            key = mixed(torch.tensor([(seed + 0x9E3779B9 * (number + 1)) % (1 << 32)], device="cuda"))
            i = torch.arange(z - a, device="cuda")
            draw_of = mixed(torch.remainder(i * 0x9E3779B9 + key, 1 << 32))
            m = _exact_step(m, torch.remainder(draw_of, 1 << 16), 14)
            v = _float32(_exact_step(_float32(torch.sqrt(v)), torch.div(draw_of, 1 << 16, rounding_mode="floor"), 30) ** 2)
        outs["m"].append(m)
        outs["v"].append(v)
    keys = ["param"] + (["master"] if case["master"] else []) + ["m", "v"]
    return tuple(torch.cat(outs[k]) for k in keys)


def _exact_step(x, random16, bias):
    """The representable value next below or above |x|: above with the chance that random16 gives."""
    size = x.abs().view(-1, BLOCK)
    top = size.amax(1, keepdim=True)
    binade = torch.clamp(torch.frexp(top)[1] - 1, min=-90)
    scale = torch.where(top > 0, _power64(binade), torch.zeros_like(top))
    y = torch.where(scale > 0, size / torch.where(scale > 0, scale, torch.ones_like(scale)), torch.zeros_like(size))
    e = torch.where(y > 0, torch.clamp(torch.frexp(y)[1] - 1, min=1 - bias), 1 - bias)
    step = _power64(e - 3)
    below = torch.floor(y / step)
    part = torch.floor((y / step - below) * 2.0 ** 20)         # the digits that the chance goes by
    above = part + 16.0 * random16.view_as(part).double() >= 2.0 ** 20
    value = (below + above.double()) * step * scale
    return (torch.sign(x).view_as(value) * value).flatten()


def exact(case, seed):
    st = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "loss": _exact_loss, "adamw": _exact_adamw}[case["kind"]](case, st)
