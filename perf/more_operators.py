"""Performance cases of the AdamW step over many tensors at once.

Four operators on the parameters, gradients and states of a worker's replica,
K tensors of n_k elements (sync units whole, or the tensors of a layer):

* ``norm``: S = sum of g^2 over all tensors, which clips the gradient (and
  which the shards of a module add up).
* ``step`` with fp32 states: with c = min(1, max_norm / (sqrt(S) + 1e-6)) and
  g' = c g in 32 bits,
      t <- t + 1,   m <- b1 m + (1 - b1) g',   v <- b2 v + (1 - b2) g'^2,
      p <- p - (lr lambda d_k p + lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)),
  d_k the tensor's factor of the weight decay (0 for gains).  A bf16 p is
  rounded to nearest or stochastically: to q floor(|p| / q + u), q the spacing
  of bf16 at p and u 16 random bits over 2^16.
* ``step`` with e4m3 states: m and v in 8 bits, a power of two as the scale of
  every 256 elements of a tensor.  The new m and v, rounded to 32 bits, step p
  and are then rounded stochastically: E = floor(log2) of the largest in the
  block (-119 at least), scale = 2^(E - 7), y = x / scale (v: at least 2^-9),
  q = 2^(max(floor(log2 |y|), -6) - 3), code = sign(y) q floor(|y| / q + u), u 20
  random bits over 2^20.  Nearest would keep v where it is: a step moves it by
  less than half the distance to its neighbours.
* ``pack`` and ``unpack``: fp32 states to e4m3 ones (t = 0 below) and back, as
  a program does at a checkpoint or when it changes over.

The random numbers are a function of the seed, t, the tensor and the element
(_key and _word).  States begin every tensor at a multiple of 256 elements.

The shapes are those of this repository's workloads: layers of the 350M and 1B
models as whole sync units and tensor by tensor, the gains beside them, the
1024 x 1024 linear layer, and ragged ones at odd offsets of a flat buffer.
"""
import torch

own = False  # set by the measuring program: the framework's kernels, or the plain form

BLOCK = 256  # elements that share a scale
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
MAX_NORM, CLIP_EPS = 1.0, 1e-6
STEP, SEED = 1000, 1234  # steps taken before; of the random numbers
HELD = torch.float8_e4m3fn


def _case(name, op, tensors, gains="", layers=1, dtype="bf16", grad="bf16", state="f32", clip=False, stochastic=False):
    """`tensors` of a layer, whose weights decay, and its `gains`, whose do not:
    "n" or "n*count", separated by commas."""
    return {"name": name, "op": op, "tensors": tensors, "gains": gains, "layers": layers, "dtype": dtype, "grad": grad,
            "state": state, "clip": clip, "stochastic": stochastic}


MODULES_350M = "1048576*4,2883584*3"
RAGGED = "100003,1,2049,333333,7,255,1000005,256,65537,511"


def listed():
    return [
        # The gradient norm of a 1B model's 49 gains: a few KB, launches and latency.
        _case("norm-gains-bf16", "norm", "", "2048*49"),
        # The gradient norm of a whole 1B model, 24 sync units.
        _case("norm-1b-bf16", "norm", "51384320*24"),
        # The gains of a 1B model, stepped beside the orthogonalised step of its matrices.
        _case("step-gains-bf16", "step", "", "2048*49"),
        # A 350M model's 216 tensors, fp32, with the clip: an ordinary training step.
        _case("step-350m-modules-f32", "step", MODULES_350M, "1024*2", layers=24, dtype="f32", grad="f32", clip=True),
        # Ragged tensors at odd offsets of a flat bf16 buffer.
        _case("step-ragged-bf16", "step", RAGGED, "1001*3", layers=3, stochastic=True),
        # Part of the 1B model as sync units, bf16 replica and gradients, fp32 states.
        _case("step-1b-bf16", "step", "51384320*6", stochastic=True),
        # The 1024 x 1024 fp32 linear layer, states in 8 bits.
        _case("step8-linear1m-f32", "step", "1048576", dtype="f32", grad="f32", state="e4m3", clip=True),
        # The ragged tensors with states in 8 bits: blocks that end inside every one.
        _case("step8-ragged-bf16", "step", RAGGED, "1001*3", layers=3, state="e4m3", stochastic=True),
        # A 350M model's 216 tensors, fp32 parameters with bf16 gradients, with the clip.
        _case("step8-350m-modules", "step", MODULES_350M, "1024*2", layers=24, dtype="f32", state="e4m3", clip=True),
        # The whole 1B model in bf16, states in 8 bits, with the clip: the largest.
        _case("step8-1b-bf16", "step", "51384320*24", state="e4m3", clip=True, stochastic=True),
        # A 350M model's states change over to 8 bits.
        _case("pack-350m", "pack", "12847104*24", state="e4m3"),
        # Part of a 1B model's states are read for a checkpoint.
        _case("unpack-1b", "unpack", "51384320*6", state="e4m3"),
    ]


def draw(rng):
    op = rng.choice(["norm", "step", "step", "step", "step", "pack", "unpack"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    state = rng.choice(["f32", "e4m3"]) if op in ("norm", "step") else "e4m3"
    total = 2e3 * (4e8 / 2e3) ** rng.random()
    kind = rng.choice(["units", "modules", "ragged"])
    gains, layers = "", 1
    if kind == "units":
        count = rng.randint(1, 24)
        tensors = "%d*%d" % (max(1, int(total / count)), count)
    elif kind == "modules":  # decoder layers with a gated FFN
        layers = rng.randint(1, 24)
        hidden = max(8, int((total / layers / 12) ** 0.5))
        ffn = int(hidden * rng.uniform(2.0, 4.0))
        tensors, gains = "%d*4,%d*3" % (hidden * hidden, hidden * ffn), "%d*2" % hidden
    else:
        sizes = [max(1, int(total / 6 * 10 ** rng.uniform(-3, 0))) for _ in range(rng.randint(2, 40))]
        tensors, gains = ",".join(str(n) for n in sizes), "%d*%d" % (rng.randint(1, 3000), rng.randint(1, 3))
    return {"op": op, "tensors": tensors, "gains": gains, "layers": layers, "dtype": dtype,
            "grad": rng.choice([dtype, "bf16", "f32"]), "state": state, "clip": rng.random() < 0.5,
            "stochastic": dtype == "bf16" and rng.random() < 0.5}


# ------------------------------------------------------------------ inputs


def _sizes(case):
    """Elements and decay factor of every tensor."""
    def parse(text):
        for part in text.split(",") if text else []:
            n, _, count = part.partition("*")
            yield from [int(n)] * int(count or 1)

    layer = [(n, 1.0) for n in parse(case["tensors"])] + [(n, 0.0) for n in parse(case["gains"])]
    return layer * case["layers"]


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _starts(sizes):
    out = [0]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def _in_blocks(x, case):
    """The flat x of all tensors with every tensor padded with zeros to whole blocks."""
    sizes = [n for n, _ in _sizes(case)]
    if all(n % BLOCK == 0 for n in sizes):
        return x
    out = torch.zeros(sum(map(_padded, sizes)), dtype=x.dtype, device=x.device)
    out[_places(sizes)] = x
    return out


def _places(sizes):
    """Where in the padded buffer every element of the flat one is."""
    n = torch.tensor(sizes, device="cuda")
    shift = torch.tensor([b - a for a, b in zip(_starts(sizes), _starts([_padded(k) for k in sizes]))][:-1], device="cuda")
    return torch.arange(sum(sizes), device="cuda") + torch.repeat_interleave(shift, n, output_size=sum(sizes))


def _nearest_held(x):
    """Padded states in 8 bits, rounded to nearest, and their scales: what an earlier step left."""
    x = x.view(-1, BLOCK)
    e = (x.abs().amax(1).view(torch.int32) >> 23).clamp(8, 254)
    scale = ((e - 7) << 23).view(torch.float32)
    return (x / scale[:, None]).to(HELD).view(-1), scale


def _tensors(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    n = sum(k for k, _ in _sizes(case))
    std = 2.0 / max(n, 1) ** 0.5  # a gradient norm of two, of which the clip leaves half

    def noise(scale, t=torch.float32):
        return torch.empty(n, device="cuda").normal_(0.0, scale, generator=gen).to(t)

    s = {"case": case}
    if case["op"] in ("norm", "step"):
        s["grad"] = noise(std, _type(case["grad"]))
    if case["op"] == "norm":
        s["sumsq"] = torch.zeros(1, dtype=torch.float64, device="cuda")
        return s
    if case["op"] == "step":
        s["param"] = noise(0.02, _type(case["dtype"]))
    used = 0.5 * std  # of the gradients that went into the states
    m = _in_blocks(noise(0.3 * used), case)
    v = _in_blocks(noise(1.0).exp_().mul_(used * used), case)
    if case["op"] == "pack" or case["state"] == "f32":
        s["m"], s["v"] = m, v
    if case["op"] == "pack":
        for name in ("held_m", "held_v"):
            s[name] = torch.zeros(m.numel(), dtype=torch.uint8, device="cuda").view(HELD)
            s[name + "_scale"] = torch.zeros(m.numel() // BLOCK, device="cuda")
    elif case["state"] == "e4m3":
        for name, x in (("held_m", m), ("held_v", v)):
            s[name], s[name + "_scale"] = _nearest_held(x)
    if case["op"] == "unpack":
        s["m"], s["v"] = torch.zeros_like(m), torch.zeros_like(v)
    return s


def _views(flat, sizes, starts):
    return [flat[a:a + n] for a, n in zip(starts, sizes)]


def prepare(case, seed):
    s = _tensors(case, seed)
    sizes = [n for n, _ in _sizes(case)]
    if own:
        from paper_2412_07210_amd import AdamW, AdamWConfig, AdamWState

        opt = s["adamw"] = AdamW(AdamWConfig(
            numel=sizes, dtype=case["dtype"], grad_dtype=case["grad"], state=case["state"], betas=(BETA1, BETA2), eps=EPS,
            weight_decay=DECAY, decay=[d for _, d in _sizes(case)], stochastic=case["stochastic"]))
        flat, blocks = _starts(sizes), _starts([_padded(n) for n in sizes])
        if "held_m" in s:
            scales = [_padded(n) // BLOCK for n in sizes]
            state = AdamWState(*[_views(s[k], sizes, blocks) for k in ("held_m", "held_v")],
                               *[_views(s[k], scales, _starts(scales)) for k in ("held_m_scale", "held_v_scale")])
        elif "m" in s:
            state = AdamWState(*[_views(s[k], sizes, blocks) for k in ("m", "v")])
        if case["op"] in ("pack", "unpack"):
            s["state"], s["plain"] = state, [_views(s[k], sizes, blocks) for k in ("m", "v")]
            return s
        grads = _views(s["grad"], sizes, flat)
        if case["op"] == "norm":
            s["plan"] = opt.prepare_grads(grads)
        else:
            opt.state_set(STEP)
            s["plan"] = opt.prepare(_views(s["param"], sizes, flat), grads, state)
        return s
    s["t"] = STEP
    if case["op"] in ("step", "pack"):
        n = torch.tensor(sizes, device="cuda")
        s["tensor"] = torch.repeat_interleave(torch.arange(len(sizes), dtype=torch.int32, device="cuda"), n, output_size=sum(sizes))
        s["start"] = torch.tensor(_starts(sizes)[:-1], device="cuda")
        s["decay"] = torch.tensor([d for _, d in _sizes(case)], device="cuda")
    if case["op"] != "norm":
        s["places"] = None if all(n % BLOCK == 0 for n in sizes) else _places(sizes)
    return s


# ------------------------------------------------------------ random numbers

A64, B64 = 0x6A09E667F3BCC909, 0xBB67AE8584CAA73B  # sqrt(2), sqrt(3), behind the point
M64, M32 = (1 << 64) - 1, (1 << 32) - 1


def _mix(z):
    z = (z & M64) ^ ((z & M64) >> 32)
    z = z * A64 & M64
    z = (z ^ (z >> 29)) * B64 & M64
    return z ^ (z >> 32)


def _key(t, tensor):
    return _mix(_mix(_mix(SEED) + t) + tensor)


def _keys(t, count):
    k = [_key(t, i) for i in range(count)]
    return [torch.tensor(x, device="cuda") for x in ([x & M32 for x in k], [x >> 32 for x in k])]


def _word(element, k0, k1):
    """32 random bits of every element, in int64."""
    k1 = k1 ^ ((element >> 32) * 0xBB67AE85 & M32)
    x = ((element & M32) ^ k0) * 0xBB67AE85 & M32
    x = (x ^ (x >> 17) ^ k1) * 0x6A09E667 & M32
    return x ^ (x >> 15)


def _second(w, k0):
    y = (w + k0) * 0x9E3779B1 & M32
    return y ^ (y >> 15)


def _turned(w):
    return (w << 16 | w >> 16) & M32


# ---------------------------------------------------------------- plain form


def _flat(x, s):
    """Padded states at the places of the tensors' elements."""
    return x if s["places"] is None else x[s["places"]]


def _decoded(s, name):
    x = s[name].float().view(-1, BLOCK) * s[name + "_scale"][:, None]
    return _flat(x.view(-1), s)


def _hold(s, name, x, word, least):
    """x in 8 bits, rounded stochastically, into s[name] and its scales."""
    places, scale = s["places"], s[name + "_scale"]
    top = x.abs()
    if places is not None:
        top = torch.zeros(s[name].numel(), device="cuda").index_copy_(0, places, top)
    e = (top.view(-1, BLOCK).amax(1).view(torch.int32) >> 23).clamp(8, 254)
    scale.copy_(((e - 7) << 23).view(torch.float32))
    by = torch.repeat_interleave(scale.double(), BLOCK)
    y = x.double() / (by if places is None else by[places])
    a = y.abs().clamp_(min=least)
    q = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), torch.frexp(a)[1].clamp_(min=-5) - 4)
    a = (a / q + (word >> 12).double() / 2 ** 20).floor_() * q
    code = a.copysign(y).float().to(HELD)
    if places is None:
        s[name].copy_(code)
    else:
        s[name].view(torch.uint8)[places] = code.view(torch.uint8)


def _words(s, t):
    k0, k1 = _keys(t, s["start"].numel())
    tensor = s["tensor"]
    k0, k1 = k0[tensor], k1[tensor]
    element = torch.arange(tensor.numel(), device="cuda") - s["start"][tensor]
    return _word(element, k0, k1), k0


def _plain_step(s):
    case, p = s["case"], s["param"]
    s["t"] += 1
    t = s["t"]
    g = s["grad"].float()
    if case["clip"]:
        c = (MAX_NORM / (s["grad"].double().square().sum().sqrt() + CLIP_EPS)).clamp(max=1.0).float()
        g = c * g
    held = case["state"] == "e4m3"
    if held:  # next to a border of the 8 bits 32 do not decide
        g = g.double()
        m = (BETA1 * _decoded(s, "held_m").double() + (1.0 - BETA1) * g).float()
        v = (BETA2 * _decoded(s, "held_v").double() + (1.0 - BETA2) * g * g).float()
    else:
        m = BETA1 * _flat(s["m"], s) + (1.0 - BETA1) * g
        v = BETA2 * _flat(s["v"], s) + (1.0 - BETA2) * g * g
    old = p.float()
    update = (LR / (1.0 - BETA1 ** t)) * m / (v.sqrt() * (1.0 - BETA2 ** t) ** -0.5 + EPS)
    new = old - ((LR * DECAY) * s["decay"][s["tensor"]] * old + update)
    if case["stochastic"] or held:
        word, k0 = _words(s, t)
    if case["stochastic"]:
        new = ((new.view(torch.int32) + (_second(word, k0) >> 16).int()) & -65536).view(torch.float32)
    p.copy_(new)
    if held:
        _hold(s, "held_m", m, word, 0.0)
        _hold(s, "held_v", v, _turned(word), 2.0 ** -9)
    elif s["places"] is None:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        s["m"][s["places"]] = m
        s["v"][s["places"]] = v
    return _outputs(s)


def _outputs(s):
    op, held = s["case"]["op"], s["case"]["state"] == "e4m3"
    if op == "norm":
        return {"sumsq": s["sumsq"]}
    names = ["param"] if op == "step" else []
    if op == "unpack" or op == "step" and not held:
        return {k: s[k] for k in names + ["m", "v"]}
    return {k: s[k] for k in names + ["held_m", "held_v", "held_m_scale", "held_v_scale"]}


def _plain_norm(s):
    s["sumsq"].copy_(s["grad"].double().square().sum())
    return _outputs(s)


def _plain_pack(s):
    word, _ = _words(s, 0)
    _hold(s, "held_m", _flat(s["m"], s), word, 0.0)
    _hold(s, "held_v", _flat(s["v"], s), _turned(word), 2.0 ** -9)
    return _outputs(s)


def _plain_unpack(s):
    for to, name in (("m", "held_m"), ("v", "held_v")):
        x = s[name].float().view(-1, BLOCK) * s[name + "_scale"][:, None]
        if s["places"] is None:
            s[to].copy_(x.view(-1))
        else:
            s[to][s["places"]] = x.view(-1)[s["places"]]
    return _outputs(s)


def run(state):
    s, case = state, state["case"]
    if own:
        if case["op"] == "norm":
            s["plan"].sum_squares(s["sumsq"])
        elif case["op"] == "step":
            s["plan"].run(LR, max_norm=MAX_NORM if case["clip"] else None, seed=SEED)
        elif case["op"] == "pack":
            s["adamw"].pack(*s["plain"], s["state"], seed=SEED)
        else:
            s["adamw"].unpack(s["state"], *s["plain"])
        return _outputs(s)
    return {"norm": _plain_norm, "step": _plain_step, "pack": _plain_pack, "unpack": _plain_unpack}[case["op"]](s)


# ------------------------------------------------- what a pass cannot do without


def work(case):
    sizes = [n for n, _ in _sizes(case)]
    n, blocks = sum(sizes), sum(_padded(k) for k in sizes) // BLOCK
    r, rg = (2 if case[k] == "bf16" else 4 for k in ("dtype", "grad"))
    if case["op"] == "norm":
        return {"bytes": rg * n + 8, "flops": 2 * n}
    if case["op"] in ("pack", "unpack"):  # both states in one form and in the other
        return {"bytes": 10 * n + 8 * blocks, "flops": 4 * n}
    states = 16 * n if case["state"] == "f32" else 4 * n + 16 * blocks
    return {"bytes": (2 * r + rg) * n + states, "flops": (16 + 3 * case["clip"]) * n}


# ------------------------------------------------------------ 64-bit reference


def _rounded(a, bits, kept, u):
    """a >= 0 in 64 bits with `kept` bits behind the leading one: those behind them,
    and u of `bits` random ones aligned to the first of them, carry or are cut off."""
    drop = 52 - kept
    return ((a.view(torch.int64) + (u << (drop - bits))) >> drop << drop).view(torch.float64)


def _exact_held(x, sizes, word, least):
    """Values in units of the scale, and the scales, of x in 64 bits, padded."""
    blocks = sum(_padded(n) for n in sizes) // BLOCK
    at = None if all(n % BLOCK == 0 for n in sizes) else _places(sizes)
    full = x if at is None else torch.zeros(blocks * BLOCK, dtype=torch.float64, device="cuda").index_copy_(0, at, x)
    scale = (full.view(-1, BLOCK).abs().amax(1).clamp_(min=2.0 ** -119).view(torch.int64) >> 52 << 52).view(torch.float64) / 128
    y = (full.view(-1, BLOCK) / scale[:, None]).view(-1)
    if at is not None:
        y = y[at]
    a = y.abs().clamp_(min=least)
    small = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0).double()  # below it the spacing is that of its neighbours above
    a = (_rounded(a + small, 20, 3, word >> 12) - small).copysign_(y)
    if at is not None:
        a = torch.zeros(blocks * BLOCK, dtype=torch.float64, device="cuda").index_copy_(0, at, a)
    return a, scale


def _exact_words(sizes, t):
    n, at, out, keys = sum(sizes), 0, [], []
    for i, size in enumerate(sizes):
        k = _key(t, i)
        x = torch.arange(size, device="cuda")
        hi = (x >> 32) * 0xBB67AE85 & M32
        x = (x & M32 ^ (k & M32)) * 0xBB67AE85 & M32
        x ^= (x >> 17) ^ (k >> 32) ^ hi
        x = x * 0x6A09E667 & M32
        out.append(x ^ (x >> 15))
        keys.append(k & M32)
        at += size
    assert at == n
    return out, keys


def exact(case, seed):
    s = _tensors(case, seed)
    sizes = [n for n, _ in _sizes(case)]
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(s["grad"], dtype=torch.float64)
        return {"sumsq": (norm * norm).view(1)}
    at = None if all(n % BLOCK == 0 for n in sizes) else _places(sizes)

    def states(name):
        x = s[name].double()
        if held:
            x = (x.view(-1, BLOCK) * s[name + "_scale"].double()[:, None]).view(-1)
        return x if at is None else x[at]

    held = case["state"] == "e4m3"
    if case["op"] == "unpack":
        return {k: (s["held_" + k].double().view(-1, BLOCK) * s["held_" + k + "_scale"].double()[:, None]).view(-1) for k in "mv"}
    if case["op"] == "pack":
        word = torch.cat(_exact_words(sizes, 0)[0])
        m, v = ((x if at is None else x[at]) for x in (s["m"].double(), s["v"].double()))
        out = {}
    else:
        t = STEP + 1
        g = s["grad"].double()
        if case["clip"]:
            g *= min(1.0, MAX_NORM / (float(torch.linalg.vector_norm(g)) + CLIP_EPS))
        m = states("held_m" if held else "m").mul_(BETA1).add_(g, alpha=1.0 - BETA1)
        v = states("held_v" if held else "v").mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
        p = s["param"].double()
        step = (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt_() + EPS)
        decay = torch.cat([torch.full((n,), 1.0 - LR * DECAY * d, dtype=torch.float64, device="cuda") for n, d in _sizes(case)])
        p.mul_(decay).sub_(step, alpha=LR)
        del step, decay
        if case["stochastic"] or held:
            words, keys = _exact_words(sizes, t)
        if case["stochastic"]:
            u = torch.cat([(lambda y: (y ^ (y >> 15)) >> 16)((w + k) * 0x9E3779B1 & M32) for w, k in zip(words, keys)])
            p = _rounded(p.abs(), 16, 7, u).copysign_(p)
        out = {"param": p}
        if not held:
            pad = (lambda x: x) if at is None else (
                lambda x: torch.zeros(s["m"].numel(), dtype=torch.float64, device="cuda").index_copy_(0, at, x))
            return {**out, "m": pad(m), "v": pad(v)}
        word = torch.cat(words)
        m, v = m.float().double(), v.float().double()  # as defined; sums of few bits lie on powers of two, next to them without it
    out["held_m"], out["held_m_scale"] = _exact_held(m, sizes, word, 0.0)
    out["held_v"], out["held_v_scale"] = _exact_held(v, sizes, (word << 16 | word >> 16) & M32, 2.0 ** -9)
    return out
