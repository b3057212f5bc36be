"""Performance cases of the orthogonalised updates.

Three operators on the flat sync units of this framework, whose matrices are
named by (offset, rows, cols):

* ``orthogonalize``: every matrix of an update U becomes the fifth
  Newton-Schulz iterate of U / ||U||_F,
      A = X X^T,  X <- a X + (b A + c A^2) X,
  a, b, c = 3.4445, -4.7750, 2.0315 (with X^T where there are more rows than
  columns), which brings its singular values near one.
* ``local_step``: one inner step of a worker on its replica,
      m <- mu m + g,  u = g + mu m,  p <- (1 - eta lambda) p - eta s O(u),
  s = 0.2 sqrt(max(rows, cols)); elements of no matrix stay as they are.
* ``outer_step``: the outer step of a unit (norms, z-test, weights, clip as in
  the plain outer step) whose Nesterov update is orthogonalised,
      b <- rho b - D,  u = rho b - D,  theta <- theta - nu s O(u),
  D the clipped weighted average; elements of no matrix take the plain
  Nesterov update; every replica is set to theta.

The shapes are those of this repository's workloads: Llama-style layers of
the 350M and 1B models, a 7B matrix, the 1024 x 1024 linear layer, and ragged
ones.  Gradients are a rank of 16 over noise, as those of a matrix are;
pseudo gradients are noise of the workers' own scales, as in the other cases.
The replicas of the outer cases are fp32: a second step right after the first
has no pseudo gradient then, where with bf16 replicas it would step along the
rounding errors of theta, which no two orders of summation agree on.
"""
import torch

own = False  # set by the measuring program: the framework's kernels, or the plain form

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
LR, MU, DECAY = 2e-3, 0.95, 0.1        # inner step
NU, RHO, CLIP, CLIP_EPS = 1e-3, 0.85, 10.0, 1e-6  # outer step
ALPHA, Z, WARMUP = 0.02, 3.0, 10


def _case(name, op, dtype, matrices, vectors=0, k=0, anomalous=0):
    """`matrices`: "rowsxcols" or "rowsxcols*count", separated by commas;
    `vectors`: elements behind them that belong to no matrix (gains)."""
    return {"name": name, "op": op, "dtype": dtype, "matrices": matrices, "vectors": vectors,
            "k": k, "anomalous": anomalous}


LAYER_350M = "1024x1024*4,2816x1024*2,1024x2816"
LAYER_1B = "2048x2048*4,5632x2048*2,2048x5632"


def listed():
    return [
        # One small matrix (a projection of a head): launches and latency.
        _case("orth-128-bf16", "orthogonalize", "bf16", "128x128"),
        # The 1024 x 1024 fp32 linear layer's update.
        _case("orth-linear1m-f32", "orthogonalize", "f32", "1024x1024"),
        # The update of one 350M decoder layer: four attention matrices, three of the FFN.
        _case("orth-350m-bf16", "orthogonalize", "bf16", LAYER_350M),
        # Ragged matrices at odd offsets, wide and tall ones in one unit.
        _case("orth-ragged-bf16", "orthogonalize", "bf16", "1001x1537,2049x517,333x333,67x1999"),
        # The FFN matrix of a 7B layer: the largest matrix, stored tall.
        _case("orth-7b-ffn-bf16", "orthogonalize", "bf16", "11008x4096"),
        # An inner step on a layer of a small model, with its gains: a few short launches.
        _case("local-small-bf16", "local_step", "bf16", "256x256*4,688x256*2,256x688", vectors=512),
        # An inner step on a 350M layer whose replica is fp32.
        _case("local-350m-f32", "local_step", "f32", LAYER_350M, vectors=2048),
        # An inner step on a 1B layer, bf16 replica.
        _case("local-1b-bf16", "local_step", "bf16", LAYER_1B, vectors=4096),
        # The 1024 x 1024 linear layer with four workers, one of them anomalous.
        _case("outer-linear1m-k4-f32", "outer_step", "f32", "1024x1024", k=4, anomalous=1),
        # The outer step of a 350M layer, eight workers.
        _case("outer-350m-k8-f32", "outer_step", "f32", LAYER_350M, vectors=2048, k=8),
        # The outer step of a 1B layer, eight workers, one of them anomalous.
        _case("outer-1b-k8-f32", "outer_step", "f32", LAYER_1B, vectors=4096, k=8, anomalous=1),
    ]


def draw(rng):
    op = rng.choice(["orthogonalize", "orthogonalize", "local_step", "local_step", "outer_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"]) if op != "outer_step" else "f32"
    k = rng.choice([2, 3, 4, 5, 8, 8, 16]) if op == "outer_step" else 0
    most = 6.0e11 if op == "orthogonalize" else 4.0e11  # multiply-adds of the plain products, of 2.2e12 listed
    hidden = int(32 * (4096 / 32) ** rng.random())
    kind = rng.choice(["square", "layer", "ragged", "ragged"])
    if kind == "square":
        parts = [(hidden, hidden, rng.randint(1, 6))]
    elif kind == "layer":  # a decoder layer with a gated FFN
        ffn = int(hidden * rng.uniform(2.0, 4.0))
        parts = [(hidden, hidden, 4), (ffn, hidden, 2), (hidden, ffn, 1)]
    else:
        parts = []
        for _ in range(rng.randint(1, 4)):
            a, b = int(24 * (3000 / 24) ** rng.random()), int(24 * (8000 / 24) ** rng.random())
            parts.append((a, b, 1))
    # the most matrices that stay within the largest listed case's work
    kept, spent = [], 0.0
    for rows, cols, count in parts:
        short, long = min(rows, cols), max(rows, cols)
        each = STEPS * (2.0 * short * short * long + short ** 3)
        fit = min(count, int((most - spent) / each))
        if fit > 0:
            kept.append((rows, cols, fit))
            spent += fit * each
    if not kept:
        kept = [(min(parts[0][0], 1024), min(parts[0][1], 2048), 1)]
    matrices = ",".join("%dx%d*%d" % p if p[2] > 1 else "%dx%d" % p[:2] for p in kept)
    vectors = 0 if op == "orthogonalize" else rng.choice([0, 2 * hidden, 2 * hidden + 1])
    anomalous = rng.choice([0, 1]) if k >= 4 else 0
    return {"op": op, "dtype": dtype, "matrices": matrices, "vectors": vectors, "k": k, "anomalous": anomalous}


# ------------------------------------------------------------------ inputs


def _groups(case):
    """(offset, count, rows, cols) of each run of equal matrices, and the unit's length."""
    out, at = [], 0
    for part in case["matrices"].split(","):
        shape, _, count = part.partition("*")
        rows, cols = (int(x) for x in shape.split("x"))
        out.append((at, int(count or 1), rows, cols))
        at += out[-1][1] * rows * cols
    return out, at + case["vectors"]


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gradient(case, gen, std):
    """A unit's gradient: a rank of 16 over noise in every matrix."""
    groups, n = _groups(case)
    g = torch.empty(n, device="cuda").normal_(0.0, std, generator=gen)
    for at, count, rows, cols in groups:
        left = torch.empty(count, rows, 16, device="cuda").normal_(0.0, std, generator=gen)
        right = torch.empty(count, 16, cols, device="cuda").normal_(0.0, 1.0, generator=gen)
        g[at:at + count * rows * cols] += (left @ right).view(-1)
    return g


def _tensors(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))
    _, n = _groups(case)
    t = _type(case)
    s = {"case": case}
    if case["op"] == "orthogonalize":
        s["x"] = _gradient(case, gen, 1e-3).to(t)
        s["out"] = torch.zeros_like(s["x"])
        return s
    theta = torch.empty(n, device="cuda").normal_(0.0, 0.02, generator=gen)
    if case["op"] == "local_step":
        s["param"] = theta.to(t)
        s["grad"] = _gradient(case, gen, 1e-3).to(t)
        s["momentum"] = _gradient(case, gen, 5e-3)
        return s
    k = case["k"]
    std = (1e-3 * (0.5 + 1.5 * torch.rand(k, generator=host, dtype=torch.float64))).tolist()
    for j in range(k - case["anomalous"], k):
        std[j] *= 20.0
    s["theta"] = theta
    s["momentum"] = torch.empty(n, device="cuda").normal_(0.0, 1e-3, generator=gen)
    s["replicas"] = [torch.empty(n, device="cuda").normal_(0.0, x, generator=gen).add_(theta).to(t) for x in std]
    norms = [float((r.double() - theta.double()).square().sum().sqrt()) for r in s["replicas"]]
    # the EMA pair of every worker after a run whose norms were steady
    mean = [g / (20.0 if j >= k - case["anomalous"] else 1.0) for j, g in enumerate(norms)]
    s["ema"] = torch.tensor([mean, [0.1 * m for m in mean]], dtype=torch.float64, device="cuda")
    return s


def prepare(case, seed):
    s = _tensors(case, seed)
    if own:
        from paper_2412_07210_amd import EditOuter, OrthoConfig, Orthogonalizer, OuterConfig

        groups, n = _groups(case)
        matrices = [(at + i * rows * cols, rows, cols) for at, count, rows, cols in groups for i in range(count)]
        # theta is fp32 in the outer step, whatever the replicas are
        s["ortho"] = Orthogonalizer(OrthoConfig(
            numel=n, matrices=matrices, dtype="f32" if case["op"] == "outer_step" else case["dtype"], scale="rms"))
        if case["op"] == "outer_step":
            s["handle"] = EditOuter(OuterConfig(
                num_workers=case["k"], layer_numel=[n], replica_dtype=case["dtype"], outer_lr=NU, momentum=RHO,
                clip_threshold=CLIP, clip_eps=CLIP_EPS, ema_alpha=ALPHA, z_threshold=Z, ema_warmup_rounds=WARMUP))
            s["handle"].state_set(0, s["ema"][0].tolist(), s["ema"][1].tolist(), WARMUP)
    return s


# ---------------------------------------------------------------- plain form


def _iterate(x):
    """The Newton-Schulz iterate of a batch of matrices, in 32 bits."""
    a, b, c = COEFFICIENTS
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    norm = x.double().square().sum(dim=(1, 2), keepdim=True).sqrt()
    x = x / torch.where(norm > 0, norm, torch.ones_like(norm)).float()
    for _ in range(STEPS):
        g = x @ x.transpose(1, 2)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.transpose(1, 2) if tall else x


def _each(case, u, write):
    """write(slice, scale, iterate as a flat tensor) for each run of equal matrices of the fp32 unit u."""
    for at, count, rows, cols in _groups(case)[0]:
        part = slice(at, at + count * rows * cols)
        write(part, 0.2 * max(rows, cols) ** 0.5, _iterate(u[part].view(count, rows, cols)).reshape(-1))


def _plain_orthogonalize(s):
    x, out = s["x"], s["out"]

    def write(part, scale, o):
        out[part] = o.to(out.dtype)

    _each(s["case"], x.float(), write)
    return {"out": out}


def _plain_local_step(s):
    p, m = s["param"], s["momentum"]
    end = p.numel() - s["case"]["vectors"]
    g = s["grad"][:end].float()
    m[:end] = MU * m[:end] + g
    u = g + MU * m[:end]

    def write(part, scale, o):
        p[part] = ((1.0 - LR * DECAY) * p[part].float() - (LR * scale) * o).to(p.dtype)

    _each(s["case"], u, write)
    return {"param": p, "momentum": m}


def _plain_outer_step(s):
    theta, b, replicas, (mean, std) = s["theta"], s["momentum"], s["replicas"], s["ema"]
    deltas = [r.float() - theta for r in replicas]
    norms = torch.stack([d.double().square().sum().sqrt() for d in deltas])
    keep = norms - mean <= Z * std
    # the EMA of the workers that passed (Eq. 1)
    new = ALPHA * norms + (1.0 - ALPHA) * mean
    spread = ((1.0 - ALPHA) * std * std + ALPHA * (norms - new) ** 2).sqrt()
    s["ema"] = torch.where(keep, torch.stack([new, spread]), s["ema"])
    w = torch.softmax(torch.where(keep, -norms, torch.full_like(norms, -torch.inf)), 0).float()
    d = torch.zeros_like(theta)
    for wj, x in zip(w, deltas):
        d += torch.where(wj > 0, wj * x, torch.zeros_like(x))
    del deltas
    beta = (CLIP / (d.double().square().sum().sqrt() + CLIP_EPS)).clamp(max=1.0).float()
    d *= beta
    b.mul_(RHO).sub_(d)
    u = RHO * b - d
    end = theta.numel() - s["case"]["vectors"]
    theta[end:] -= NU * u[end:]

    def write(part, scale, o):
        theta[part] -= (NU * scale) * o

    _each(s["case"], u, write)
    for r in replicas:
        r.copy_(theta)
    return {"theta": theta, "momentum": b, "replicas": list(replicas)}


def run(state):
    op = state["case"]["op"]
    if own:
        s = state
        if op == "orthogonalize":
            s["ortho"].orthogonalize(s["x"], s["out"])
            return {"out": s["out"]}
        if op == "local_step":
            s["ortho"].local_step(s["param"], s["grad"], s["momentum"], lr=LR, mu=MU, weight_decay=DECAY)
            return {"param": s["param"], "momentum": s["momentum"]}
        s["handle"].step_layer_ortho(0, s["ortho"], s["theta"], s["momentum"], s["replicas"])
        return {"theta": s["theta"], "momentum": s["momentum"], "replicas": list(s["replicas"])}
    return {"orthogonalize": _plain_orthogonalize, "local_step": _plain_local_step,
            "outer_step": _plain_outer_step}[op](state)


# ------------------------------------------------- what a pass cannot do without


def work(case):
    groups, n = _groups(case)
    r = 2 if case["dtype"] == "bf16" else 4
    flops = 0.0
    for _, count, rows, cols in groups:
        short, long = min(rows, cols), max(rows, cols)
        # X X^T and A^2 are symmetric: half of each; then the product with X
        flops += count * STEPS * (short * (short + 1.0) * (long + short) + 2.0 * short * short * long)
    if case["op"] == "orthogonalize":
        return {"bytes": 2 * r * n, "flops": flops}
    m = n - case["vectors"]
    if case["op"] == "local_step":  # param and momentum both ways, the gradient in
        return {"bytes": (3 * r + 8) * m, "flops": flops + 8 * m}
    k = case["k"]
    # theta, the momentum and every replica once each way
    return {"bytes": (16 + 2 * k * r) * n, "flops": flops + (k + k * (k + 1) + 3 * k + 6) * n}


# ------------------------------------------------------------ 64-bit reference


def _polynomial(u, rows, cols):
    """The iterate of one matrix by X <- (a I + (b I + c A) A) X in 64 bits."""
    a, b, c = COEFFICIENTS
    x = u.double().view(rows, cols)
    if rows > cols:
        x = x.t().contiguous()
    size = float(torch.linalg.vector_norm(x))
    if size > 0:
        x = x / size
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        g = torch.mm(x, x.t())
        x = torch.mm(a * eye + torch.mm(b * eye + c * g, g), x)
    return (x.t() if rows > cols else x).reshape(-1)


def _matrices(case):
    for at, count, rows, cols in _groups(case)[0]:
        for i in range(count):
            yield slice(at + i * rows * cols, at + (i + 1) * rows * cols), rows, cols


def exact(case, seed):
    s = _tensors(case, seed)
    if case["op"] == "orthogonalize":
        out = s["out"].double()
        for part, rows, cols in _matrices(case):
            out[part] = _polynomial(s["x"][part], rows, cols)
        return {"out": out}
    if case["op"] == "local_step":
        p, m = s["param"].double(), s["momentum"].double()
        for part, rows, cols in _matrices(case):
            g = s["grad"][part].double()
            m[part] = MU * m[part] + g
            o = _polynomial(g + MU * m[part], rows, cols)
            p[part] = p[part] - LR * DECAY * p[part] - LR * 0.2 * max(rows, cols) ** 0.5 * o
        return {"param": p, "momentum": m}
    theta = s["theta"].double()
    mean, std = s["ema"].tolist()
    norms = [float(torch.linalg.vector_norm(r.double() - theta)) for r in s["replicas"]]
    good = [j for j, g in enumerate(norms) if not g - mean[j] > Z * std[j]]
    least = min(norms[j] for j in good)
    w = {j: torch.exp(torch.tensor(least - norms[j], dtype=torch.float64)).item() for j in good}
    total = sum(w.values())
    d = torch.zeros_like(theta)
    for j in good:
        d += (w[j] / total) * (s["replicas"][j].double() - theta)
    d *= min(CLIP / (float(torch.linalg.vector_norm(d)) + CLIP_EPS), 1.0)
    b = RHO * s["momentum"].double() - d
    u = RHO * b - d
    new = theta - NU * u
    for part, rows, cols in _matrices(case):
        new[part] = theta[part] - NU * 0.2 * max(rows, cols) ** 0.5 * _polynomial(u[part], rows, cols)
    return {"theta": new, "momentum": b, "replicas": [new] * case["k"]}
