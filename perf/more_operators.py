"""Measured cases of the operators at the two ends of a language model's training step and behind
the exchange of its gradients: the embedding of tokens and its gradient, the cross entropy of a
linear output layer over a large vocabulary and its gradient, and the orthogonalised update of a
weight matrix.

`own` False: plain torch operations in 32 bits, rounded once at the end.  `own` True: the calls
of this package.  Both take what prepare() gives."""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)     # of the odd polynomial that a step applies
EPS = 1e-7


# ---- cases ---------------------------------------------------------------------------------

def listed():
    return [
        # the next token of one answer: latency
        dict(name="embed-token", op="embed", rows=1, cols=4096, vocabulary=65536, dtype="bf16",
             out="bf16", padded=0.0),
        # a micro-batch of 16 K tokens with padding, rows scaled by the root of the width
        dict(name="embed-batch", op="embed", rows=16384, cols=4096, vocabulary=65536,
             dtype="bf16", out="bf16", padded=0.125),
        # one sequence of a small model, gradient in binary32 as the compressors read it
        dict(name="embed-grad-small", op="embed_grad", rows=512, cols=768, vocabulary=8192,
             dtype="bf16", out="f32", padded=0.0),
        # the micro-batch above: few tokens take most places, most rows of the table get none
        dict(name="embed-grad-large", op="embed_grad", rows=16384, cols=4096, vocabulary=65536,
             dtype="bf16", out="bf16", padded=0.125),
        # an odd width, tokens and vocabulary that nothing divides
        dict(name="embed-grad-odd", op="embed_grad", rows=8191, cols=1001, vocabulary=32001,
             dtype="f16", out="f32", padded=0.0),
        # scoring one short answer
        dict(name="loss-small", op="loss", rows=87, width=768, vocabulary=8192, dtype="f16",
             ignored=0.0),
        # a validation batch; a quarter of the tokens (the questions) has no target
        dict(name="loss-large", op="loss", rows=8192, width=2048, vocabulary=65536, dtype="bf16",
             ignored=0.25),
        # a ragged batch of a small model, odd in all sizes, with a penalty on the normaliser
        dict(name="loss-grad-odd", op="loss_grad", rows=515, width=1001, vocabulary=8193,
             dtype="f16", ignored=0.1, penalty=True),
        # the training step of a 4096-wide model over 64 K tokens of vocabulary
        dict(name="loss-grad-large", op="loss_grad", rows=8192, width=4096, vocabulary=65536,
             dtype="bf16", ignored=0.0, penalty=False),
        # the update of the first layer of a small feed-forward block, as it was aggregated
        dict(name="update-small", op="update", batch=1, rows=2048, cols=512, dtype="f32"),
        # several matrices of one shape that no tile divides
        dict(name="update-odd", op="update", batch=4, rows=777, cols=1001, dtype="f32"),
        # a 4096-wide projection
        dict(name="update-large", op="update", batch=1, rows=4096, cols=4096, dtype="bf16"),
    ]


def _size(rng, low, high):
    """A size spread over the logarithm of its range; one in three is a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 0.34:
        v = max(64, v // 64 * 64)
    return min(max(v, low), high)


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "loss", "loss_grad", "update"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "embed_grad"):
        cols = _size(rng, 64, 8192)
        rows = _size(rng, 1, min(65536, 16384 * 4096 // cols))
        vocabulary = _size(rng, 256, min(262144, 65536 * 4096 // cols))
        out = rng.choice([dtype, "f32"]) if op == "embed_grad" else rng.choice([dtype, "bf16"])
        if "f32" in (dtype, out):
            rows, vocabulary = max(1, rows // 2), max(256, vocabulary // 2)
        return dict(op=op, rows=rows, cols=cols, vocabulary=vocabulary, dtype=dtype, out=out,
                    padded=rng.choice([0.0, 0.3]))
    if op == "update":
        rows, cols = _size(rng, 32, 4096), _size(rng, 32, 4096)
        batch = min(rng.choice([1, 1, 2, 5]),
                    max(1, 4096 ** 3 // (rows * cols * min(rows, cols))))
        return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=dtype)
    width = _size(rng, 64, 4096)
    rows = _size(rng, 1, 16384)
    vocabulary = _size(rng, 256, 131072)
    most = 8192 * 2048 * 65536 if op == "loss" else 8192 * 4096 * 65536
    while rows * width * vocabulary > most:
        rows = rows // 2 + 1
    c = dict(op=op, rows=rows, width=width, vocabulary=vocabulary,
             dtype=rng.choice(["bf16", "bf16", "f16"]), ignored=rng.choice([0.0, 0.4]))
    if op == "loss_grad":
        c["penalty"] = rng.random() < 0.3
    return c


def work(case):
    c = case
    if c["op"] == "embed":          # a row of the table or none, and a row of the output
        m = c["rows"] * c["cols"]
        read = (1 - c["padded"]) * m * DTYPES[c["dtype"]].itemsize
        return {"bytes": read + m * DTYPES[c["out"]].itemsize + 8 * c["rows"], "flops": m}
    if c["op"] == "embed_grad":
        m = (1 - c["padded"]) * c["rows"] * c["cols"]
        b = m * DTYPES[c["dtype"]].itemsize + 8 * c["rows"]
        return {"bytes": b + c["vocabulary"] * c["cols"] * DTYPES[c["out"]].itemsize, "flops": m}
    if c["op"] == "update":         # by the shorter side s: s s l and s s s and s s l a step
        short, long = sorted((c["rows"], c["cols"]))
        m = c["batch"] * short * long
        # (the first two products are symmetric: half of each is enough)
        return {"bytes": m * (DTYPES[c["dtype"]].itemsize + 2),
                "flops": STEPS * c["batch"] * short * short * (3 * long + short)}
    t, d, v = (1 - c["ignored"]) * c["rows"], c["width"], c["vocabulary"]
    if c["op"] == "loss":
        return {"bytes": 2 * (t + v) * d + 16 * c["rows"], "flops": 2 * t * d * v}
    return {"bytes": 4 * (c["rows"] + v) * d + 16 * c["rows"], "flops": 6 * t * d * v}


# ---- inputs --------------------------------------------------------------------------------

def _tokens(count, vocabulary, padded, g, dev):
    """Tokens as text has them: the k-th most frequent one about 1 / k times as often as the first,
    at places of the vocabulary that have nothing to do with it; padding is negative."""
    u = torch.rand(count, generator=g, device=dev, dtype=torch.float64)
    k = (torch.exp(u * math.log(vocabulary + 1)) - 1).long().clamp(0, vocabulary - 1)
    t = torch.randperm(vocabulary, generator=g, device=dev)[k]
    if padded:
        t[torch.rand(count, generator=g, device=dev) < padded] = -1
    return t


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    s = {"case": c}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    if c["op"] in ("embed", "embed_grad"):
        s["tokens"] = _tokens(c["rows"], c["vocabulary"], c["padded"], g, dev)
        s["scale"] = math.sqrt(c["cols"])
        if c["op"] == "embed":
            s["table"] = (0.02 * normal(c["vocabulary"], c["cols"])).to(DTYPES[c["dtype"]])
        else:
            s["dy"] = (1e-3 * normal(c["rows"], c["cols"])).to(DTYPES[c["dtype"]])
        return s
    if c["op"] == "update":
        # a few directions carry most of a gradient, the rest is noise
        rank = max(1, min(c["rows"], c["cols"]) // 2)
        fall = torch.arange(1, rank + 1, device=dev) ** -0.5
        x = normal(c["batch"], c["rows"], rank) * fall @ normal(c["batch"], rank, c["cols"])
        x = 1e-3 * (x + normal(c["batch"], c["rows"], c["cols"]))
        s["g"] = x.to(DTYPES[c["dtype"]])
        s["scale"] = math.sqrt(max(1.0, c["rows"] / c["cols"]))
        return s
    t, d, v, dt = c["rows"], c["width"], c["vocabulary"], DTYPES[c["dtype"]]
    s["table"] = (2.5 / math.sqrt(d) * normal(v, d)).to(dt)
    s["targets"] = _tokens(t, v, 0.0, g, dev)
    # normalised rows that lean towards their target, some far, some not at all
    lean = 4 * torch.rand(t, 1, generator=g, device=dev)
    s["x"] = (normal(t, d) + lean / 2.5 * s["table"][s["targets"]].float()).to(dt)
    s["targets"][torch.rand(t, generator=g, device=dev) < c["ignored"]] = -1
    s["scale"] = 1.0
    if c["op"] == "loss_grad":      # what the forward pass has left, and the loss's own gradient
        counts = s["targets"] >= 0
        w = s["table"].float()
        s["lse"] = torch.cat([torch.logsumexp(x.float() @ w.t(), 1) for x in s["x"].split(2048)])
        s["lse"] = torch.where(counts, s["lse"], 0.0)
        s["dloss"] = counts.float() / counts.sum().clamp(min=1)
        if c["penalty"]:            # the mean of 1e-4 lse^2
            s["dlse"] = 2e-4 * s["lse"] * s["dloss"]
    return s


# ---- plain forms ---------------------------------------------------------------------------

def _plain(s):
    c = s["case"]
    if c["op"] == "embed":
        t = s["tokens"].unsqueeze(1)
        rows = s["scale"] * s["table"][s["tokens"].clamp(min=0)].float()
        return {"out": torch.where(t < 0, 0.0, rows).to(DTYPES[c["out"]])}
    if c["op"] == "embed_grad":
        there = (s["tokens"] >= 0).unsqueeze(1)
        dy = torch.where(there, s["scale"] * s["dy"].float(), 0.0)
        dt = torch.zeros(c["vocabulary"], c["cols"], device=dy.device)
        dt.index_add_(0, s["tokens"].clamp(min=0), dy)
        return {"dtable": dt.to(DTYPES[c["out"]])}
    if c["op"] == "update":
        a, b, f = COEFFICIENTS
        x = s["g"].float()
        wide = c["rows"] <= c["cols"]
        x = x if wide else x.transpose(1, 2)
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(STEPS):
            y = x @ x.transpose(1, 2)
            x = a * x + (b * y + f * (y @ y)) @ x
        x = s["scale"] * (x if wide else x.transpose(1, 2))
        return {"out": x.bfloat16()}
    w, x = s["table"].float(), s["x"].float()
    logits = s["scale"] * (x @ w.t())
    counts = s["targets"] >= 0
    at = s["targets"].clamp(min=0).unsqueeze(1)
    if c["op"] == "loss":
        top = logits.amax(1, keepdim=True)
        hit = logits.gather(1, at).squeeze(1)
        lse = logits.sub_(top).exp_().sum(1).log() + top.squeeze(1)
        return {"loss": torch.where(counts, lse - hit, 0.0), "lse": torch.where(counts, lse, 0.0)}
    both = s["dloss"] + s["dlse"] if c["penalty"] else s["dloss"]
    d = logits.sub_(s["lse"].unsqueeze(1)).exp_().mul_(both.unsqueeze(1))
    d.scatter_add_(1, at, -s["dloss"].unsqueeze(1))
    d.masked_fill_(~counts.unsqueeze(1), 0.0)
    dt = DTYPES[c["dtype"]]
    return {"dx": (s["scale"] * (d @ w)).to(dt), "dtable": (s["scale"] * (d.t() @ x)).to(dt)}


# ---- the package's calls -------------------------------------------------------------------

def _kernels(s):
    import paper_1905_10988_b200 as nc
    c = s["case"]
    code = {"f32": nc.DTYPE_F32, "bf16": nc.DTYPE_BF16, "f16": nc.DTYPE_F16}
    if "out" not in s:           # buffers that a training loop keeps from step to step
        s["out"] = _buffers(nc, s)
    o = s["out"]
    if c["op"] == "embed":
        nc.nc_embedding_forward(s["tokens"], 8, c["rows"], s["table"], code[c["dtype"]],
                                c["vocabulary"], c["cols"], c["cols"], s["scale"], o["out"],
                                code[c["out"]], c["cols"])
        return {"out": o["out"]}
    if c["op"] == "embed_grad":
        nc.nc_embedding_backward(s["tokens"], 8, c["rows"], s["dy"], code[c["dtype"]], c["cols"],
                                 c["cols"], s["scale"], c["vocabulary"], o["dtable"],
                                 code[c["out"]], c["cols"], False, o["ws"], o["ws_bytes"])
        return {"dtable": o["dtable"]}
    if c["op"] == "update":
        m = c["rows"] * c["cols"]
        nc.nc_orthogonalize(s["g"], code[c["dtype"]], c["batch"], c["rows"], c["cols"], c["cols"],
                            m, COEFFICIENTS * STEPS, STEPS, EPS, s["scale"], o["out"],
                            nc.DTYPE_BF16, c["cols"], m, o["ws"], o["ws_bytes"])
        return {"out": o["out"]}
    t, d, v, dt = c["rows"], c["width"], c["vocabulary"], code[c["dtype"]]
    if c["op"] == "loss":
        nc.nc_linear_cross_entropy_forward(s["x"], dt, t, d, d, s["table"], v, d, s["targets"], 8,
                                           s["scale"], o["loss"], o["lse"], o["ws"],
                                           o["ws_bytes"])
        return {"loss": o["loss"], "lse": o["lse"]}
    nc.nc_linear_cross_entropy_backward(s["x"], dt, t, d, d, s["table"], v, d, s["targets"], 8,
                                        s["scale"], s["lse"], s["dloss"], s.get("dlse"), o["dx"],
                                        d, o["dtable"], dt, d, False, o["ws"], o["ws_bytes"])
    return {"dx": o["dx"], "dtable": o["dtable"]}


def _buffers(nc, s):
    c, dev = s["case"], "cuda"
    if c["op"] == "embed":
        return {"out": torch.empty(c["rows"], c["cols"], dtype=DTYPES[c["out"]], device=dev)}
    if c["op"] == "embed_grad":
        b = nc.nc_embedding_backward_workspace_bytes(c["rows"], c["vocabulary"], c["cols"])
        o = {"dtable": torch.empty(c["vocabulary"], c["cols"], dtype=DTYPES[c["out"]], device=dev)}
    elif c["op"] == "update":
        b = nc.nc_orthogonalize_workspace_bytes(c["batch"], c["rows"], c["cols"])
        o = {"out": torch.empty(c["batch"], c["rows"], c["cols"], dtype=torch.bfloat16,
                                device=dev)}
    elif c["op"] == "loss":
        b = nc.nc_linear_cross_entropy_forward_workspace_bytes(c["rows"], c["width"],
                                                               c["vocabulary"])
        f32 = dict(dtype=torch.float32, device=dev)
        o = {"loss": torch.empty(c["rows"], **f32), "lse": torch.empty(c["rows"], **f32)}
    else:
        b = nc.nc_linear_cross_entropy_backward_workspace_bytes(c["rows"], c["width"],
                                                                c["vocabulary"])
        o = {"dx": torch.empty_like(s["x"]), "dtable": torch.empty_like(s["table"])}
    return {**o, "ws": torch.empty(b, dtype=torch.uint8, device=dev), "ws_bytes": b}


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "embed":
        out = s["scale"] * s["table"].double().index_select(0, s["tokens"].clamp(min=0))
        return {"out": out * (s["tokens"] >= 0).double()[:, None]}
    if c["op"] == "embed_grad":
        # sums over the runs of equal tokens in sorted order, by differences of running sums
        keep = (s["tokens"] >= 0).nonzero().reshape(-1)
        t, order = torch.sort(s["tokens"][keep], stable=True)
        out = torch.zeros(c["vocabulary"], c["cols"], dtype=torch.float64, device=t.device)
        if t.numel() == 0:
            return {"dtable": out}
        ids, n = torch.unique_consecutive(t, return_counts=True)
        ends = n.cumsum(0)
        for at in range(0, c["cols"], 512):
            run_sum = s["dy"][keep[order], at:at + 512].double().cumsum(0)
            got = run_sum[ends - 1]
            got[1:] -= run_sum[ends[:-1] - 1]
            out[ids, at:at + 512] = s["scale"] * got
        return {"dtable": out}
    if c["op"] == "update":
        a, b, f = COEFFICIENTS
        out = []
        for x in s["g"].double():
            x = x / (torch.linalg.matrix_norm(x) + EPS)
            for _ in range(STEPS):  # from the side that is shorter
                if c["rows"] > c["cols"]:
                    y = x.t() @ x
                    x = x @ (a * torch.eye(c["cols"], device=x.device) + b * y + f * y @ y)
                else:
                    y = x @ x.t()
                    x = (a * torch.eye(c["rows"], device=x.device) + b * y + f * y @ y) @ x
            out.append(s["scale"] * x)
        return {"out": torch.stack(out)}
    w = s["table"].double()
    first, second, dtable = [], [], torch.zeros_like(w)
    for at in range(0, c["rows"], 1024):
        x, t = s["x"][at:at + 1024].double(), s["targets"][at:at + 1024]
        z, there = s["scale"] * torch.einsum("td,vd->tv", x, w), (t >= 0).double()
        hot = torch.zeros_like(z)
        hot[torch.arange(t.numel(), device=t.device), t.clamp(min=0)] = 1.0
        if c["op"] == "loss":
            lse = torch.logsumexp(z, 1)
            first.append(there * (lse - (hot * z).sum(1)))
            second.append(there * lse)
            continue
        p = torch.exp(z - s["lse"][at:at + 1024].double()[:, None])
        dl = s["dloss"][at:at + 1024].double()[:, None]
        dz = (p - hot) * dl
        if c["penalty"]:
            dz += p * s["dlse"][at:at + 1024].double()[:, None]
        dz *= s["scale"] * there[:, None]
        first.append(torch.einsum("tv,vd->td", dz, w))
        dtable += torch.einsum("tv,td->vd", dz, x)
    if c["op"] == "loss":
        return {"loss": torch.cat(first), "lse": torch.cat(second)}
    return {"dx": torch.cat(first), "dtable": dtable}
