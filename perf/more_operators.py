"""What a rebuilt network is trained on and answers with, as cases that can be timed: the log
probabilities of given targets with their entropy, top alternatives and gradient; the norm of a
network's gradients, and their clipping; and low-rank adapters of many requests beside a projection
that they share, with their gradients.

Sizes are this repository's networks', powers of two as dense networks have them, and odd ones."""
import math
import random

import torch

own = False

DTYPES = dict(fp32=torch.float32, bf16=torch.bfloat16, fp16=torch.float16)
BYTES = dict(fp32=4, bf16=2, fp16=2)
MAX_NORM = 1.0
MOST_LOGITS = 1 << 28          # rows * cols of the largest listed logits
MOST_GRADS = 1 << 28           # elements of the largest listed gradients
MOST_ADAPTED = 1 << 26         # m * (n + k) of the largest listed adapters

_ops = []


def _handle():
    """The framework's operators, one handle a program."""
    if not _ops:
        from paper_2309_06973_amd.q8 import Q8
        _ops.append(Q8())
    return _ops[0]


# --------------------------------------------------------------------------- the cases
def _logp(rows, cols, dtype, **kw):
    return dict(kind="log_probs", rows=rows, cols=cols, dtype=dtype,
                **{**dict(top=0, entropy=False, scale=1.0, ignored=0.0, banned=0.0, train=False), **kw})


def _clip(count, total, dtype, keep=1.0):
    return dict(kind="clip", count=count, total=total, dtype=dtype, keep=keep)


def _adapters(m, n, k, rank, adapters, dtype, **kw):
    return dict(kind="adapters", m=m, n=n, k=k, rank=rank, adapters=adapters, dtype=dtype,
                **{**dict(codes=False, runs=True, train=False), **kw})


def listed():
    return [
        # one token's answer: its distribution's entropy and the twenty likeliest alternatives
        dict(name="log_probs_token_odd", **_logp(1, 50001, "bf16", top=20, entropy=True, banned=0.2)),
        # a test set through an image classifier of 200 classes: the label's log probability, the best five
        dict(name="log_probs_classes", **_logp(10000, 200, "fp32", top=5)),
        # a batch of requests that answer, with a temperature
        dict(name="log_probs_batch", **_logp(128, 131072, "bf16", top=20, entropy=True, scale=1.25)),
        # a training step on a wide odd output with an entropy term, and its gradient
        dict(name="log_probs_train_odd", **_logp(2048, 50001, "fp16", entropy=True, ignored=0.1, train=True)),
        # a large batch's training step, padded positions among them, and its gradient
        dict(name="log_probs_train_wide", **_logp(8192, 32768, "bf16", ignored=0.2, train=True)),
        # the gradients of a tiny network: latency
        dict(name="clip_tiny", **_clip(8, 24112, "fp32")),
        # a residual network of 161 tensors that trains on under its mask
        dict(name="clip_masked", **_clip(161, 25502912, "fp32", keep=0.3)),
        # a wide network of a few large tensors
        dict(name="clip_wide", **_clip(17, MOST_GRADS, "fp32")),
        # one token beside an 8-bit projection, which has its input in 8 bits
        dict(name="adapters_token", **_adapters(1, 4096, 4096, 16, 8, "bf16", codes=True)),
        # a batch of requests beside a rebuilt layer, an adapter a row
        dict(name="adapters_requests_odd", **_adapters(48, 3277, 3541, 8, 32, "fp16", runs=False)),
        # prompts of six requests beside an 8-bit projection
        dict(name="adapters_prompts", **_adapters(8192, 4096, 4096, 16, 6, "bf16", codes=True)),
        # a training step of three adapters: forward, and the gradients of input and adapters
        dict(name="adapters_train", **_adapters(4096, 2048, 2048, 32, 3, "bf16", train=True)),
    ]


def draw(rng: random.Random):
    log = lambda a, b: int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))
    # three in five a multiple of some power of two, the others as they come
    size = lambda v: max(1, v // 64 * 64) if v >= 64 and rng.random() < 0.6 else v
    kind = rng.choice(["log_probs", "log_probs", "clip", "adapters", "adapters"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    half = 2 if dtype == "fp32" else 1
    if kind == "log_probs":
        cols = size(log(10, 131072))
        rows = log(1, min(16384, MOST_LOGITS // cols // half))
        train = rng.random() < 0.5
        return _logp(rows, cols, dtype, top=0 if train or rows * cols > MOST_LOGITS // 8 else
                     rng.choice([0, 1, min(5, cols), min(20, cols)]), entropy=rng.random() < 0.5,
                     scale=rng.choice([1.0, 1.0, 0.7, 1.25]), ignored=rng.choice([0.0, 0.2]) if train else 0.0,
                     banned=rng.choice([0.0, 0.5]), train=train)
    if kind == "clip":
        total = log(1000, MOST_GRADS)
        return _clip(log(1, min(400, total // 100)), total, dtype, rng.choice([1.0, 1.0, 0.5, 0.1]))
    n, k, rank = size(log(16, 8192)), size(log(16, 8192)), rng.choice([1, 4, 8, 12, 16, 16, 32, 64])
    m = log(1, min(8192, MOST_ADAPTED // (n + k) // half))
    train = rng.random() < 0.4
    return _adapters(m, n, k, rank, log(1, 64), dtype, codes=not train and rng.random() < 0.4,
                     runs=train or rng.random() < 0.6, train=train)


# --------------------------------------------------------------------------- inputs
def _sizes(count, total):
    """Elements of a network's `count` tensors: a few hold most of them, vectors hold hardly any."""
    rng = random.Random(count * 1000003 + total)
    share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(count)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    sizes[sizes.index(max(sizes))] += total - sum(sizes)
    return sizes


def _activations(g, rows, cols):
    """Normal values with a scale of its own for each channel and each token."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.7 * torch.randn(cols, generator=g, device="cuda"))
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    return x


def _logits(s, g):
    rows, cols = s["rows"], s["cols"]
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda")) * 2.0
    x += torch.randn(cols, generator=g, device="cuda")
    s["target"] = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    if s["banned"]:                     # places that this answer may not take
        off = torch.rand(cols, generator=g, device="cuda") < s["banned"]
        off[0] = False
        x[:, off] = float("-inf")
        s["target"][off[s["target"]]] = 0
    s["target"][torch.rand(rows, generator=g, device="cuda") < s["ignored"]] = -1
    # a target that the network has learned something about
    hit = (s["target"] >= 0) & (torch.rand(rows, generator=g, device="cuda") < 0.7)
    x.scatter_add_(1, s["target"].clamp(min=0)[:, None], 6.0 * hit[:, None].float())
    s["x"] = x.to(DTYPES[s["dtype"]])
    if s["train"]:                      # of the mean over the targets, and of an entropy term; fp16 trains with a scaled loss
        loss = (65536.0 if s["dtype"] == "fp16" else 1.0) / rows
        s["g_logp"] = torch.where(s["target"] >= 0, -loss, 0.0)
        s["g_entropy"] = torch.full((rows,), -0.01 * loss, device="cuda") if s["entropy"] else None


def _grads(s, g):
    t = DTYPES[s["dtype"]]
    scale = lambda: float(torch.exp(torch.randn(1, generator=g, device="cuda") - 5.0))
    s["grads"] = [(torch.randn(n, generator=g, device="cuda") * scale()).to(t) for n in _sizes(s["count"], s["total"])]
    s["masks"] = None
    if s["keep"] < 1.0:
        s["masks"] = [(torch.rand(x.shape, generator=g, device="cuda") < s["keep"]).to(torch.uint8) for x in s["grads"]]
    s["arena"] = torch.empty(s["total"], dtype=t, device="cuda")       # one tensor behind the other
    s["out"] = list(s["arena"].split([x.numel() for x in s["grads"]]))


def _which(s, g):
    """The adapter of each row, -1: none.  Requests' rows one after another, or as they come."""
    m, many = s["m"], s["adapters"]
    if not s["runs"]:
        return torch.randint(-1 if m > 1 else 0, many, (m,), generator=g, device="cuda")
    cut = torch.randint(0, m + 1, (min(m, many) - 1,), generator=g, device="cuda").sort().values
    of = torch.randperm(many, generator=g, device="cuda")
    if m > 8 and many > 3:
        of[0] = -1                       # a request without an adapter
    return of[torch.bucketize(torch.arange(m, device="cuda"), cut, right=True)]


def _adapted(s, g):
    m, n, k, rank, many = (s[i] for i in ("m", "n", "k", "rank", "adapters"))
    t = DTYPES[s["dtype"]]
    x = _activations(g, m, k)
    if s["codes"]:                       # rows as an 8-bit product reads them
        top = x.abs().amax(1, keepdim=True).clamp_min(1e-30)
        s["q"] = torch.zeros((m, -(-k // 16) * 16), dtype=torch.int8, device="cuda")
        s["q"][:, :k] = torch.round(x * (127.0 / top)).to(torch.int8)
        s["q_scale"] = (top / 127.0).reshape(-1).contiguous()
    else:
        s["x"] = x.to(t)
    s["a"] = (torch.randn(many, rank, k, generator=g, device="cuda") / math.sqrt(k)).to(t)
    s["b"] = (torch.randn(many, n, rank, generator=g, device="cuda") * (0.1 / math.sqrt(rank))).to(t)
    s["scale"] = 0.5 + 2.0 * torch.rand(many, generator=g, device="cuda")
    s["which"] = _which(s, g)
    s["y"] = _activations(g, m, n).to(t)
    if s["train"]:
        s["g"] = (_activations(g, m, n) * 1e-3).to(t)
        s["down"] = torch.empty(m, rank, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    {"log_probs": _logits, "clip": _grads, "adapters": _adapted}[case["kind"]](s, g)
    if own:
        s["ops"] = _handle()
        if s.get("codes"):
            from paper_2309_06973_amd.q8 import Q8Matrix
            s["x"] = Q8Matrix(s["q"], s["q_scale"], s["k"])
    return s


# --------------------------------------------------------------------------- one pass
def _run_own(s):
    ops = s["ops"]
    if s["kind"] == "log_probs":
        r = ops.log_probs(s["x"], s["target"], scale=s["scale"], entropy=s["entropy"], top=s["top"])
        outputs = dict(logp=r.logp, lse=r.lse)
        if s["entropy"]:
            outputs["entropy"] = r.entropy
        if s["top"]:
            outputs.update(top=r.top, index=r.index)
        if s["train"]:
            outputs["grad"] = ops.log_probs_grad(s["x"], s["target"], r.norm, s["g_logp"], entropy=r.entropy,
                                                 g_entropy=s["g_entropy"], scale=s["scale"])
        return outputs
    if s["kind"] == "clip":
        return dict(norm=ops.clip_grad_norm(s["grads"], MAX_NORM, masks=s["masks"], out=s["out"]), out=s["arena"])
    if not s["train"]:
        return ops.adapters(s["y"], s["x"], s["a"], s["b"], s["which"], scale=s["scale"])
    y = ops.adapters(s["y"], s["x"], s["a"], s["b"], s["which"], scale=s["scale"], down=s["down"])
    dx, da, db = ops.adapters_grad(s["g"], s["x"], s["a"], s["b"], s["which"], scale=s["scale"], down=s["down"])
    return dict(y=y, dx=dx, da=da, db=db)


def _run_log_probs(s):
    x, target = s["x"].float(), s["target"]
    z = x * s["scale"]
    best = z.amax(1, keepdim=True)
    e = torch.exp(z - best)
    total = e.sum(1, keepdim=True)
    lse = best + torch.log(total)
    given = target >= 0
    at = target.clamp(min=0)[:, None]
    logp = torch.where(given, (z.gather(1, at) - lse)[:, 0], 0.0)
    outputs = dict(logp=logp, lse=lse[:, 0])
    if s["entropy"] or s["train"]:
        p = e / total
    if s["entropy"]:
        log_p = (z - lse).clamp(min=-1e30)
        entropy = -(p * log_p).sum(1, keepdim=True)
        outputs["entropy"] = entropy[:, 0]
    if s["top"]:
        # one whole number a place: its logit's order, then the lower index
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -2147483648 - bits, bits)
        key = (order << 32) + (4294967295 - torch.arange(x.shape[1], device=x.device))
        index = 4294967295 - (torch.topk(key, s["top"], dim=1).values & 4294967295)
        outputs.update(top=z.gather(1, index) - lse, index=index)
    if s["train"]:
        g = torch.where(given, s["g_logp"], 0.0)[:, None]
        d = -p * g
        d.scatter_add_(1, at, g)
        if s["entropy"]:
            d -= s["g_entropy"][:, None] * p * (log_p + entropy)
        outputs["grad"] = (d * s["scale"]).to(s["x"].dtype)
    return outputs


def _run_clip(s):
    kept = [x.float() for x in s["grads"]]
    if s["masks"]:
        kept = [x * (m != 0) for x, m in zip(kept, s["masks"])]
    norm = torch.stack([torch.sum(x * x, dtype=torch.float64) for x in kept]).sum().sqrt()
    factor = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0).float()
    torch._foreach_copy_(s["out"], torch._foreach_mul(kept, factor))
    return dict(norm=norm.float(), out=s["arena"])


def _run_adapters(s):
    """All adapters' products, a row's own kept."""
    m, n, k, rank, many = (s[i] for i in ("m", "n", "k", "rank", "adapters"))
    x = s["q"][:, :k].float() * s["q_scale"][:, None] if s["codes"] else s["x"].float()
    a = s["a"].float().reshape(many * rank, k)
    b = s["b"].float().permute(0, 2, 1).reshape(many * rank, n)
    own_scale = (s["which"][:, None] == torch.arange(many, device=x.device)) * s["scale"]
    down = (x @ a.t()).view(m, many, rank) * own_scale[:, :, None]
    down = down.reshape(m, many * rank)
    y = (s["y"].float() + down @ b).to(s["y"].dtype)
    if not s["train"]:
        return y
    g = s["g"].float()
    up = ((g @ b.t()).view(m, many, rank) * own_scale[:, :, None]).reshape(m, many * rank)
    db = (g.t() @ down).view(n, many, rank).permute(1, 0, 2).contiguous()
    return dict(y=y, dx=(up @ a).to(s["g"].dtype), da=(up.t() @ x).view(many, rank, k), db=db)


def run(s):
    if own:
        return _run_own(s)
    return {"log_probs": _run_log_probs, "clip": _run_clip, "adapters": _run_adapters}[s["kind"]](s)


# --------------------------------------------------------------------------- what a pass needs
def work(case):
    t = BYTES[case["dtype"]]
    if case["kind"] == "log_probs":
        rows, e = case["rows"], case["rows"] * case["cols"]
        # read x and targets; write log probabilities, sums, entropies, alternatives; then the gradient
        small = rows * (8 + 4 + 4 + (4 if case["entropy"] else 0) + 12 * case["top"])
        return dict(bytes=e * t * (2 if case["train"] else 1) + small,
                    flops=e * (4 + (2 if case["entropy"] else 0) + (4 if case["train"] else 0)))
    if case["kind"] == "clip":
        return dict(bytes=case["total"] * (2 * t + (1 if case["keep"] < 1.0 else 0)), flops=3 * case["total"])
    m, n, k, rank = case["m"], case["n"], case["k"], case["rank"]
    adapters = min(m, case["adapters"]) * rank * (n + k) * t
    read = m * (k + 4) if case["codes"] else m * k * t
    work = dict(bytes=read + 2 * m * n * t + 8 * m + adapters, flops=2 * m * rank * (n + k))
    if case["train"]:                    # read the output's gradient; write the input's and the adapters'
        work["bytes"] += m * (n + k) * t + case["adapters"] * rank * (n + k) * 4
        work["flops"] *= 3
    return work


# --------------------------------------------------------------------------- the definition in 64 bits
def _exact_log_probs(s):
    parts = []
    for i in range(0, s["rows"], 256):
        z = s["x"][i:i + 256].double() * s["scale"]
        target = s["target"][i:i + 256]
        lse = torch.logsumexp(z, 1)
        log_p = z - lse[:, None]
        rows = torch.arange(z.shape[0], device=z.device)
        inside = target >= 0
        part = dict(logp=torch.where(inside, log_p[rows, target.clamp(min=0)], 0.0), lse=lse)
        p = log_p.exp()
        if s["entropy"]:
            part["entropy"] = torch.special.entr(p).sum(1)
        if s["top"]:
            index = torch.sort(s["x"][i:i + 256].double(), dim=1, descending=True, stable=True).indices[:, :s["top"]]
            part.update(top=torch.take_along_dim(log_p, index, 1), index=index)
        if s["train"]:
            here = torch.zeros_like(p)
            here[rows[inside], target[inside]] = 1.0
            d = s["g_logp"][i:i + 256].double()[:, None] * (here * inside[:, None] - p * inside[:, None])
            if s["entropy"]:             # d(-sum p log p) / dz, places without probability left out
                d += s["g_entropy"][i:i + 256].double()[:, None] * (torch.special.entr(p) - p * part["entropy"][:, None])
            part["grad"] = (d * s["scale"]).float()
        parts.append(part)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_clip(s):
    kept = [x.double() if s["masks"] is None else torch.where(s["masks"][i] != 0, x.double(), 0.0)
            for i, x in enumerate(s["grads"])]
    norm = math.sqrt(math.fsum(float(torch.dot(x, x)) for x in kept))
    factor = min(1.0, MAX_NORM / (norm + 1e-6))
    return dict(norm=torch.tensor(norm, dtype=torch.float64, device="cuda"), out=torch.cat(kept) * factor)


def _exact_adapters(s):
    x = s["q"][:, :s["k"]].double() * s["q_scale"].double()[:, None] if s["codes"] else s["x"].double()
    y = s["y"].double()
    dx, da, db = torch.zeros_like(x), torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda"), \
        torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for i in range(s["adapters"]):
        rows = torch.nonzero(s["which"] == i)[:, 0]
        if not len(rows):
            continue
        a, b, c = s["a"][i].double(), s["b"][i].double(), float(s["scale"][i])
        down = torch.mm(x[rows], a.t().contiguous())
        y[rows] += c * torch.mm(down, b.t().contiguous())
        if s["train"]:
            g = s["g"][rows].double()
            up = c * torch.mm(g, b)
            dx[rows] = torch.mm(up, a)
            da[i] = torch.mm(up.t().contiguous(), x[rows])
            db[i] = c * torch.mm(g.t().contiguous(), down)
    return dict(y=y, dx=dx, da=da, db=db) if s["train"] else y


def exact(case, seed):
    s = prepare(case, seed)
    return {"log_probs": _exact_log_probs, "clip": _exact_clip, "adapters": _exact_adapters}[case["kind"]](s)
