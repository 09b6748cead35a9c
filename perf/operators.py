"""Operators that stand around a clipped step, as cases that can be timed and compared.

* layer norm, forward: output, normalised input (what the norms of the gain's gradient read), mean, 1/std
* layer norm, backward: input gradient, every example's sums for gain and shift, their squared norms
* the preference loss on the LM head's logits of paired sequences: loss, log-probabilities, logit gradients
* orthogonalised updates: Newton-Schulz products on the noised sums of a model's linear layers

Where `own` is false everything is computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

V_GPT2 = 50257
IGNORED = -1                                   # target of a prompt or padding token
COEFS = (3.4445, -4.7750, 2.0315)              # the quintic that the Muon optimiser iterates
STEPS = 5
EPS_NS = 1e-7
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one short sequence through a narrow norm: a launch and its latency
        dict(name="ln_one_short", op="ln", B=1, T=16, p=64, dtype="f32", params="f32", hat=True),
        # a GPT-2-small norm at the batch of the flagship step; its normalised input is kept for the gain's norm
        dict(name="ln_small", op="ln", B=64, T=256, p=768, dtype="bf16", params="f32", hat=True),
        # an odd width, which no vector load fits, over a ragged batch
        dict(name="ln_odd_f32", op="ln", B=21, T=203, p=1001, dtype="f32", params="f32", hat=False),
        # the smallest step's norm, backwards
        dict(name="ln_back_tiny", op="ln_back", B=4, T=16, p=64, dtype="f32", params="f32"),
        # few examples at the full context: the sums run over long sequences
        dict(name="ln_back_context", op="ln_back", B=6, T=1024, p=768, dtype="bf16", params="bf16"),
        # GPT-2 medium, long sequences, a large batch
        dict(name="ln_back_medium", op="ln_back", B=64, T=512, p=1024, dtype="bf16", params="f32"),
        # one pair of short answers over a small vocabulary
        dict(name="pref_tiny", op="pref", B=1, T=16, V=1000, dtype="f32", smoothing=0.0),
        # answers of ordinary length, GPT-2's vocabulary, padded pitch
        dict(name="pref_ordinary", op="pref", B=16, T=128, V=V_GPT2, dtype="bf16", smoothing=0.0),
        # fp32 logits of ragged length, smoothed labels
        dict(name="pref_ragged_f32", op="pref", B=5, T=333, V=V_GPT2, dtype="f32", smoothing=0.1),
        # the smallest step's one matrix
        dict(name="ns_tiny", op="ns", d_model=64, blocks=1, square=True, dtype="f32", out="f32"),
        # every linear layer of DistilGPT2
        dict(name="ns_distil", op="ns", d_model=768, blocks=6, square=False, dtype="f32", out="f32"),
        # every linear layer of GPT-2 medium, updates in bf16
        dict(name="ns_medium", op="ns", d_model=1024, blocks=24, square=False, dtype="f32", out="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["ln", "ln_back", "pref", "ns"])
    top = max(work(c)["bytes"] for c in listed())
    while True:
        if op in ("ln", "ln_back"):
            c = dict(op=op, B=log_int(1, 96), T=log_int(1, 1024), p=log_int(16, 4096), dtype=rng.choice(["f32", "bf16"]),
                     params=rng.choice(["f32", "bf16"]))
            if op == "ln":
                c["hat"] = rng.random() < 0.5
            most = work(dict(listed()[5]))["bytes"]
        elif op == "pref":
            c = dict(op=op, B=log_int(1, 32), T=log_int(1, 512), V=log_int(50, V_GPT2), dtype=rng.choice(["f32", "bf16"]),
                     smoothing=rng.choice([0.0, 0.0, 0.1]))
            most = top
        else:
            c = dict(op=op, d_model=log_int(24, 1024), blocks=log_int(1, 24), square=rng.random() < 0.3, dtype=rng.choice(["f32", "bf16"]),
                     out=rng.choice(["f32", "bf16"]))
            most = top
        if work(c)["bytes"] <= most:
            return c


def _shapes(case):
    """(rows, columns) of each kind of linear layer's weight gradient."""
    d = case["d_model"]
    return [(d, d)] if case["square"] else [(3 * d, d), (d, d), (4 * d, d), (d, 4 * d)]


def work(case):
    op = case["op"]
    if op == "ns":
        # one symmetric product X X^T, one A A^T, one B X per step
        flops = size = 0
        for r, c in _shapes(case):
            m, n = min(r, c), max(r, c)
            flops += STEPS * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)
            size += r * c
        each = (4 if case["dtype"] == "f32" else 2) + (4 if case["out"] == "f32" else 2)
        return {"bytes": case["blocks"] * size * each, "flops": case["blocks"] * flops}
    es = 4 if case["dtype"] == "f32" else 2
    if op == "pref":
        rows = 2 * case["B"] * case["T"]
        n = rows * case["V"]
        return {"bytes": 2 * es * n + 4 * rows + 20 * case["B"], "flops": 6 * n}
    rows, p, ps = case["B"] * case["T"], case["p"], 4 if case["params"] == "f32" else 2
    n = rows * p
    if op == "ln":
        return {"bytes": (3 if case["hat"] else 2) * es * n + 8 * rows + 2 * ps * p, "flops": 8 * n}
    return {"bytes": 3 * es * n + 8 * rows + ps * p + 8 * case["B"] * p + 4 * case["B"], "flops": 14 * n}


def _inputs(case, seed):
    """The tensors of a case, without anything that belongs to one side."""
    dev, g = "cuda", torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dt = case["op"], DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device=dev).normal_(0.0, std, generator=g)

    if op in ("ln", "ln_back"):
        B, T, p, pt = case["B"], case["T"], case["p"], DTYPES[case["params"]]
        # a residual stream: tokens of different size, off centre, a few columns larger than the rest
        size = torch.exp(normal(B, T, 1, std=0.5, dtype=torch.float32))
        column = 1.0 + 4.0 * (torch.rand(p, generator=g, device=dev) < 0.02)
        x = (size * (normal(B, T, p, dtype=torch.float32) * column + 0.2)).to(dt)
        s = dict(x=x, gain=(1.0 + normal(p, std=0.2, dtype=torch.float32)).to(pt), shift=normal(p, std=0.1, dtype=pt))
        if op == "ln_back":
            s["g"] = normal(B, T, p, std=1e-2)
            x = x.float()
            var, mean = torch.var_mean(x, dim=-1, unbiased=False)
            s.update(mean=mean, rstd=torch.rsqrt(var + 1e-5))
        return s
    if op == "pref":
        B, T, V = case["B"], case["T"], case["V"]
        unit = 16 // torch.empty(0, dtype=dt).element_size()
        pitch = (V + unit - 1) // unit * unit              # rows on 16-byte boundaries, as the head's gradient needs them
        logits = normal(B, 2 * T, pitch, std=1.5)
        targets = torch.randint(0, V, (B, 2, T), generator=g, device=dev, dtype=torch.int32)
        # a prompt that both answers share, answers of different length, padding behind them
        at = torch.arange(T, device=dev)
        prompt = torch.randint(0, T // 4 + 1, (B, 1, 1), generator=g, device=dev)
        length = torch.randint(T // 2, T + 1, (B, 2, 1), generator=g, device=dev)
        targets[(at < prompt) | (at >= length)] = IGNORED
        # likely targets, and a reference model that nearly agrees
        index = targets.view(B, 2 * T, 1).clamp(min=0).long()
        x = logits.gather(2, index) + 6.0
        logits.scatter_(2, index, x)
        x = x.float().squeeze(2).view(B, 2, T)
        logp = x - torch.log(V * math.exp(1.125) + torch.exp(x))
        ref = (logp * (targets >= 0)).sum(-1) + normal(B, 2, std=2.0, dtype=torch.float32)
        return dict(logits=logits, targets=targets, ref=ref)
    # noised clipped sums: a Gaussian draw over a sum of few directions; all layers of a kind behind one another
    kinds = []
    for r, c in _shapes(case):
        k = case["blocks"]
        signal = normal(k, r, 4, dtype=torch.float32) @ normal(k, 4, c, dtype=torch.float32)
        kinds.append((0.8 * normal(k, r, c, dtype=torch.float32) + 0.3 * signal).to(dt))
    return dict(kinds=kinds)


def prepare(case, seed):
    s = _inputs(case, seed)
    op, dev = case["op"], "cuda"
    f32 = dict(dtype=torch.float32, device=dev)
    s["case"] = case
    if op == "ln":
        s.update(y=torch.empty_like(s["x"]), hat=torch.empty_like(s["x"]) if case["hat"] else None,
                 mean=torch.empty(s["x"].shape[:2], **f32), rstd=torch.empty(s["x"].shape[:2], **f32))
    elif op == "ln_back":
        B, T, p = s["x"].shape
        s.update(dx=torch.empty_like(s["x"]), gain_sums=torch.empty(B, p, **f32), shift_sums=torch.empty(B, p, **f32),
                 sq=torch.zeros(B, **f32))
    elif op == "pref":
        s.update(G=torch.zeros_like(s["logits"]), loss=torch.empty(case["B"], **f32), logp=torch.empty(case["B"], 2, **f32),
                 status=torch.zeros(1, dtype=torch.int32, device=dev))
    else:
        s.update(outs=[torch.empty(k.shape, dtype=DTYPES[case["out"]], device=dev) for k in s["kinds"]],
                 status=torch.zeros(1, dtype=torch.int32, device=dev))
        s["mats"] = [m for k in s["kinds"] for m in k]
        s["updates"] = [m for k in s["outs"] for m in k]
        s["scales"] = [_scale(m.shape) for m in s["mats"]]
    if own:                                    # workspaces, allocated once as a training program does
        from paper_2609_40335_b200 import binding as dp
        if op == "ln_back":
            need = dp.dp_layernorm_backward_ws_bytes(B, T, p)
        elif op == "pref":
            need = dp.dp_preference_loss_ws_bytes(case["B"], case["T"])
        elif op == "ns":
            need = dp.dp_orthogonalize_ws_bytes(s["mats"])
        else:
            need = 0
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    return s


def _scale(shape):
    return math.sqrt(max(1.0, shape[-2] / shape[-1]))


BETA = 0.1                                     # of the preference loss


def run(s):
    op, case = s["case"]["op"], s["case"]
    if own:
        return {"ln": _own_ln, "ln_back": _own_ln_back, "pref": _own_pref, "ns": _own_ns}[op](s, case)
    return {"ln": _plain_ln, "ln_back": _plain_ln_back, "pref": _plain_pref, "ns": _plain_ns}[op](s, case)


def _own_ln(s, case):
    from paper_2609_40335_b200 import binding as dp
    dp.dp_layernorm(s["x"], s["gain"], s["shift"], 1e-5, Y=s["y"], X_hat=s["hat"], mean=s["mean"], rstd=s["rstd"])
    return {"y": s["y"], "hat": s["hat"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_ln_back(s, case):
    from paper_2609_40335_b200 import binding as dp
    s["sq"].zero_()
    dp.dp_layernorm_backward(s["g"], s["x"], s["gain"], s["mean"], s["rstd"], dX=s["dx"], gain_sums=s["gain_sums"],
                             shift_sums=s["shift_sums"], sq=s["sq"], ws=s["ws"])
    return {"dx": s["dx"], "gain_sums": s["gain_sums"], "shift_sums": s["shift_sums"], "sq": s["sq"]}


def _own_pref(s, case):
    from paper_2609_40335_b200 import binding as dp
    dp.dp_preference_loss(s["logits"], s["targets"], s["ref"], BETA, loss=s["loss"], logp=s["logp"], G=s["G"], V=case["V"],
                          smoothing=case["smoothing"], ws=s["ws"], dev_status=s["status"])
    return {"loss": s["loss"], "logp": s["logp"], "G": s["G"][:, :, :case["V"]]}


def _own_ns(s, case):
    from paper_2609_40335_b200 import binding as dp
    dp.dp_orthogonalize(s["mats"], s["updates"], scales=s["scales"], coefs=[COEFS] * STEPS, eps=EPS_NS, ws=s["ws"],
                        dev_status=s["status"])
    return list(s["outs"])


def _plain_ln(s, case):
    x, dt = s["x"].float(), s["x"].dtype
    mean = x.mean(-1)
    x = x - mean[..., None]
    rstd = torch.rsqrt((x * x).mean(-1) + 1e-5)
    hat = x * rstd[..., None]
    y = hat * s["gain"].float() + s["shift"].float()
    return {"y": y.to(dt), "hat": hat.to(dt) if case["hat"] else None, "mean": mean, "rstd": rstd}


def _plain_ln_back(s, case):
    g = s["g"].float()
    hat = (s["x"].float() - s["mean"][..., None]) * s["rstd"][..., None]
    gain_sums, shift_sums = (g * hat).sum(1), g.sum(1)
    sq = (gain_sums * gain_sums).sum(-1) + (shift_sums * shift_sums).sum(-1)
    g = g * s["gain"].float()
    dx = (g - g.mean(-1, keepdim=True) - hat * (g * hat).mean(-1, keepdim=True)) * s["rstd"][..., None]
    return {"dx": dx.to(s["x"].dtype), "gain_sums": gain_sums, "shift_sums": shift_sums, "sq": sq}


def _plain_pref(s, case):
    B, T, V = case["B"], case["T"], case["V"]
    x = s["logits"][:, :, :V].float()
    targets = s["targets"].view(B, 2 * T, 1)
    valid, index = targets >= 0, targets.clamp(min=0).long()
    x = x - x.amax(-1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(-1, keepdim=True)
    token = (x.gather(2, index) - torch.log(total)) * valid
    logp = token.view(B, 2, T).double().sum(-1)            # differences of long sums: 64 bits
    margin = logp - s["ref"].double()
    h = BETA * (margin[:, 0] - margin[:, 1])
    eps = case["smoothing"]
    loss = (1 - eps) * torch.log1p(torch.exp(-h)) + eps * torch.log1p(torch.exp(h))
    slope = BETA * (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h))
    c = torch.stack([slope, -slope], 1).float()[:, :, None].expand(B, 2, T).reshape(B, 2 * T, 1) * valid
    G = -c * (e / total)
    G.scatter_add_(2, index, c)
    return {"loss": loss.float(), "logp": logp.float(), "G": G.to(s["logits"].dtype)}


def _newton_schulz(M, coefs, dtype):
    """Of a stack of matrices, in `dtype`."""
    a, b, c = coefs
    x = M.to(dtype)
    if x.shape[1] > x.shape[2]:
        x = x.transpose(1, 2)
    norm = M.double().square().sum((1, 2), keepdim=True).sqrt() + EPS_NS
    x = x / norm.to(dtype)
    for _ in range(STEPS):
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.transpose(1, 2) if M.shape[1] > M.shape[2] else x


def _plain_ns(s, case):
    return [(_newton_schulz(k, COEFS, torch.float32) * _scale(k.shape)).to(DTYPES[case["out"]]).contiguous() for k in s["kinds"]]


# ---- from the definitions, in 64 bits ------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"ln": _exact_ln, "ln_back": _exact_ln_back, "pref": _exact_pref, "ns": _exact_ns}[case["op"]](s, case)


def _exact_ln(s, case):
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=-1, unbiased=False)
    rstd = 1.0 / torch.sqrt(var + 1e-5)
    hat = (x - mean.unsqueeze(-1)) * rstd.unsqueeze(-1)
    return {"y": torch.addcmul(s["shift"].double(), hat, s["gain"].double()), "hat": hat if case["hat"] else None, "mean": mean,
            "rstd": rstd}


def _exact_ln_back(s, case):
    """By automatic differentiation of the norm, each example by itself."""
    dx, gs, ss, sq = [], [], [], []
    for i in range(case["B"]):
        # the statistics that the call is given are those of x but for their rounding: dx follows them
        x, g = s["x"][i].double(), s["g"][i].double()
        mean, rstd = s["mean"][i].double().unsqueeze(-1), s["rstd"][i].double().unsqueeze(-1)
        gain = s["gain"].double().requires_grad_()
        shift = torch.zeros_like(gain).requires_grad_()
        hat = (x - mean) * rstd
        gg, gb = torch.autograd.grad(hat * gain + shift, (gain, shift), g)
        # Jacobian of the norm: rstd * (I - (1 1^T + hat hat^T) / p)
        u = g * gain.detach()
        p = x.shape[-1]
        dx.append(rstd * (u - u.sum(-1, keepdim=True) / p - hat * torch.einsum("tp,tp->t", u, hat).unsqueeze(-1) / p))
        gs.append(gg)
        ss.append(gb)
        sq.append(gg.dot(gg) + gb.dot(gb))
    return {"dx": torch.stack(dx), "gain_sums": torch.stack(gs), "shift_sums": torch.stack(ss), "sq": torch.stack(sq)}


def _exact_pref(s, case):
    """By automatic differentiation of the loss, pair by pair."""
    T, V, eps = case["T"], case["V"], case["smoothing"]
    losses, logps, grads = [], [], []
    for i in range(case["B"]):
        x = s["logits"][i, :, :V].double().requires_grad_()
        t = s["targets"][i].reshape(-1).long()
        token = -torch.nn.functional.cross_entropy(x, t, ignore_index=IGNORED, reduction="none")
        logp = token.view(2, T).sum(1)
        h = BETA * ((logp[0] - s["ref"][i, 0].double()) - (logp[1] - s["ref"][i, 1].double()))
        log_sigmoid = torch.nn.functional.logsigmoid
        loss = -(1 - eps) * log_sigmoid(h) - eps * log_sigmoid(-h)
        grads.append(torch.autograd.grad(loss, x)[0].to(torch.float32 if case["dtype"] == "bf16" else torch.float64))
        losses.append(loss.detach())
        logps.append(logp.detach())
    return {"loss": torch.stack(losses), "logp": torch.stack(logps), "G": torch.stack(grads)}


def _exact_ns(s, case):
    """The same polynomial on the singular values would need a decomposition of each matrix; in 64 bits the
    products themselves are exact enough.  Horner's form on the right-hand Gram matrix, one matrix at a time."""
    a, b, c = COEFS
    found = []
    for k in s["kinds"]:
        stack = []
        for M in k.double():
            x = M / (torch.linalg.matrix_norm(M) + EPS_NS)
            tall = x.shape[0] > x.shape[1]
            for _ in range(STEPS):
                gram = x.T @ x if tall else x @ x.T
                poly = gram @ (c * gram)
                poly += b * gram
                poly.diagonal().add_(a)
                x = x @ poly if tall else poly @ x
            stack.append(x * _scale(M.shape))
        found.append(torch.stack(stack))
    return found
