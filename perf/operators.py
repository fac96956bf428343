"""Performance cases of the operators around the frozen int8 convolutions: what is tuned and served beside them.

``norm``: group norm with an activation over the maps that a convolution hands on or takes in, channels last or in
planes; forward, forward and backward of a training step, or forward into the next convolution's int8 activations.
``adapter``: the low-rank adapters of many requests at once, added to a projection that all requests share; forward
(a prompt's or a batch of single tokens), or forward and backward of a training step.  ``distill``: the loss against a
teacher's top logits; loss and gradient of a training step in one call, or the loss first and its gradient later.

A case is one pass through one operator on data that lies in device memory.  Where ``own`` is true the passes are calls
of the package's operators, else the same formulas in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
EPS = 1e-5


def norm(name, N, C, H, W, groups, type="bf16", layout="nhwc", act="silu", form="forward"):
    case = {"op": "norm", "N": N, "C": C, "H": H, "W": W, "groups": groups, "type": type, "layout": layout,
            "act": act, "form": form}
    return dict(case, name=name) if name else case


def adapter(name, tokens, inputs, outputs, rank, adapters, type="bf16", form="forward", mixed=False):
    case = {"op": "adapter", "tokens": tokens, "inputs": inputs, "outputs": outputs, "rank": rank,
            "adapters": adapters, "type": type, "form": form, "mixed": mixed}
    return dict(case, name=name) if name else case


def distill(name, rows, classes, top, type="bf16", tail=False, form="step"):
    case = {"op": "distill", "rows": rows, "classes": classes, "top": top, "type": type, "tail": tail, "form": form}
    return dict(case, name=name) if name else case


def listed():
    return [
        # One image's deepest map: the latency of a single request.
        norm("norm_b1_c512_s7", 1, 512, 7, 7, 32),
        # Odd everything, one training step: 23 channels to a group, a map of 31x45 pixels.
        norm("norm_train_ragged_b7", 7, 184, 31, 45, 8, type="f16", act="gelu", form="train"),
        # Between two int8 convolutions: float32 planes in, the next layer's int8 planes out.
        norm("norm_i8_c256_s14_b128", 128, 256, 14, 14, 32, type="f32", layout="nchw", act="relu", form="i8"),
        # The widest maps, channels last.
        norm("norm_c64_s224_b32", 32, 64, 224, 224, 32),
        # A training step on the float32 planes that a convolution puts out.
        norm("norm_train_c128_s56_b64", 64, 128, 56, 56, 32, type="f32", layout="nchw", act="relu", form="train"),
        # One token through a classifier's adapter: 512 features to 1000 classes.
        adapter("adapter_token", 1, 512, 1000, 8, 4),
        # A batch of single tokens, each with an adapter of its own: reading the adapters is the work.
        adapter("adapter_tokens_64", 64, 4096, 4096, 16, 64, mixed=True),
        # Prompts of eight requests of different lengths.
        adapter("adapter_prompts", 16384, 4096, 4096, 32, 8),
        # A training step of three adapters, odd counts, float32.
        adapter("adapter_train_ragged", 5003, 2048, 1000, 12, 3, type="f32", form="train"),
        # A classifier's batch against ten stored logits an image.
        distill("distill_b64_c1000", 64, 1000, 10, type="f32"),
        # A vocabulary of odd size, the rest of the teacher's mass as one more outcome; the loss first, the gradient later.
        distill("distill_ragged", 777, 32003, 33, type="f16", tail=True, form="apart"),
        # A long sequence over a large vocabulary: the logits are the largest tensor of a training step.
        distill("distill_s4096_v131072", 4096, 131072, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "adapter", "distill"])
    while True:
        if op == "norm":
            groups = rng.choice([1, 4, 8, 16, 32])
            each = _log_int(rng, 1, 1024 // groups if groups > 1 else 96)
            h = _log_int(rng, 1, 224)
            case = norm(None, _log_int(rng, 1, 64), groups * each, h, max(1, min(224, int(h * rng.uniform(0.5, 2)))),
                        groups, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice(["nhwc", "nchw"]),
                        rng.choice(["none", "relu", "silu", "gelu"]), rng.choice(["forward", "train", "i8"]))
            limit = 4.2e8
        elif op == "adapter":
            few = rng.random() < 0.4  # single tokens, each with its own adapter, or a prompt's and a training step's
            tokens = _log_int(rng, 1, 256) if few else _log_int(rng, 64, 16384)
            case = adapter(None, tokens, _log_int(rng, 64, 4096), _log_int(rng, 64, 4096), _log_int(rng, 1, 64),
                           _log_int(rng, 1, 64) if few else _log_int(rng, 1, 8), rng.choice(["bf16", "bf16", "f16", "f32"]),
                           "forward" if few else rng.choice(["forward", "train"]), few)
            limit = 4.1e8
        else:
            classes = _log_int(rng, 10, 131072)
            case = distill(None, _log_int(rng, 1, 4096), classes, min(classes // 2, _log_int(rng, 1, 128)),
                           rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.4, rng.choice(["step", "apart"]))
            limit = 2.2e9
        if work(case)["bytes"] > limit:
            continue
        # (the spread of a handful of values is no statistic: nobody normalises over fewer than these)
        if op != "norm" or case["C"] // case["groups"] * case["H"] * case["W"] >= 64:
            return case


def work(case):
    size = BYTES[case["type"]]
    if case["op"] == "norm":
        n = case["N"] * case["C"] * case["H"] * case["W"]
        if case["form"] == "train":  # x in, y out; then x and its output's gradient in, its own gradient out
            return {"bytes": 5 * n * size, "flops": 40 * n}
        return {"bytes": n * (size + (1 if case["form"] == "i8" else size)), "flops": 15 * n}
    if case["op"] == "adapter":
        t, k, m, r, a = (case[x] for x in ("tokens", "inputs", "outputs", "rank", "adapters"))
        bank = min(a, t) * r * (k + m) * size
        if case["form"] == "train":  # x, base in, y out; then y's gradient, x, the shared gradient in, x's gradient out, and the bank's
            return {"bytes": t * (3 * k + 3 * m) * size + 3 * bank, "flops": 6 * t * r * (k + m)}
        return {"bytes": t * (k + 2 * m) * size + bank, "flops": 2 * t * r * (k + m)}
    n, k = case["rows"] * case["classes"], case["rows"] * case["top"]
    return {"bytes": n * size * (2 if case["form"] == "step" else 3) + 8 * k + 8 * case["rows"], "flops": 8 * n}


def _lengths(tokens, requests, g):
    """Which adapter each token has: runs of ragged lengths, the requests' tokens one behind the other."""
    cut = torch.sort(torch.randint(0, tokens + 1, (requests - 1,), generator=g, device="cuda"))[0]
    return torch.searchsorted(cut, torch.arange(tokens, device="cuda"), right=True).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, type=None):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(type or dtype)

    state = dict(case)
    if case["op"] == "norm":
        shape = case["N"], case["C"], case["H"], case["W"]
        order = torch.channels_last if case["layout"] == "nhwc" else torch.contiguous_format
        # channels have means and spreads of their own, as a convolution's outputs do
        spread = torch.rand(case["C"], generator=g, device="cuda").view(1, -1, 1, 1) * 1.5 + 0.5
        mean = torch.randn(case["C"], generator=g, device="cuda").view(1, -1, 1, 1)
        x = torch.randn(*shape, generator=g, device="cuda")
        state["x"] = (x * spread + mean).to(dtype).contiguous(memory_format=order)
        state["weight"] = normal(case["C"], scale=0.2, shift=1.0, type=torch.float32)
        state["bias"] = normal(case["C"], scale=0.2, type=torch.float32)
        if case["form"] == "train":
            state["dy"] = normal(*shape).contiguous(memory_format=order)
        if case["form"] == "i8":
            state["y_scale"] = 4.0 / 127
            state["step"] = torch.tensor(state["y_scale"], dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "adapter":
        t, k, m, r, a = (case[x] for x in ("tokens", "inputs", "outputs", "rank", "adapters"))
        if case["mixed"]:  # one request in sixteen has no adapter
            ids = torch.randint(0, a, (t,), generator=g, device="cuda")
            state["ids"] = torch.where(torch.rand(t, generator=g, device="cuda") < 1 / 16, -1, ids).to(torch.int32)
        else:
            state["ids"] = _lengths(t, a, g)
        state["x"], state["base"] = normal(t, k), normal(t, m)
        state["down"] = normal(a, r, k, scale=k ** -0.5)
        state["up"] = normal(a, m, r, scale=r ** -0.5)
        state["scale"] = torch.rand(a, generator=g, device="cuda") + 0.5
        if case["form"] == "train":
            state["dy"], state["dx_base"] = normal(t, m), normal(t, k)
    else:
        rows, classes, top = case["rows"], case["classes"], case["top"]
        state["temperature"] = 2.0
        state["logits"] = normal(rows, classes, scale=2.5)
        # the teacher's largest logits: near the student's, sorted downwards, places without repeats
        step = classes // top
        first = torch.randint(0, step, (rows, top), generator=g, device="cuda") + torch.arange(top, device="cuda") * step
        state["index"] = torch.gather(first, 1, torch.rand(rows, top, generator=g, device="cuda").argsort(1)).to(torch.int32)
        values = torch.sort(torch.randn(rows, top, generator=g, device="cuda") * 1.5 + 6.0, 1, descending=True)[0]
        if case["tail"]:  # log-probabilities whose sum leaves something for the rest
            rest = torch.rand(rows, 1, generator=g, device="cuda") * 0.3 + 0.05
            values = torch.log_softmax(values / state["temperature"], 1) + torch.log1p(-rest)
        state["values"] = values
        # the share of each row in the mean; one row in eight is padding.  Gradients in 16 bits with five bits of
        # exponent are taken of a loss that is scaled up
        kept = (torch.rand(rows, generator=g, device="cuda") >= 1 / 8).float()
        state["row_scale"] = kept / rows * (1024.0 if case["type"] == "f16" else 1.0)
    return state


def run(s):
    if own:
        return _own(s)
    return {"norm": _plain_norm, "adapter": _plain_adapter, "distill": _plain_distill}[s["op"]](s)


def _own(s):
    from paper_2407_02913_amd import adapt

    if s["op"] == "norm":
        args = s["groups"], s["weight"], s["bias"], EPS, s["act"]
        if s["form"] == "i8":
            return adapt.group_norm_i8(s["x"], *args, y_scale=s["y_scale"]) * s["step"]
        if s["form"] == "forward":
            return adapt.group_norm(s["x"], *args)
        y, stats = adapt.group_norm_forward(s["x"], *args)
        return (y,) + adapt.group_norm_backward(s["dy"], s["x"], stats, *args)
    if s["op"] == "adapter":
        bank = s["ids"], s["down"], s["up"], s["scale"]
        y = adapt.add_adapters(s["base"], s["x"], *bank)
        if s["form"] == "forward":
            return y
        return (y,) + adapt.add_adapters_backward(s["dy"], s["x"], *bank, dx_base=s["dx_base"])
    teacher = s["values"], s["index"]
    how = {"temperature": s["temperature"], "tail": s["tail"]}
    if s["form"] == "step":
        return adapt.distill_loss_and_grad(s["logits"], *teacher, row_scale=s["row_scale"], **how)
    loss, stats = adapt.distill_loss(s["logits"], *teacher, row_scale=s["row_scale"], **how)
    return loss, adapt.distill_grad(s["logits"], *teacher, stats, row_scale=s["row_scale"], **how)


def _plain_norm(s):
    x, act = s["x"].float().unflatten(1, (s["groups"], -1)), s["act"]
    mean = x.mean((2, 3, 4), keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean((2, 3, 4), keepdim=True) + EPS)
    hat = d * rstd
    w, b = (s[k].view(1, s["groups"], -1, 1, 1) for k in ("weight", "bias"))
    z = hat * w + b
    if act == "relu":
        y = torch.clamp(z, min=0.0)
    elif act == "silu":
        half = 1.0 / (1.0 + torch.exp(-z))
        y = z * half
    elif act == "gelu":
        half = 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5))
        y = z * half
    else:
        y = z
    if s["form"] == "i8":
        q = torch.clamp(torch.round(y.flatten(1, 2) / s["y_scale"]), -127, 127)
        return q.to(torch.int8).contiguous() * s["step"]
    y = y.flatten(1, 2).to(s["x"].dtype)
    if s["form"] == "forward":
        return y
    dz = s["dy"].float().unflatten(1, (s["groups"], -1))
    if act == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    elif act == "silu":
        dz = dz * (half + z * half * (1.0 - half))
    elif act == "gelu":
        dz = dz * (half + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5)
    db = dz.sum((0, 3, 4)).reshape(-1)
    dw = (dz * hat).sum((0, 3, 4)).reshape(-1)
    dh = dz * w
    dx = rstd * (dh - dh.mean((2, 3, 4), keepdim=True) - hat * (dh * hat).mean((2, 3, 4), keepdim=True))
    return y, dx.flatten(1, 2).to(s["x"].dtype), dw, db


def _plain_adapter(s):
    a, r = s["adapters"], s["rank"]
    # every adapter for every token, in one product; then each token keeps its own
    down = s["down"].float().reshape(a * r, -1)
    up = s["up"].float().transpose(1, 2).reshape(a * r, -1)
    mine = s["ids"].view(-1, 1) == torch.arange(a, device="cuda").view(1, -1)
    mine = (mine * s["scale"]).repeat_interleave(r, 1)
    x = s["x"].float()
    h = (x @ down.t()) * mine
    y = (s["base"].float() + h @ up).to(s["x"].dtype)
    if s["form"] == "forward":
        return y
    dy = s["dy"].float()
    g = (dy @ up.t()) * mine
    dx = (s["dx_base"].float() + g @ down).to(s["x"].dtype)
    d_down = (g.t() @ x).view(a, r, -1)
    d_up = (h.t() @ dy).view(a, r, -1).transpose(1, 2)
    return y, dx, d_down.to(s["x"].dtype), d_up.to(s["x"].dtype).contiguous()


def _plain_distill(s):
    t, index = s["temperature"], s["index"].long()
    z = s["logits"].float() / t
    e = torch.exp(z - z.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    at = torch.gather(z, 1, index) - z.amax(1, keepdim=True) - torch.log(total)  # log q at the teacher's places
    kept = s["row_scale"] != 0
    if s["tail"]:
        p = torch.exp(s["values"])
        p_rest = torch.clamp(1.0 - p.sum(1), min=0.0)
        q_rest = e.scatter(1, index, 0.0).sum(1) / total[:, 0]
        loss = (p * (s["values"] - at)).sum(1) + p_rest * (torch.log(p_rest) - torch.log(q_rest))
        # the rest's share of the gradient: its own places grow with it
        ratio = (p_rest / q_rest).view(-1, 1)
        grad = e / total
        top = torch.gather(grad, 1, index)
        grad = (grad * (1.0 - ratio)).scatter(1, index, top - p)
    else:
        u = s["values"] / t
        f = torch.exp(u - u.amax(1, keepdim=True))
        p = f / f.sum(1, keepdim=True)
        loss = (p * (torch.log(p) - at)).sum(1)
        grad = (e / total).scatter_add(1, index, -p)
    loss = torch.where(kept, loss * (t * t), 0.0)
    return loss, (grad * (s["row_scale"] * t).view(-1, 1)).to(s["logits"].dtype)


def exact(case, seed):
    """The definitions in float64, taken from the inputs anew."""
    s = prepare(case, seed)
    if s["op"] == "norm":
        return _exact_norm(s)
    return _exact_adapter(s) if s["op"] == "adapter" else _exact_distill(s)


def _exact_norm(s):
    n, c, h, w = s["x"].shape
    x = s["x"].double().contiguous().view(n, s["groups"], -1)
    var, mean = torch.var_mean(x, 2, unbiased=False, keepdim=True)
    sd = torch.sqrt(var + EPS)
    hat = ((x - mean) / sd).view(n, c, h * w)
    gamma, beta = s["weight"].double().view(1, c, 1), s["bias"].double().view(1, c, 1)
    z = hat * gamma + beta
    if s["act"] == "relu":
        y, slope = z.clamp(min=0), (z > 0).double()
    elif s["act"] == "silu":
        y, slope = z * torch.sigmoid(z), torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    elif s["act"] == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        y, slope = z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        y, slope = z, torch.ones_like(z)

    def out(v):
        return v.view(n, c, h, w)

    if s["form"] == "i8":
        return out(torch.round(y / s["y_scale"]).clamp(-127, 127) * s["step"].double())
    if s["form"] == "forward":
        return out(y)
    dz = s["dy"].double().contiguous().view(n, c, h * w) * slope
    d_beta, d_gamma = dz.sum((0, 2)), (dz * hat).sum((0, 2))
    u, v = (dz * gamma).view(n, s["groups"], -1), hat.view(n, s["groups"], -1)
    dx = (u - u.mean(2, keepdim=True) - v * (u * v).mean(2, keepdim=True)) / sd
    return out(y), out(dx), d_gamma, d_beta


def _exact_adapter(s):
    x, up, down = s["x"].double(), s["up"].double(), s["down"].double()
    y = s["base"].double()
    train = s["form"] == "train"
    if train:
        dy, dx, d_down, d_up = s["dy"].double(), s["dx_base"].double(), torch.zeros_like(down), torch.zeros_like(up)
    for a in range(s["adapters"]):
        at = torch.nonzero(s["ids"] == a)[:, 0]
        scale = float(s["scale"][a])
        h = x[at] @ down[a].t()
        y[at] += scale * (h @ up[a].t())
        if train:
            g = scale * (dy[at] @ up[a])
            dx[at] += g @ down[a]
            d_down[a] = g.t() @ x[at]
            d_up[a] = scale * (dy[at].t() @ h)
    return (y, dx, d_down, d_up) if train else y


def _exact_distill(s):
    t, index, rows = s["temperature"], s["index"].long(), s["row_scale"].double()
    log_q = torch.log_softmax(s["logits"].double() / t, 1)
    q = torch.exp(log_q)
    if s["tail"]:
        log_p = s["values"].double()
        p = torch.exp(log_p)
        p_rest = 1 - p.sum(1)
        q_rest = q.scatter(1, index, 0).sum(1)
        loss = (p * (log_p - log_q.gather(1, index))).sum(1) + p_rest * (p_rest.log() - q_rest.log())
        # with r = q_rest: d(-p_rest log r)/dz_v = -(p_rest / r) q_v ([v in the rest] - r)
        inside = torch.zeros_like(q).scatter(1, index, 1)
        grad = q * p.sum(1, keepdim=True)
        grad.scatter_add_(1, index, -p)
        grad -= (p_rest / q_rest).view(-1, 1) * q * (1 - inside - q_rest.view(-1, 1))
    else:
        log_p = torch.log_softmax(s["values"].double() / t, 1)
        p = torch.exp(log_p)
        loss = (p * (log_p - log_q.gather(1, index))).sum(1)
        grad = q.scatter_add(1, index, -p)
    return torch.where(rows != 0, loss * t * t, 0.0), grad * (rows * t).view(-1, 1)
