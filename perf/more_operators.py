"""The operators around a vocabulary: which calls are timed, on what inputs, and what they compute.

``run`` makes one pass: a forward call, or a forward call and the gradients that a training step takes from it.

  head       log-probabilities of given labels from hidden states h (N, D) and the vocabulary's weight w (V, D), with
             logits x = scale h w^T that are never kept, and on request the log of the sum of their exponentials.
             Gradients: h and w.
  norm       layer norm over rows of D, with or without weight and bias.  Gradients: the rows, weight and bias.
  embedding  scaled rows of a table by given tokens.  Gradient: the table.

Conventions: a label outside [0, V) marks a row without one (log-probability 0, no gradient through it); a token outside
the table gives a row of zeros and no gradient.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
          "int32": torch.int32, "int64": torch.int64}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4, "int32": 4, "int64": 8}


def _head(name, rows, classes, width, dtype, train=False, labelled=1.0, log_sums=False, scale=1.0, label="int64", pad=0):
    case = {"op": "head", "rows": rows, "classes": classes, "width": width, "dtype": dtype, "train": train,
            "labelled": labelled, "log_sums": log_sums, "scale": scale, "label": label, "pad": pad}
    return dict(case, name=name) if name else case


def _norm(name, rows, width, dtype, train=False, affine="", pad=0):
    case = {"op": "norm", "rows": rows, "width": width, "dtype": dtype, "train": train, "affine": affine, "pad": pad}
    return dict(case, name=name) if name else case


def _embedding(name, tokens, rows, width, dtype, train=False, scale=1.0, token="int64"):
    case = {"op": "embedding", "tokens": tokens, "rows": rows, "width": width, "dtype": dtype, "train": train,
            "scale": scale, "token": token}
    return dict(case, name=name) if name else case


def listed():
    return [
        # scoring one sampled token from its hidden state (latency)
        _head("token_1x32768x1024", 1, 32768, 1024, "bf16"),
        # scoring a prompt against a vocabulary of odd size
        _head("prompt_509x50021x1024", 509, 50021, 1024, "bf16", log_sums=True),
        # a training step, a few rows without a label
        _head("head_train_4096x32768x1024", 4096, 32768, 1024, "bf16", train=True, labelled=0.95),
        # a training step on answers alone: half of a batch are prompts, whose rows have no label
        _head("answers_train_8192x131072x2048", 8192, 131072, 2048, "bf16", train=True, labelled=0.5),
        # a small training step with odd sizes everywhere and a penalty on the log of the sum, at a temperature
        _head("odd_train_1003x8191x777", 1003, 8191, 777, "f16", train=True, labelled=0.9, log_sums=True, scale=0.5),
        # a training step in 32 bits
        _head("head_train_2048x16384x1024", 2048, 16384, 1024, "f32", train=True, label="int32"),
        # the norm of one token (latency)
        _norm("norm_token_1x4096", 1, 4096, "bf16", affine="bf16"),
        # a training step's norm over a batch, parameters kept in 32 bits
        _norm("norm_train_16384x2048", 16384, 2048, "bf16", train=True, affine="f32"),
        # the same over rows of odd length out of padded ones
        _norm("norm_train_3001x1001", 3001, 1001, "f32", train=True, affine="f32", pad=23),
        # the rows of a few streams' new tokens (latency)
        _embedding("tokens_64_of_32768x1024", 64, 32768, 1024, "bf16"),
        # a training step's lookup and the table's gradient, tokens by their frequency
        _embedding("tokens_train_16384_of_50021x1024", 16384, 50021, 1024, "bf16", train=True, scale=32.0),
        # a small vocabulary, whose rows are used many times, of odd width
        _embedding("tokens_train_60001_of_259x257", 60001, 259, 257, "f32", train=True, token="int32"),
    ]


def _log(rng, lo, hi):
    """A whole number spread over its logarithm; half of those above 64 are multiples of 16."""
    hi = max(lo, hi)
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, n // 16 * 16) if n > 64 and rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["head", "head", "norm", "embedding"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    train = rng.random() < 0.6
    if op == "head":
        most = 1 << (39 if dtype != "f32" else 36)              # rows * classes * width
        width = _log(rng, 16, 4096)
        classes = _log(rng, 2, min(131072, (1 << 28) // width))
        rows = _log(rng, 1, min(8192, most // (width * classes)))
        return _head(None, rows, classes, width, dtype, train, rng.choice([1.0, 1.0, 0.95, 0.7, 0.3]),
                     rng.random() < 0.3, rng.choice([1.0, 1.0, 0.5, 1.25]), rng.choice(["int64", "int32"]),
                     rng.choice([0, 0, 0, 8, 13]))
    if op == "norm":
        width = _log(rng, 16, 16384)
        rows = _log(rng, 1, min(1 << 16, (1 << 26) // width))
        return _norm(None, rows, width, dtype, train, rng.choice(["", dtype, dtype, "f32"]), rng.choice([0, 0, 0, 1, 24]))
    width = _log(rng, 1, 4096)
    rows = _log(rng, 2, min(131072, (1 << 27) // width))
    tokens = _log(rng, 1, min(1 << 16, (1 << 26) // width))
    return _embedding(None, tokens, rows, width, dtype, train, rng.choice([1.0, 8.0, 0.3]), rng.choice(["int64", "int32"]))


def _labelled(case):
    return max(1, int(round(case["rows"] * case["labelled"])))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    state = {"case": case}
    dtype = _TYPES[case["dtype"]]

    def normal(shape, scale=1.0, kind=dtype):
        return (torch.randn(shape, generator=gen, device=dev) * scale).to(kind)

    def uniform(shape):
        return torch.rand(shape, generator=gen, device=dev)

    if case["op"] == "head":
        n, v, d = case["rows"], case["classes"], case["width"]
        weight = normal((v, d), 1.0 / math.sqrt(d))
        label = torch.randint(0, v, (n,), generator=gen, device=dev)
        # normed hidden states that point to their label, some hardly and some so that it has nearly all of the mass
        hidden = torch.randn((n, d + case["pad"]), generator=gen, device=dev)
        hidden[:, :d] += 0.5 * math.sqrt(d) * uniform((n, 1)) * weight[label].float()
        keep = torch.rand(n, generator=gen, device=dev).argsort() < _labelled(case)
        state["labels"] = torch.where(keep, label, torch.full_like(label, -100)).to(_TYPES[case["label"]])
        state["hidden"] = hidden.to(dtype)[:, :d].detach()
        state["weight"] = weight
        if case["train"]:
            # of a loss summed over the rows (a mean's 1 / n is applied to the scale of the loss)
            state["up_log_probs"] = -(0.5 + uniform((n,)))
            state["up_log_sums"] = 0.02 * uniform((n,)) if case["log_sums"] else None
            state["hidden"].requires_grad_(True)
            state["weight"].requires_grad_(True)
        return state
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        # a stream of hidden states: rows of differing size and mean, a few channels that stand out
        x = torch.randn((n, d + case["pad"]), generator=gen, device=dev)
        x *= 1.0 + 9.0 * (uniform((d + case["pad"],)) < 0.01)
        x = x * (0.5 + 2.0 * uniform((n, 1))) + 0.5 * torch.randn((n, 1), generator=gen, device=dev)
        state["x"] = x.to(dtype)[:, :d].detach()
        state["weight"] = state["bias"] = None
        if case["affine"]:
            state["weight"] = (1.0 + normal((d,), 0.1, torch.float32)).to(_TYPES[case["affine"]])
            state["bias"] = normal((d,), 0.1, _TYPES[case["affine"]])
        if case["train"]:
            state["up"] = normal((n, d))
            for name in ("x", "weight", "bias"):
                if state[name] is not None:
                    state[name].requires_grad_(True)
        return state
    n, v, d = case["tokens"], case["rows"], case["width"]
    # tokens by rank: the chance of the r-th most frequent falls as 1 / (r + 2.7); some are padding
    mass = (1.0 / (torch.arange(v, device=dev, dtype=torch.float64) + 2.7)).cumsum(0)
    rank = torch.searchsorted(mass, torch.rand(n, generator=gen, device=dev, dtype=torch.float64) * mass[-1])
    order = torch.rand(v, generator=gen, device=dev).argsort()
    token = order[rank.clamp_max(v - 1)]
    if n > 64:
        token = torch.where(uniform((n,)) < 0.03, torch.full_like(token, -1), token)
    state["tokens"] = token.to(_TYPES[case["token"]])
    state["table"] = normal((v, d), 1.0 / math.sqrt(d))
    if case["train"]:
        state["up"] = normal((n, d), 0.1)
        state["table"].requires_grad_(True)
    return state


def _run_own(state):
    from paper_2608_24738_amd import training
    case = state["case"]
    if case["op"] == "head":
        got = training.head_log_probs(state["hidden"], state["weight"], state["labels"], scale=case["scale"],
                                      log_sums=case["log_sums"])
        out = [got.log_probs] + ([got.log_sums] if case["log_sums"] else [])
        if case["train"]:
            ups = [state["up_log_probs"]] + ([state["up_log_sums"]] if case["log_sums"] else [])
            grads = torch.autograd.grad(out, [state["hidden"], state["weight"]], ups)
            out = [t.detach() for t in out] + list(grads)
        return out
    if case["op"] == "norm":
        leaves = [state[name] for name in ("x", "weight", "bias") if state[name] is not None]
        out = training.layer_norm(state["x"], state["weight"], state["bias"])
    else:
        leaves = [state["table"]]
        out = training.embedding(state["tokens"], state["table"], scale=case["scale"])
    if case["train"]:
        return [out.detach()] + list(torch.autograd.grad([out], leaves, [state["up"]]))
    return [out]


def _plain_head(state):
    case = state["case"]
    hidden, weight = state["hidden"].detach(), state["weight"].detach()
    h, w = hidden.float(), weight.float()
    classes = case["classes"]
    x = (h @ w.t()) * case["scale"]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    s = e.sum(1, keepdim=True)
    sums = m + s.log()
    label = state["labels"].long()
    valid = (label >= 0) & (label < classes)
    index = torch.where(valid, label, torch.zeros_like(label))[:, None]
    logp = torch.where(valid, (x.gather(1, index) - m - s.log())[:, 0], torch.zeros_like(s[:, 0]))
    out = [logp] + ([sums[:, 0]] if case["log_sums"] else [])
    if case["train"]:
        up = torch.where(valid, state["up_log_probs"], torch.zeros_like(logp))
        back = up if state["up_log_sums"] is None else up - state["up_log_sums"]
        grad = e.mul_(-back[:, None] / s)
        grad.scatter_add_(1, index, up[:, None])
        grad *= case["scale"]
        out += [(grad @ w).to(hidden.dtype), (grad.t() @ h).to(weight.dtype)]
    return out


def _plain_norm(state):
    case = state["case"]
    x = state["x"].detach()
    v = x.float()
    centred = v - v.mean(1, keepdim=True)
    r = 1.0 / ((centred * centred).mean(1, keepdim=True) + 1e-5).sqrt()
    t = centred * r
    weight, bias = state["weight"], state["bias"]
    y = t if weight is None else t * weight.detach().float() + bias.detach().float()
    out = [y.to(x.dtype)]
    if case["train"]:
        up = state["up"].float()
        g = up if weight is None else up * weight.detach().float()
        out.append((r * (g - g.mean(1, keepdim=True) - t * (g * t).mean(1, keepdim=True))).to(x.dtype))
        if weight is not None:
            out += [(up * t).sum(0).to(weight.dtype), up.sum(0).to(bias.dtype)]
    return out


def _plain_embedding(state):
    case = state["case"]
    table, token = state["table"].detach(), state["tokens"].long()
    valid = (token >= 0) & (token < case["rows"])
    index = torch.where(valid, token, torch.zeros_like(token))
    rows = table[index].float() * case["scale"]
    out = [torch.where(valid[:, None], rows, torch.zeros_like(rows)).to(table.dtype)]
    if case["train"]:
        up = state["up"].float()
        up = torch.where(valid[:, None], up, torch.zeros_like(up))
        grad = torch.zeros(table.shape, device=table.device).index_add_(0, index, up)
        out.append((grad * case["scale"]).to(table.dtype))
    return out


def run(state):
    if own:
        return _run_own(state)
    with torch.no_grad():
        return {"head": _plain_head, "norm": _plain_norm, "embedding": _plain_embedding}[state["case"]["op"]](state)


def work(case):
    size, train = _BYTES[case["dtype"]], case["train"]
    if case["op"] == "head":
        n = case["rows"] if case["log_sums"] else _labelled(case)
        v, d = case["classes"], case["width"]
        outs = 4 * case["rows"] * (1 + case["log_sums"])
        data = (n * d + v * d) * size + case["rows"] * _BYTES[case["label"]] + outs
        if train:
            data += (case["rows"] * d + v * d) * size + outs
        return {"bytes": data, "flops": (8 if train else 2) * n * v * d}
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        params = 2 * case["width"] * _BYTES[case["affine"]] if case["affine"] else 0
        return {"bytes": (4 if train else 2) * n * size + (2 if train else 1) * params, "flops": (20 if train else 8) * n}
    n, table = case["tokens"] * case["width"], case["rows"] * case["width"]
    used = min(n, table)
    data = case["tokens"] * _BYTES[case["token"]] + (used + n) * size
    if train:
        data += (n + table) * size
    return {"bytes": data, "flops": (2 if train else 1) * n}


def exact(case, seed):
    state = prepare(case, seed)
    with torch.no_grad():
        return {"head": _exact_head, "norm": _exact_norm, "embedding": _exact_embedding}[case["op"]](case, state)


def _exact_head(case, state):
    h, w = state["hidden"].detach().double(), state["weight"].detach().double()
    n, v, scale = case["rows"], case["classes"], case["scale"]
    label = state["labels"].long()
    step = max(1, (1 << 27) // v)
    logps, sums, rows = [], [], []
    grad = torch.zeros_like(w)
    for i in range(0, n, step):
        part, y = h[i:i + step], label[i:i + step]
        logits = scale * torch.mm(part, w.T)
        given = torch.arange(v, device=h.device)[None] == y[:, None]
        total = torch.logsumexp(logits, 1)
        # a row without a label picks nothing
        logps.append(torch.where(given, logits - total[:, None], 0.0).sum(1))
        sums.append(total)
        if case["train"]:
            a = state["up_log_probs"][i:i + step].double() * given.any(1)
            slope = -a[:, None] * torch.softmax(logits, 1)
            if case["log_sums"]:
                slope += state["up_log_sums"][i:i + step].double()[:, None] * torch.softmax(logits, 1)
            slope[given] += a[given.any(1)]
            rows.append(scale * torch.mm(slope, w))
            grad += scale * torch.mm(slope.T, part)
    out = [torch.cat(logps)] + ([torch.cat(sums)] if case["log_sums"] else [])
    return out + ([torch.cat(rows), grad] if case["train"] else [])


def _exact_norm(case, state):
    x = state["x"].detach().double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    unit = (x - mean) / torch.sqrt(var + 1e-5)
    gain = torch.ones(case["width"], dtype=torch.float64, device=x.device)
    shift = torch.zeros_like(gain)
    if case["affine"]:
        gain, shift = state["weight"].detach().double(), state["bias"].detach().double()
    out = [unit * gain + shift]
    if case["train"]:
        up = state["up"].double()
        back = up * gain
        # what is left of the gradient beside the constant and the normed row, both of which the norm takes out
        back = back - back.mean(1, keepdim=True) - unit * (unit * back).mean(1, keepdim=True)
        out.append(back / torch.sqrt(var + 1e-5))
        if case["affine"]:
            out += [(unit * up).sum(0), up.sum(0)]
    return out


def _exact_embedding(case, state):
    token = state["tokens"].long()
    held = ((token >= 0) & (token < case["rows"])).nonzero()[:, 0]
    table = state["table"].detach().double()
    out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device=table.device)
    out[held] = case["scale"] * table[token[held]]
    if not case["train"]:
        return [out]
    # sums over runs of equal tokens, as differences of one running sum
    order = held[torch.argsort(token[held], stable=True)]
    value, count = torch.unique_consecutive(token[order], return_counts=True)
    end = count.cumsum(0)
    running = torch.cat([torch.zeros(1, case["width"], dtype=torch.float64, device=table.device),
                         state["up"].double()[order].cumsum(0)])
    grad = torch.zeros_like(table)
    grad[value] = case["scale"] * (running[end] - running[end - count])
    return [out, grad]
