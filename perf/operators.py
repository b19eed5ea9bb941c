"""The operators of a training step on distances: which calls are timed, on what inputs, and what they compute.

``run`` makes one pass: a forward call, or a forward call and the gradients that a training step takes from it.

  labels    log-probabilities of given labels over axis 1 of the logits, with the entropy, the k most likely classes and
            the expected value of a field under the softmax (the boundary loss of a signed distance field).  Two layouts:
            rows (positions, classes), and maps (B, classes, *spatial).
  relative  a learned bias by buckets of the distance between a query's and a key's position, on a sequence (signed
            offsets) or a grid of patches, alone or added to attention scores.
  distance  the same bias from a given distance field, alone or added to logits.

Conventions: a label outside [0, classes) marks an element without one (log-probability 0, no gradient through it); the
bucket of a distance d is the number of edges <= d; a distance is a float32, each operation that makes it rounded.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
          "uint8": torch.uint8, "int32": torch.int32, "int64": torch.int64}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4, "uint8": 1, "int32": 4, "int64": 8}


def _labels(name, shape, dtype, label, train=False, entropy=False, top_k=0, field=False, pad=0):
    case = {"op": "labels", "shape": "x".join(str(n) for n in shape), "dtype": dtype, "label": label, "train": train,
            "entropy": entropy, "top_k": top_k, "field": field, "pad": pad}
    return dict(case, name=name) if name else case


def _relative(name, query, key, heads, buckets, metric, dtype, batch=0, train=False, sampling="", offset=0):
    case = {"op": "relative", "query": "x".join(str(n) for n in query), "key": "x".join(str(n) for n in key),
            "heads": heads, "buckets": buckets, "metric": metric, "dtype": dtype, "batch": batch, "train": train,
            "sampling": sampling, "offset": offset}
    return dict(case, name=name) if name else case


def _distance(name, batch, shape, heads, buckets, dtype, distance="f32", add=False, train=False):
    case = {"op": "distance", "batch": batch, "shape": "x".join(str(n) for n in shape), "heads": heads,
            "buckets": buckets, "dtype": dtype, "distance": distance, "add": add, "train": train}
    return dict(case, name=name) if name else case


def listed():
    return [
        # scoring one sampled token: its log-probability, the entropy and the five likeliest tokens (latency)
        _labels("token_131072", (1, 131072), "bf16", "int64", entropy=True, top_k=5),
        # scoring a prompt against a vocabulary of odd size, out of rows padded for the matrix product before it
        _labels("prompt_512x50021", (512, 50021), "bf16", "int64", entropy=True, top_k=5, pad=43),
        # a training step over rows: log-probabilities and an entropy term, with the logits' gradient
        _labels("rows_train_4096x32768", (4096, 32768), "bf16", "int64", train=True, entropy=True),
        # prediction on the benchmark's volumes: likeliest class, its log-probability and the uncertainty
        _labels("volumes_8x4x128", (8, 4, 128, 128, 128), "bf16", "uint8", entropy=True, top_k=1),
        # a training step with the boundary loss on those volumes: log-probabilities and the expected signed field
        _labels("volumes_train_8x4x128", (8, 4, 128, 128, 128), "f32", "uint8", train=True, field=True),
        # a training step on photographs of an odd size with some twenty classes
        _labels("images_train_16x21x375x500", (16, 21, 375, 500), "bf16", "uint8", train=True),
        # one new token against a sequence of odd length (latency)
        _relative("token_bias_4099", (1,), (4099,), 16, 32, "offset", "bf16", offset=4098),
        # a training step's scores over sequences, with the table's gradient
        _relative("sequence_train_2048", (2048,), (2048,), 16, 32, "offset", "bf16", batch=2, train=True),
        # scores over a grid of image patches
        _relative("patches_32x32", (32, 32), (32, 32), 12, 40, "euclidean", "f16", batch=8),
        # a training step over windows of an anisotropic volume
        _relative("window_train_9x11x10", (9, 11, 10), (9, 11, 10), 3, 24, "euclidean", "f32", batch=4, train=True,
                  sampling="2.5,0.8,0.8"),
        # a training step with a learned prior by the distance to the nearest mark, added to the logits of each class
        _distance("images_prior_train_32x512", 32, (512, 512), 4, 24, "bf16", add=True, train=True),
        # maps for three channels from the chamfer distances of ragged volumes
        _distance("volumes_prior_2x155x240x237", 2, (155, 240, 237), 3, 64, "f32", distance="int32"),
    ]


def _log(rng, lo, hi):
    """A whole number spread over its logarithm; half of those above 64 are multiples of 16."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, n // 16 * 16) if n > 64 and rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["rows", "maps", "maps", "relative", "relative", "distance"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    train = rng.random() < 0.5
    if op == "rows":
        classes = _log(rng, 2, 131072)
        rows = _log(rng, 1, max(1, min(1 << 16, (1 << 27) // (classes * (_BYTES[dtype] // 2)))))
        return _labels(None, (rows, classes), dtype, rng.choice(["int64", "int32"]), train=train,
                       entropy=rng.random() < 0.6, top_k=rng.choice([0, 0, 1, 5, 8]) if classes >= 8 else 0,
                       pad=rng.choice([0, 0, 0, 1, 43]))
    if op == "maps":
        rank = rng.choice([2, 3])
        classes = rng.choice([2, 3, 4, 5, 8, 16, 21, 64, 150])
        total = (1 << 26) // (classes * (_BYTES[dtype] // 2))
        hi = max(9, min(640 if rank == 2 else 160, int(total ** (1.0 / rank))))
        shape = tuple(_log(rng, 7, hi) for _ in range(rank))
        batch = _log(rng, 1, max(1, min(32, total // math.prod(shape))))
        return _labels(None, (batch, classes) + shape, dtype, rng.choice(["uint8", "int64"]), train=train,
                       entropy=rng.random() < 0.5, top_k=rng.choice([0, 1, 1, 2]), field=rng.random() < 0.5)
    if op == "relative":
        rank = rng.choice([1, 1, 2, 3])
        hi = {1: 4096, 2: 48, 3: 13}[rank]
        key = tuple(_log(rng, 2, hi) for _ in range(rank))
        form = rng.choice(["token", "square", "square"])
        query = (1,) * rank if form == "token" else key
        pairs = math.prod(query) * math.prod(key)
        heads = rng.choice([1, 3, 4, 8, 12, 16, 20, 32])
        batch = rng.choice([0, 1, 2, 3, 8])
        while batch * heads * pairs > 1 << 26 and batch:
            batch //= 2
        while heads * pairs > 1 << 27:
            heads //= 2
        metric = rng.choice(["offset", "euclidean"]) if rank == 1 else rng.choice(["euclidean", "taxicab", "chessboard"])
        sampling = "2.5,0.8,0.8" if rank == 3 and metric == "euclidean" and rng.random() < 0.5 else ""
        return _relative(None, query, key, heads, rng.choice([8, 16, 24, 32, 40, 64]), metric, dtype, batch, train,
                         sampling, key[0] - 1 if form == "token" else 0)
    rank = rng.choice([2, 3])
    heads = rng.choice([1, 2, 3, 4, 8, 21])
    total = (1 << 25) // heads
    hi = min(800 if rank == 2 else 240, int(total ** (1.0 / rank)))
    shape = tuple(_log(rng, 7, hi) for _ in range(rank))
    batch = _log(rng, 1, max(1, min(32, total // math.prod(shape))))
    return _distance(None, batch, shape, heads, rng.choice([8, 16, 24, 32, 64, 128]), dtype,
                     rng.choice(["f32", "f32", "int32"]), rng.random() < 0.5, train)


def _ints(text):
    return tuple(int(n) for n in text.split("x"))


def _marks(gen, batch, shape, count, lo, hi):
    """Signed distance to a union of `count` balls with radii U[lo, hi] of the smallest extent: positive inside."""
    dev = gen.device
    out = torch.full((batch,) + shape, -math.inf, device=dev)
    axes = [torch.arange(n, device=dev, dtype=torch.float32) for n in shape]
    for _ in range(count):
        radius = (lo + (hi - lo) * torch.rand(batch, generator=gen, device=dev)) * min(shape)
        square = 0
        for a, axis in enumerate(axes):
            centre = torch.rand(batch, generator=gen, device=dev) * shape[a]
            delta = axis[None, :] - centre[:, None]
            square = square + (delta * delta).reshape((batch,) + (1,) * a + (-1,) + (1,) * (len(shape) - 1 - a))
        out = torch.maximum(out, radius.reshape((batch,) + (1,) * len(shape)) - square.sqrt())
    return out


def _edges(buckets, signed, reach):
    """buckets - 1 ascending edges: one a unit for the nearest half, then growing by a constant factor up to `reach`.
    Signed offsets have half of them on either side of zero."""
    if signed:
        half = _edges((buckets - 1) // 2 + 1, False, reach)
        return [-e for e in reversed(half)] + half + [2.0 * half[-1]] * ((buckets - 1) % 2)
    exact = max(1, buckets // 2)
    far = buckets - 1 - exact
    reach = max(reach, 2.0 * exact)
    out = [0.5 + i for i in range(exact)]
    return out + [0.5 + exact * (reach / exact) ** ((i + 1) / (far + 1)) for i in range(far)]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    state = {"case": case}
    dtype = _TYPES[case["dtype"]]

    def normal(shape, scale, kind):
        return (torch.randn(shape, generator=gen, device=dev) * scale).to(kind)

    if case["op"] == "labels":
        shape = _ints(case["shape"])
        spatial = (shape[0],) + shape[2:]
        if len(shape) == 2:
            # rows: a network's logits over a vocabulary, the given token half the time a likely one
            wide = (shape[0], shape[1] + case["pad"])
            logits = normal(wide, 2.5, dtype)[:, :shape[1]]
            likely = logits[:, :64].float().argmax(1)
            label = torch.where(torch.rand(shape[0], generator=gen, device=dev) < 0.5, likely,
                                torch.randint(0, shape[1], (shape[0],), generator=gen, device=dev))
            ignored = torch.rand(shape[0], generator=gen, device=dev) < (0.05 if shape[0] > 1 else -1.0)
            label = torch.where(ignored, torch.full_like(label, -100), label)
        else:
            # maps: smooth logits with noise, labels in regions, a few elements without a label
            region = _marks(gen, shape[0], shape[2:], 12, 0.05, 0.25)
            label = (region / (0.04 * min(shape[2:]) + 1.0)).floor().clamp(-1, shape[1] - 2).long() + 1
            logits = normal(shape, 1.5, torch.float32)
            logits.scatter_add_(1, label[:, None], torch.full_like(region, 2.0)[:, None])
            logits = logits.to(dtype)
            ignored = torch.rand(spatial, generator=gen, device=dev) < 0.03
            label = torch.where(ignored, torch.full_like(label, 255 if case["label"] == "uint8" else -100), label)
        state["logits"] = logits
        state["labels"] = label.to(_TYPES[case["label"]])
        state["field"] = None
        if case["field"]:
            # a signed distance field of each class
            state["field"] = torch.stack([_marks(gen, shape[0], shape[2:], 6, 0.05, 0.25) for _ in range(shape[1])], 1)
        if case["train"]:
            # of a loss summed over the elements (a mean's 1 / n is applied to the scale of the loss)
            state["up_log_probs"] = -torch.rand(spatial, generator=gen, device=dev)
            if case["entropy"]:
                state["up_entropy"] = normal(spatial, 0.01, torch.float32)
            if case["field"]:
                state["up_field"] = normal(spatial, 0.01, torch.float32)
            state["logits"].requires_grad_(True)
        return state

    heads, buckets = case["heads"], case["buckets"]
    if case["op"] == "relative":
        query, key = _ints(case["query"]), _ints(case["key"])
        reach = float(max(key)) if case["metric"] in ("offset", "chessboard") else float(sum(key))
        edges = _edges(buckets, case["metric"] == "offset", reach)
        batch = case["batch"]
        full = (math.prod(query), math.prod(key))
        state["query"], state["key"] = query, key
        state["sampling"] = tuple(float(s) for s in case["sampling"].split(",")) if case["sampling"] else None
        add = batch > 0
        lead = (batch, heads) if add else (heads,)
    else:
        shape = _ints(case["shape"])
        edges = _edges(buckets, False, 0.5 * min(shape))
        # distance to the nearest mark
        field = (-_marks(gen, case["batch"], shape, 12, 0.01, 0.06)).clamp_min(0.0)
        state["distances"] = field.round().to(torch.int32) if case["distance"] == "int32" else field
        full = shape
        add = case["add"]
        lead = (case["batch"], heads)
    state["edges"] = torch.tensor(edges, dtype=torch.float32, device=dev)
    # a table kept in 32 bits where it is added to scores or logits, in their type where it stands alone
    state["table"] = normal((buckets, heads), 1.0, torch.float32 if add else dtype)
    state["add"] = normal(lead + full, 2.0, dtype) if add else None
    if case["train"]:
        n = math.prod(full)
        state["up"] = normal(lead + full, 1.0 / math.sqrt(n), dtype)
        state["table"].requires_grad_(True)
    return state


def _run_own(state):
    from paper_2608_24738_amd import training
    case = state["case"]
    if case["op"] == "labels":
        got = training.label_log_probs(state["logits"], state["labels"], entropy=case["entropy"], top_k=case["top_k"],
                                       field=state["field"])
        out = [got.log_probs]
        if case["entropy"]:
            out.append(got.entropy)
        if case["field"]:
            out.append(got.field_mean)
        if case["train"]:
            ups = [state["up_log_probs"]]
            ups += [state["up_entropy"]] if case["entropy"] else []
            ups += [state["up_field"]] if case["field"] else []
            grads = torch.autograd.grad(out, [state["logits"]], ups)
            out = [t.detach() for t in out] + list(grads)
        if case["top_k"]:
            out += [got.top_log_probs, got.top_indices]
        return out
    if case["op"] == "relative":
        bias = training.relative_bias(state["table"], state["edges"], state["query"], state["key"],
                                      query_offset=case["offset"], metric=case["metric"], sampling=state["sampling"],
                                      add=state["add"])
    else:
        bias = training.distance_bias(state["distances"], state["table"], state["edges"], add=state["add"])
    if case["train"]:
        grads = torch.autograd.grad([bias], [state["table"]], [state["up"]])
        return [bias.detach()] + list(grads)
    return [bias]


def _plain_labels(state):
    case = state["case"]
    logits, label = state["logits"].detach(), state["labels"].long()
    classes = logits.shape[1]
    x = logits.float()
    m = x.amax(1, keepdim=True)
    x = x - m
    e = x.exp()
    s = e.sum(1, keepdim=True)
    lp = x - s.log()
    p = e / s
    valid = (label >= 0) & (label < classes)
    index = torch.where(valid, label, torch.zeros_like(label))[:, None]
    out = [torch.where(valid, lp.gather(1, index)[:, 0], torch.zeros_like(s[:, 0]))]
    if case["entropy"]:
        entropy = -(p * lp).sum(1)
        out.append(entropy)
    if case["field"]:
        mean = (p * state["field"]).sum(1)
        out.append(mean)
    if case["train"]:
        up = torch.where(valid, state["up_log_probs"], torch.zeros_like(out[0]))
        grad = -p * up[:, None]
        grad.scatter_add_(1, index, up[:, None])
        if case["entropy"]:
            grad -= state["up_entropy"][:, None] * p * (lp + entropy[:, None])
        if case["field"]:
            grad += state["up_field"][:, None] * p * (state["field"] - mean[:, None])
        out.append(grad.to(logits.dtype))
    if case["top_k"]:
        number = torch.arange(classes, device=x.device).reshape((1, -1) + (1,) * (x.dim() - 2))
        values, indices = [], []
        for _ in range(case["top_k"]):
            best = x.amax(1, keepdim=True)
            first = torch.where(x == best, number, classes).amin(1, keepdim=True)
            values.append(lp.gather(1, first))
            indices.append(first)
            x = torch.where(number == first, -math.inf, x)
        out += [torch.cat(values, 1), torch.cat(indices, 1).int()]
    return out


def _grid(shape, dev):
    axes = torch.meshgrid(*[torch.arange(n, device=dev) for n in shape], indexing="ij")
    return [a.reshape(-1) for a in axes]


def _plain_distance(state):
    """Distances between every query and every key, in float32."""
    case = state["case"]
    dev = state["edges"].device
    total = None
    for a, (q, k) in enumerate(zip(_grid(state["query"], dev), _grid(state["key"], dev))):
        delta = (k[None, :] - (q[:, None] + (case["offset"] if a == 0 else 0))).float()
        if case["metric"] == "offset":
            return delta
        if state["sampling"]:
            delta = delta * state["sampling"][a]
        term = delta * delta if case["metric"] == "euclidean" else delta.abs()
        if total is None:
            total = term
        else:
            total = torch.maximum(total, term) if case["metric"] == "chessboard" else total + term
    return total.sqrt() if case["metric"] == "euclidean" else total


def _plain_bias(state):
    case = state["case"]
    table, add = state["table"].detach(), state["add"]
    if case["op"] == "relative":
        d = _plain_distance(state)
    else:
        d = state["distances"].float()
    bucket = torch.zeros(d.shape, dtype=torch.int32, device=d.device)
    for edge in state["edges"]:
        bucket += d >= edge
    bias = table.float().t()[:, bucket]
    if case["op"] == "distance":
        bias = bias.transpose(0, 1)
    out = [(bias + add.float()).to(add.dtype) if add is not None else bias.to(table.dtype)]
    if case["train"]:
        number = torch.arange(case["buckets"], device=d.device, dtype=torch.int32)
        grad = torch.zeros(case["buckets"], case["heads"], device=d.device)
        up = state["up"].reshape((-1, case["heads"], math.prod(d.shape if case["op"] == "relative" else d.shape[1:])))
        shared = case["op"] == "relative"
        chunk = max(1, (1 << 28) // case["buckets"])
        for b in range(up.shape[0]):
            flat = bucket.reshape(-1) if shared else bucket[b].reshape(-1)
            for i in range(0, flat.numel(), chunk):
                member = (flat[i:i + chunk, None] == number).float()
                grad += (up[b, :, i:i + chunk].float() @ member).t()
        out.append(grad.to(table.dtype))
    return out


def run(state):
    if own:
        return _run_own(state)
    with torch.no_grad():
        return _plain_labels(state) if state["case"]["op"] == "labels" else _plain_bias(state)


def work(case):
    size = _BYTES[case["dtype"]]
    if case["op"] == "labels":
        shape = _ints(case["shape"])
        total = math.prod(shape)
        n = total // shape[1]
        read = total * size + n * _BYTES[case["label"]] + (total * 4 if case["field"] else 0)
        write = n * 4 * (1 + case["entropy"] + case["field"] + 2 * case["top_k"])
        flops = total * (4 + 2 * case["entropy"] + 2 * case["field"])
        if case["train"]:
            read += n * 4 * (1 + case["entropy"] + case["field"])
            write += total * size
            flops += total * (3 + 3 * case["entropy"] + 3 * case["field"])
        return {"bytes": read + write, "flops": flops}
    if case["op"] == "relative":
        n = math.prod(_ints(case["query"])) * math.prod(_ints(case["key"])) * case["heads"] * max(1, case["batch"])
        add, read = case["batch"] > 0, 0
    else:
        n = case["batch"] * math.prod(_ints(case["shape"]))
        read, add = 4 * n, case["add"]
        n *= case["heads"]
    read += n * size * add + case["buckets"] * (4 + case["heads"] * (4 if add else size))
    write, flops = n * size, n * add
    if case["train"]:
        read += n * size
        write += case["buckets"] * case["heads"] * (4 if add else size)
        flops += n
    return {"bytes": read + write, "flops": flops}


def exact(case, seed):
    state = prepare(case, seed)
    with torch.no_grad():
        return _exact_labels(case, state) if case["op"] == "labels" else _exact_bias(case, state)


def _exact_labels(case, state):
    classes = state["logits"].shape[1]
    flat = state["logits"].detach().movedim(1, -1)
    lead = flat.shape[:-1]
    flat = flat.reshape(-1, classes)
    label = state["labels"].reshape(-1).long()
    field = state["field"].movedim(1, -1).reshape(-1, classes) if case["field"] else None
    wants = 1 + case["entropy"] + case["field"] + case["train"] + 2 * (case["top_k"] > 0)
    parts = [[] for _ in range(wants)]
    step = max(1, (1 << 25) // classes)
    for i in range(0, flat.shape[0], step):
        x = flat[i:i + step].double()
        lp = x - torch.logsumexp(x, 1, keepdim=True)
        p = torch.softmax(x, 1)
        y = label[i:i + step]
        given = (torch.arange(classes, device=x.device)[None] == y[:, None]).double()
        has = given.sum(1)
        got = [(lp * given).sum(1)]
        if case["entropy"]:
            h = -torch.special.xlogy(p, p).sum(1)
            got.append(h)
        if case["field"]:
            phi = field[i:i + step].double()
            f = (p * phi).sum(1)
            got.append(f)
        if case["train"]:
            a = state["up_log_probs"].reshape(-1)[i:i + step].double()
            slope = -(a * has)[:, None].expand(-1, classes).clone()       # d loss / d p, times p, less its mean
            if case["entropy"]:
                slope -= state["up_entropy"].reshape(-1)[i:i + step].double()[:, None] * (lp + h[:, None])
            if case["field"]:
                slope += state["up_field"].reshape(-1)[i:i + step].double()[:, None] * (phi - f[:, None])
            got.append(p * slope + given * a[:, None])
        if case["top_k"]:
            order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top_k"]]
            got += [lp.gather(1, order), order.int()]
        for part, piece in zip(parts, got):
            part.append(piece)
    out = []
    for part in parts:
        whole = torch.cat(part)
        out.append(whole.reshape(lead) if whole.dim() == 1 else whole.reshape(lead + (-1,)).movedim(-1, 1).contiguous())
    return out


def _exact_bias(case, state):
    table, add = state["table"].detach().double(), state["add"]
    edges = state["edges"]
    if case["op"] == "relative":
        # float32 distances, as the operator defines them
        import numpy as np
        place = [np.stack([g.ravel() for g in np.meshgrid(*[np.arange(n) for n in shape], indexing="ij")], 1)
                 for shape in (state["query"], state["key"])]
        place[0][:, 0] += case["offset"]
        delta = (place[1][None] - place[0][:, None]).astype(np.float32)
        if state["sampling"]:
            delta = delta * np.asarray(state["sampling"], np.float32)
        if case["metric"] == "offset":
            d = delta[..., 0]
        elif case["metric"] == "chessboard":
            d = np.abs(delta).max(2)
        else:
            terms = delta * delta if case["metric"] == "euclidean" else np.abs(delta)
            d = terms[..., 0]
            for a in range(1, terms.shape[2]):
                d = d + terms[..., a]
            d = np.sqrt(d) if case["metric"] == "euclidean" else d
        d = torch.from_numpy(np.ascontiguousarray(d)).to(edges.device)
    else:
        d = state["distances"].float()
    bucket = torch.searchsorted(edges, d, right=True)
    heads = case["heads"]
    if case["op"] == "relative":
        value = table[bucket.reshape(-1)].t().reshape((heads,) + tuple(d.shape))
    else:
        value = torch.stack([table[:, h][bucket] for h in range(heads)], 1)
    out = [value + add.double() if add is not None else value]
    if case["train"]:
        up = state["up"].reshape((-1, heads) + (tuple(d.shape) if case["op"] == "relative" else tuple(d.shape[1:])))
        grad = torch.zeros(case["buckets"], heads, dtype=torch.float64, device=d.device)
        for b in range(up.shape[0]):
            which = (bucket if case["op"] == "relative" else bucket[b]).reshape(-1)
            for h in range(heads):
                grad[:, h] += torch.bincount(which, up[b, h].reshape(-1).double(), minlength=case["buckets"])
        out.append(grad)
    return out
