"""Operators of a training step around the DCNv4 module, as measurable cases: layer norm, dropout, the two fused
at the end of a residual branch, and the classifier's cross entropy out of the last linear layer; each with its
gradient.

Feature maps enter as rows: P pixels (or tokens) of C channels.  `run` computes a case either through the
framework's entry points (`own`) or in plain torch operations in 32 bits, rounded once at the end.

Dropout's decisions are part of its definition, so both forms make them alike: the Philox 4x32 generator with ten
rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011), key = the 64-bit seed,
counter = (block, offset) of 64 bits each; element i takes 16 bits, number i % 8 of block i / 8 (low half of a word
first), and is dropped where they are below round(p * 65536).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16}
ES = {"f32": 4, "f16": 2}
M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF
IGNORE = -100


def _rows(name, op, dtype, P, C, p=0.0):
    return {"name": name, "op": op, "dtype": dtype, "P": P, "C": C, "p": p}


def _loss(name, op, dtype, P, K, V, ignored=0.0):
    return {"name": name, "op": op, "dtype": dtype, "P": P, "K": K, "V": V, "ignored": ignored}


def listed():
    return [
        # one 7x7 map of the last stage in inference: latency
        _rows("norm_f16_49x1024", "norm", "f16", 49, 1024),
        # stage 1 of a classification backbone, batch 64: forward and backward of a training step in single precision
        _rows("norm_train_f32_200704x128", "norm_train", "f32", 64 * 56 * 56, 128),
        # the backward pass alone at an odd resolution and width
        _rows("norm_backward_f16_5883x321", "norm_backward", "f16", 3 * 37 * 53, 321),
        # the hidden layer of a stage 3 block, whose width is four times the map's
        _rows("dropout_f16_12544x2048", "dropout", "f16", 64 * 14 * 14, 2048, 0.1),
        # a branch joined to its residual, forward and backward, at an odd length
        _rows("dropout_train_f32_13357x191", "dropout_train", "f32", 13357, 191, 0.25),
        # the end of a branch and the norm in front of the next one: inference-sized forward, then training steps of a
        # detection map and of wide rows
        _rows("branch_f16_50176x256", "branch", "f16", 64 * 28 * 28, 256, 0.1),
        _rows("branch_train_f16_134400x256", "branch_train", "f16", 2 * 200 * 336, 256, 0.1),
        _rows("branch_train_f32_2047x4096", "branch_train", "f32", 2047, 4096, 0.2),
        # a classifier on pooled features: one batch, a thousand classes
        _loss("loss_f16_64x1024_1000", "loss", "f16", 64, 1024, 1000),
        # dense prediction: many pixels, few classes, some pixels without a label
        _loss("loss_train_f16_51200x256_150", "loss_train", "f16", 51200, 256, 150, 0.1),
        # many rows and many classes: the largest matrix products
        _loss("loss_train_f16_8192x1024_40009", "loss_train", "f16", 8192, 1024, 40009, 0.05),
        # the same in single precision, smaller
        _loss("loss_backward_f32_2000x768_10007", "loss_backward", "f32", 2000, 768, 10007, 0.05),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    dtype = rng.choice(["f16", "f16", "f32"])
    op = rng.choice(["norm", "norm_train", "norm_backward", "dropout", "dropout_train", "branch", "branch_train", "branch_train",
                     "loss", "loss_train", "loss_train", "loss_backward"])
    if op.startswith("loss"):
        P, K, V = _log(rng, 1, 16384), 32 * max(1, _log(rng, 64, 2048) // 32), _log(rng, 2, 60000)
        most = 3e11 if dtype == "f16" else 4e10                 # products: below the largest listed case of the type
        while float(P) * K * V > most:
            P = (P + 1) // 2
        case = _loss("", op, dtype, P, K, V, rng.choice([0.0, 0.1]))
    else:
        C = _log(rng, 16, 8192)
        if rng.random() < 0.5:
            C = (C + 31) // 32 * 32
        P = max(1, min(_log(rng, 1, 200000), 20_000_000 // C))
        case = _rows("", op, dtype, P, C, 0.0 if op.startswith("norm") else rng.choice([0.05, 0.1, 0.2, 0.5]))
    del case["name"]
    return case


def prepare(case, seed):
    dt, op, dev = DTYPES[case["dtype"]], case["op"], "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape, scale=1.0, shift=0.0):
        return (torch.randn(shape, generator=gen, device=dev) * scale + shift).to(dt)

    s = {"op": op, "eps": 1e-6}
    if op.startswith("loss"):
        P, K, V = case["P"], case["K"], case["V"]
        # normalised features, a classifier whose logits have a spread of about 2; target drawn anywhere
        s["x"], s["w"], s["b"] = randn(P, K), randn(V, K, scale=2.0 / math.sqrt(K)), randn(V, scale=0.1)
        target = torch.randint(0, V, (P,), generator=gen, device=dev)
        ignored = torch.rand((P,), generator=gen, device=dev) < case["ignored"]
        s["target"] = torch.where(ignored, torch.full_like(target, IGNORE), target)
        # the mean over the labelled rows, with the loss scaled as training in half precision does
        count = (s["target"] != IGNORE).sum().clamp(min=1).float()
        scale = 65536.0 if case["dtype"] == "f16" else 1.0
        s["grad_loss"] = torch.where(ignored, torch.zeros(P, device=dev), (scale / count).expand(P)).contiguous()
        if op == "loss_backward":                               # what the forward pass left
            s["lse"] = _logits(s["x"], s["w"], s["b"]).logsumexp(-1)
        if own:
            from paper_2401_06197_amd import binding as dcn
            need = dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn._dtype_code(s["x"]), op != "loss")
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=dev)
        return s
    P, C = case["P"], case["C"]
    s["x"] = randn(P, C, scale=1.5, shift=0.3)
    if not op.startswith("norm"):
        s["p"], s["seed"], s["offset"] = case["p"], seed * 1_000_003 + 17, 5 + seed % 7
        s["residual"] = randn(P, C)
    if not op.startswith("dropout"):
        s["gamma"], s["beta"] = randn(C, scale=0.2, shift=1.0), randn(C, scale=0.2)
    if op not in ("norm", "dropout", "branch"):
        s["grad_y"] = randn(P, C)
    if op == "branch_train":
        s["grad_z"] = randn(P, C)
    if op == "norm_backward":                                   # what the forward pass left
        x = s["x"].double()
        s["mean"] = x.mean(-1).float()
        s["rstd"] = (x.var(-1, unbiased=False) + s["eps"]).rsqrt().float()
    if own and op in ("norm_train", "norm_backward", "branch_train"):
        from paper_2401_06197_amd import binding as dcn
        s["workspace"] = torch.empty(dcn.dcnv4_layer_norm_workspace_bytes(P, C), dtype=torch.uint8, device=dev)
    return s


def _run_own(s):
    from paper_2401_06197_amd import binding as dcn
    op = s["op"]
    if op == "norm":
        return dcn.dcnv4_layer_norm(s["x"], s["gamma"], s["beta"], eps=s["eps"])
    if op == "norm_train":
        y, mean, rstd = dcn.dcnv4_layer_norm(s["x"], s["gamma"], s["beta"], eps=s["eps"], stats=True)
        return (y, *dcn.dcnv4_layer_norm_backward(s["x"], s["gamma"], mean, rstd, s["grad_y"], workspace=s["workspace"]))
    if op == "norm_backward":
        return dcn.dcnv4_layer_norm_backward(s["x"], s["gamma"], s["mean"], s["rstd"], s["grad_y"], workspace=s["workspace"])
    if op == "dropout":
        return dcn.dcnv4_dropout(s["x"], s["p"], s["seed"], s["offset"])
    if op == "dropout_train":
        return (dcn.dcnv4_dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["residual"]),
                dcn.dcnv4_dropout_backward(s["grad_y"], s["p"], s["seed"], s["offset"]))
    if op.startswith("branch"):
        z, y, mean, rstd = dcn.dcnv4_dropout_add_layer_norm(s["x"], s["residual"], s["gamma"], s["beta"], s["p"], s["seed"], s["offset"], eps=s["eps"])
        if op == "branch":
            return z, y
        return (z, y, *dcn.dcnv4_dropout_add_layer_norm_backward(z, s["gamma"], mean, rstd, s["grad_y"], s["p"], s["seed"], s["offset"],
                                                                grad_z=s["grad_z"], workspace=s["workspace"]))
    kw = {"b": s["b"], "ignore_index": IGNORE, "workspace": s["workspace"]}
    if op == "loss_backward":
        return dcn.dcnv4_linear_cross_entropy_backward(s["x"], s["w"], s["target"], s["lse"], s["grad_loss"], **kw)
    loss, lse = dcn.dcnv4_linear_cross_entropy(s["x"], s["w"], s["target"], **kw)
    if op == "loss":
        return loss, lse
    return (loss, *dcn.dcnv4_linear_cross_entropy_backward(s["x"], s["w"], s["target"], lse, s["grad_loss"], **kw))


def _kept(n, p, seed, offset, device):
    """1 / (1 - p) where an element stays, else 0 (Philox in 64-bit integers: a product of two words wraps, its two
    words are still right)."""
    blocks = (n + 7) // 8
    i = torch.arange(blocks, device=device, dtype=torch.int64)
    c = [i & LOW, i >> 32, torch.full_like(i, offset & LOW), torch.full_like(i, (offset >> 32) & LOW)]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        a, b = c[0] * M0, c[2] * M1
        c = [((b >> 32) & LOW) ^ c[1] ^ k0, b & LOW, ((a >> 32) & LOW) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    bits = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], -1).reshape(-1)[:n]
    t = int(math.floor(p * 65536 + 0.5))
    return (bits >= t).float() * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _norm(x, gamma, beta, eps):
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    return (x - mean) * rstd * gamma + beta, mean, rstd


def _norm_backward(x, gamma, mean, rstd, grad_y):
    xhat, g = (x - mean) * rstd, grad_y * gamma
    grad_x = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return grad_x, (grad_y * xhat).sum(0), grad_y.sum(0)


def _logits(x, w, b):
    return x.float() @ w.float().T + b.float()


def run(s):
    if own:
        return _run_own(s)
    op, dt = s["op"], s["x"].dtype
    f = {k: v.float() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op.startswith("norm"):
        x, out = f["x"], []
        if op == "norm_backward":
            mean, rstd = f["mean"][:, None], f["rstd"][:, None]
        else:
            y, mean, rstd = _norm(x, f["gamma"], f["beta"], s["eps"])
            if op == "norm":
                return y.to(dt)
            out = [y]
        return tuple(t.to(dt) for t in (*out, *_norm_backward(x, f["gamma"], mean, rstd, f["grad_y"])))
    if not op.startswith("loss"):
        kept = _kept(s["x"].numel(), s["p"], s["seed"], s["offset"], s["x"].device).reshape(s["x"].shape)
        if op == "dropout":
            return (f["x"] * kept).to(dt)
        z = f["residual"] + f["x"] * kept
        if op == "dropout_train":
            return z.to(dt), (f["grad_y"] * kept).to(dt)
        z = z.to(dt)                                            # an output, and what the norm reads
        y, mean, rstd = _norm(z.float(), f["gamma"], f["beta"], s["eps"])
        if op == "branch":
            return z, y.to(dt)
        grad, grad_gamma, grad_beta = _norm_backward(z.float(), f["gamma"], mean, rstd, f["grad_y"])
        grad = grad + f["grad_z"]
        return z, y.to(dt), (grad * kept).to(dt), grad.to(dt), grad_gamma.to(dt), grad_beta.to(dt)
    logits = _logits(s["x"], s["w"], s["b"])
    labelled = s["target"] != IGNORE
    at = torch.where(labelled, s["target"], torch.zeros_like(s["target"]))[:, None]
    if op == "loss_backward":
        lse = s["lse"][:, None]
    else:
        top = logits.max(-1, keepdim=True).values
        lse = (logits - top).exp().sum(-1, keepdim=True).log() + top
        loss = torch.where(labelled, (lse - logits.gather(1, at))[:, 0], torch.zeros_like(lse[:, 0]))
        if op == "loss":
            return loss, lse[:, 0]
    grad = (logits - lse).exp()
    grad.scatter_add_(1, at, torch.full_like(lse, -1.0))
    grad = grad * torch.where(labelled, s["grad_loss"], torch.zeros_like(s["grad_loss"]))[:, None]
    grads = tuple(t.to(dt) for t in (grad @ f["w"], grad.T @ f["x"], grad.sum(0)))
    return grads if op == "loss_backward" else (loss, *grads)


def work(case):
    op, es = case["op"], ES[case["dtype"]]
    if op.startswith("loss"):
        P, K, V = case["P"], case["K"], case["V"]
        once = P * K + V * K + V                                # x, w, b, and their gradients
        product = 2.0 * P * K * V
        if op == "loss":
            return {"bytes": float(es * once + 12 * P), "flops": product}
        # the logits, and the two products of their gradient (in a whole step the logits are needed once)
        return {"bytes": float(2 * es * once + 16 * P), "flops": 3 * product}
    n, C = case["P"] * case["C"], case["C"]
    tensors = {"norm": 2, "norm_train": 4, "norm_backward": 3, "dropout": 2, "dropout_train": 5, "branch": 4, "branch_train": 8}[op]
    vectors = {"norm": 2, "norm_train": 4, "norm_backward": 3, "branch": 2, "branch_train": 4}.get(op, 0)
    flops = {"norm": 8, "norm_train": 20, "norm_backward": 12, "dropout": 2, "dropout_train": 4, "branch": 10, "branch_train": 26}[op]
    return {"bytes": float(es * (tensors * n + vectors * C)), "flops": float(flops * n)}


def _exact_kept(n, p, seed, offset, device):
    """The decisions once more, in unsigned words on the host."""
    words = np.zeros((4, (n + 7) // 8), dtype=np.uint64)
    words[0] = np.arange(words.shape[1], dtype=np.uint64)
    words[2:] = [[offset & LOW], [(offset >> 32) & LOW]]
    key = np.array([seed & LOW, (seed >> 32) & LOW], dtype=np.uint64)
    for _ in range(10):
        even, odd = words[0] * np.uint64(M0), words[2] * np.uint64(M1)
        words = np.stack([(odd >> np.uint64(32)) ^ words[1] ^ key[0], odd & np.uint64(LOW),
                          (even >> np.uint64(32)) ^ words[3] ^ key[1], even & np.uint64(LOW)])
        key = (key + np.array([W0, W1], dtype=np.uint64)) & np.uint64(LOW)
    halves = np.ascontiguousarray(words.T.astype("<u4")).view("<u2").reshape(-1)[:n]
    limit = math.floor(p * 65536 + 0.5)
    keep = torch.from_numpy(halves >= limit).to(device)
    return keep.double() / (1.0 - limit / 65536.0) if limit < 65536 else torch.zeros(n, dtype=torch.float64, device=device)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    x = d["x"]
    if op.startswith("loss"):
        labels = s["target"]
        have = labels.ge(0)
        loss, every, gx, gw, gb = [], [], [], torch.zeros_like(d["w"]), torch.zeros_like(d["b"])
        step = max(1, 2 ** 28 // d["w"].shape[0])
        for i in range(0, x.shape[0], step):                    # some rows at a time
            rows, ok = x[i:i + step], have[i:i + step]
            logits = rows @ d["w"].T + d["b"]
            logp = torch.log_softmax(logits, -1)
            every.append((logits - logp)[:, 0])
            hot = torch.zeros_like(logp)
            hot[ok, labels[i:i + step][ok]] = 1.0
            loss.append(-(torch.where(hot > 0, logp, torch.zeros_like(logp))).sum(-1))
            if op == "loss":
                continue
            delta = (logp.exp() - hot) * (d["grad_loss"][i:i + step] * ok)[:, None]
            gx.append(delta @ d["w"])
            gw += delta.T @ rows
            gb += delta.sum(0)
        if op == "loss":
            return torch.cat(loss), torch.cat(every)
        grads = (torch.cat(gx), gw, gb)
        return grads if op == "loss_backward" else (torch.cat(loss), *grads)
    kept = None if op.startswith("norm") else _exact_kept(x.numel(), s["p"], s["seed"], s["offset"], x.device).reshape(x.shape)
    if op == "dropout":
        return x * kept
    if op == "dropout_train":
        return d["residual"] + x * kept, d["grad_y"] * kept
    z = x if kept is None else d["residual"] + x * kept
    # what the norm reads is the stored sum
    source = z if kept is None else z.to(s["x"].dtype).double()
    n = source.shape[-1]
    centred = source - source.sum(-1, keepdim=True) / n
    sigma = (centred.pow(2).sum(-1, keepdim=True) / n + s["eps"]).sqrt()
    unit = centred / sigma
    y = unit * d["gamma"] + d["beta"]
    first = () if op == "norm_backward" else (y,) if kept is None else (z, y)
    if "grad_y" not in d:
        return first if kept is not None else y
    gy = d["grad_y"]
    through = gy * d["gamma"]
    grad = (through - through.sum(-1, keepdim=True) / n - unit * ((through * unit).sum(-1, keepdim=True) / n)) / sigma
    last = ((gy * unit).sum(0), gy.sum(0))
    if kept is None:
        return (*first, grad, *last)
    grad = grad + d["grad_z"]
    return (*first, grad * kept, grad, *last)
