"""More operators of a training step around the DCNv4 module, as measurable cases: the gated feed-forward layer, the
backward pass of the linear layer, the two ends of a residual block with norms, scale and gate, and the AdamW step
over a network's tensors.

Feature maps enter as rows: P pixels of K (or C) channels.  `run` computes a case either through the framework's entry
points (`own`) or in plain torch operations in 32 bits, rounded once at the end (moments in 64, where they are rounded
to 8 bits).

Gated layer: h = act(x Wg^T + bg) * (x Wu^T + bu), w = (Wg, Wu), b = (bg, bu); act: silu or gelu (with erf).

Block ends: z = residual + gate * scale * first(x), y = second(z); first and second: layer norms, each of which may be
missing; scale per channel, gate per image.  Forms: "post" has the first norm, "pre" the second, "both" both.

AdamW: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps),
g = grad * factor.  States of 8 bits: m and r = sqrt(v) in e4m3 times an fp32 scale per 256 elements of a tensor, which is their
largest magnitude / 448 (below 2^-100: zeros); what is rounded is m or r times 448 / that magnitude.  m is rounded to nearest,
r to one of its two neighbours, up where the 16 bits of the Philox 4x32 generator with ten rounds (Salmon, Moraes, Dror, Shaw:
Parallel random numbers: as easy as 1, 2, 3; 2011) say so, and never from above zero to zero.  Key = seed; counter =
(i / 8 + tensor * 2^40, t), 64 bits each; element i takes number i % 8 of the block's eight halves, low half of a word first.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16}
ES = {"f32": 4, "f16": 2}
BLOCK = 256                                                     # elements that share a scale
BETAS, ADAM_EPS, LR, DECAY, NORM_EPS = (0.9, 0.999), 1e-8, 1e-3, 0.05, 1e-6
M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _gated(name, op, dtype, P, K, F, act):
    return {"name": name, "op": op, "dtype": dtype, "P": P, "K": K, "F": F, "act": act}


def _linear(name, dtype, P, K, N):
    return {"name": name, "op": "linear_backward", "dtype": dtype, "P": P, "K": K, "N": N}


def _end(name, op, dtype, images, rows, C, form):
    return {"name": name, "op": op, "dtype": dtype, "images": images, "rows": rows, "C": C, "form": form}


def _adam(name, dtype, bits, C, blocks, classes, step):
    return {"name": name, "op": "adamw", "dtype": dtype, "bits": bits, "C": C, "blocks": blocks, "classes": classes, "step": step}


def listed():
    return [
        # one 7x7 map of the last stage in inference: latency
        _gated("gated_f16_49x1024_2728", "gated", "f16", 49, 1024, 2728, "silu"),
        # a stage 3 block's feed-forward part, batch 64, in a training step: the largest matrix products
        _gated("gated_train_f16_12544x512_2048", "gated_train", "f16", 64 * 14 * 14, 512, 2048, "silu"),
        # the same part at an odd resolution and widths, and in single precision
        _gated("gated_train_f16_5883x352_936", "gated_train", "f16", 3 * 37 * 53, 352, 936, "gelu"),
        _gated("gated_train_f32_3001x256_680", "gated_train", "f32", 3001, 256, 680, "silu"),
        # the projection down behind it; a small layer of odd sizes in single precision
        _linear("linear_backward_f16_12544x2048_512", "f16", 64 * 14 * 14, 2048, 512),
        _linear("linear_backward_f32_2047x384_1000", "f32", 2047, 384, 1000),
        # the end of a block: one map in inference; a training step of a detection map whose branch ends in a norm; both norms, at
        # an odd resolution and width
        _end("end_f16_49x1024_both", "end", "f16", 1, 49, 1024, "both"),
        _end("end_train_f16_134400x256_post", "end_train", "f16", 2, 200 * 336, 256, "post"),
        _end("end_train_f32_5883x321_both", "end_train", "f32", 3, 37 * 53, 321, "both"),
        # a module of 64 channels (latency); a network of 24 blocks from 128 channels on with states of 8 bits; wide layers with a
        # classifier of many classes, states of 32 bits
        _adam("adamw_f32_64_module", "f32", 32, 64, 1, 0, 1),
        _adam("adamw_f16_128_network_8bit", "f16", 8, 128, 24, 1000, 11),
        _adam("adamw_f16_256_classes", "f16", 32, 256, 4, 15003, 501),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["gated", "gated_train", "gated_train", "linear_backward", "end", "end_train", "end_train", "adamw"])
    dtype = rng.choice(["f16", "f16", "f32"])
    if op in ("gated", "gated_train", "linear_backward"):
        P, K, F = _log(rng, 1, 50000), _log(rng, 32, 2048) // 16 * 16, _log(rng, 32, 4096) // 8 * 8
        most = 1.2e10 if dtype == "f16" else 5e8                # P K F: below the largest listed case of the type
        while float(P) * K * F > most:
            P = (P + 1) // 2
        if op == "linear_backward":
            case = _linear("", dtype, P, K, F)
        else:
            case = _gated("", op, dtype, P, K, F, rng.choice(["silu", "gelu"]))
    elif op in ("end", "end_train"):
        C = _log(rng, 16, 8192)
        if rng.random() < 0.5:
            C = (C + 31) // 32 * 32
        images = _log(rng, 1, 64)
        rows = max(1, min(_log(rng, 1, 50000), 20_000_000 // C // images))
        case = _end("", op, dtype, images, rows, C, rng.choice(["post", "pre", "both"]))
    else:
        case = _adam("", dtype, rng.choice([8, 32]), rng.choice([16, 24, 40, 64, 80, 96]), _log(rng, 1, 24), rng.choice([0, 0, 37, 1000]),
                     _log(rng, 1, 100000))
    del case["name"]
    return case


def _shapes(case):
    """A network's tensors: blocks in four stages (a sixth, a sixth, a half, a sixth of them) of C, 2C, 4C, 8C channels."""
    shapes, n = [], case["blocks"]
    for i in range(n):
        stage = 0 if 6 * i < n else 1 if 3 * i < n else 2 if 6 * i < 5 * n else 3
        C = case["C"] << stage
        om = C // 16 * 32 if C >= 16 else 32
        shapes += [(C, C), (C,), (om, C), (om,), (C, C), (C,), (C,), (C,), (C,), (2, 2 * C, C), (2, 2 * C), (C, 2 * C), (C,)]
    if case["classes"]:
        shapes += [(case["classes"], 8 * case["C"]), (case["classes"],)]
    return shapes


def prepare(case, seed):
    op, dt, dev = case["op"], DTYPES[case["dtype"]], "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape, scale=1.0, shift=0.0, dtype=None):
        return (torch.randn(shape, generator=gen, device=dev) * scale + shift).to(dtype or dt)

    s = {"op": op}
    if op in ("gated", "gated_train"):
        P, K, F = case["P"], case["K"], case["F"]
        s["act"] = case["act"]
        s["x"], s["w"], s["b"] = randn(P, K), randn(2, F, K, scale=1.0 / math.sqrt(K)), randn(2, F, scale=0.1)
        if op == "gated_train":
            s["grad_h"] = randn(P, F, scale=0.05)
        if own:
            from paper_2401_06197_amd import binding as dcn
            need = dcn.dcnv4_gated_linear_workspace_bytes(P, K, F, dcn._dtype_code(s["x"]), op == "gated_train")
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    elif op == "linear_backward":
        P, K, N = case["P"], case["K"], case["N"]
        s["x"], s["w"], s["b"], s["grad_y"] = randn(P, K), randn(N, K, scale=1.0 / math.sqrt(K)), randn(N), randn(P, N, scale=0.05)
        if own:
            from paper_2401_06197_amd import binding as dcn
            need = dcn.dcnv4_linear_backward_workspace_bytes(P, K, N, dcn._dtype_code(s["x"]))
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    elif op in ("end", "end_train"):
        images, rows, C, form = case["images"], case["rows"], case["C"], case["form"]
        s["form"] = form
        s["x"], s["residual"] = randn(images, rows, C, scale=1.5, shift=0.3), randn(images, rows, C)
        s["scale"] = randn(C, scale=0.2, shift=0.5)
        # branches that a training step leaves out, the others scaled up for it
        kept = torch.rand((images,), generator=gen, device=dev) >= 0.1
        s["gate"] = kept.float() / 0.9 if op == "end_train" else None
        if form != "pre":
            s["gamma1"], s["beta1"] = randn(C, scale=0.2, shift=1.0), randn(C, scale=0.2)
        if form != "post":
            s["gamma2"], s["beta2"] = randn(C, scale=0.2, shift=1.0), randn(C, scale=0.2)
        if op == "end_train":
            s["grad_z"] = randn(images, rows, C)
            s["grad_y"] = randn(images, rows, C) if form != "post" else None
            if own:
                from paper_2401_06197_amd import binding as dcn
                need = dcn.dcnv4_norm_scale_add_norm_workspace_bytes(images * rows, C, images)
                s["workspace"] = torch.empty(need, dtype=torch.uint8, device=dev)
    else:
        _prepare_adam(s, case, randn, dev, seed)
    return s


def _prepare_adam(s, case, randn, dev, seed):
    """A network's tensors in one buffer each for parameters, gradients and so on, every tensor from a multiple of 256 elements on."""
    shapes = _shapes(case)
    sizes = np.array([math.prod(x) for x in shapes], dtype=np.int64)
    starts = np.concatenate([[0], np.cumsum((sizes + BLOCK - 1) // BLOCK * BLOCK)])
    n, dt = int(starts[-1]), DTYPES[case["dtype"]]
    of = np.repeat(np.arange(len(shapes)), np.diff(starts) // BLOCK)           # each block's tensor
    # elements of the tensors, and not of what lies between them
    inside = torch.from_numpy(np.minimum(sizes[of] - (np.arange(n // BLOCK) * BLOCK - starts[of]), BLOCK)).to(dev)
    live = (torch.arange(BLOCK, device=dev)[None] < inside[:, None]).reshape(-1)
    up = 1024.0 if case["dtype"] == "f16" else 1.0                              # as training in half precision scales its loss
    s["step"], s["seed"], s["bits"] = case["step"], seed * 1_000_003 + 29, case["bits"]
    s["p"] = torch.where(live, randn(n, scale=0.05, dtype=torch.float32), 0.0)
    s["grad"] = torch.where(live, randn(n, scale=0.01 * up), 0.0).to(dt)
    s["factors"] = torch.tensor([1.0 / up, 0.7], device=dev)
    s["copy"] = torch.where(live, s["p"], 0.0).to(dt) if case["dtype"] == "f16" else None
    m = torch.where(live, randn(n, scale=0.003, dtype=torch.float32), 0.0)
    r = torch.where(live, randn(n, scale=0.003, shift=0.01, dtype=torch.float32).abs(), 0.0)
    if case["bits"] == 8:
        def blocks(v):
            v = v.view(-1, BLOCK)
            scale = v.abs().amax(-1) / 448.0
            return (v / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(-1), scale
        s["m"], ms = blocks(m)
        s["v"], rs = blocks(r)
        s["scales"] = torch.stack([ms, rs], -1).contiguous()
        # number of each block's first eight elements, as the generator counts them
        s["first"] = torch.from_numpy((np.arange(n // BLOCK) * BLOCK - starts[of]) // 8 + of * 2 ** 40).to(dev)
    else:
        s["m"], s["v"] = m, r * r
    decays = [DECAY if len(x) > 1 else 0.0 for x in shapes]
    s["decay"] = torch.tensor(decays, device=dev)[torch.from_numpy(of).to(dev)][:, None]
    if own:
        from paper_2401_06197_amd import binding as dcn

        def views(flat, width=1):
            return [flat[int(a) // width:int(a) // width + (int(k) + width - 1) // width] for a, k in zip(starts, sizes)]
        s["plan"] = dcn.dcnv4_adamw_plan(views(s["p"]), views(s["grad"]), views(s["m"]), views(s["v"]), lr=LR, weight_decay=decays,
                                         scales=views(s["scales"], BLOCK) if case["bits"] == 8 else None,
                                         copies=None if s["copy"] is None else views(s["copy"]))


def _run_own(s):
    from paper_2401_06197_amd import binding as dcn
    op = s["op"]
    if op in ("gated", "gated_train"):
        h = dcn.dcnv4_gated_linear(s["x"], s["w"], s["b"], activation=s["act"], workspace=s["workspace"])
        if op == "gated":
            return h
        return (h, *dcn.dcnv4_gated_linear_backward(s["x"], s["w"], s["grad_h"], s["b"], activation=s["act"], workspace=s["workspace"]))
    if op == "linear_backward":
        return dcn.dcnv4_linear_backward(s["x"], s["w"], s["grad_y"], s["b"], workspace=s["workspace"])
    if op in ("end", "end_train"):
        first = (s["gamma1"], s["beta1"]) if "gamma1" in s else None
        second = (s["gamma2"], s["beta2"]) if "gamma2" in s else None
        z, y, *stats = dcn.dcnv4_norm_scale_add_norm(s["x"], s["residual"], s["scale"], s["gate"], first, second, eps=NORM_EPS)
        if op == "end":
            return z, y
        return (z, y, *dcn.dcnv4_norm_scale_add_norm_backward(s["x"], z, s["scale"], s["gate"], first, second, stats, s["grad_y"], s["grad_z"],
                                                              workspace=s["workspace"]))
    dcn.dcnv4_adamw_step(s["plan"], s["step"], betas=BETAS, eps=ADAM_EPS, seed=s["seed"], factors_on_device=s["factors"])
    return _adam_outputs(s)


def _adam_outputs(s):
    return s["p"], s["m"], s["v"], s.get("scales"), s["copy"]


def _act(a, act):
    """act(a) and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + (-a).exp())
        return a * s, s * (1.0 + a * (1.0 - s))
    phi = 0.5 * torch.erfc(a * -math.sqrt(0.5))
    return a * phi, phi + a * (a * a * -0.5).exp() * (1.0 / math.sqrt(2.0 * math.pi))


def _norm(x):
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + NORM_EPS).rsqrt()
    return (x - mean) * rstd, rstd


def _norm_backward(unit, rstd, g):
    return rstd * (g - g.mean(-1, keepdim=True) - unit * (g * unit).mean(-1, keepdim=True))


def _philox(first, step, seed):
    """Eight 16-bit numbers for each of 32 blocks from `first` on, block after block (in 64-bit integers: a product of two
    words wraps, its two words are still right)."""
    i = (first[:, None] + torch.arange(BLOCK // 8, device=first.device)).reshape(-1)
    c = [i & LOW, i >> 32, torch.full_like(i, step & LOW), torch.full_like(i, (step >> 32) & LOW)]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        a, b = c[0] * M0, c[2] * M1
        c = [((b >> 32) & LOW) ^ c[1] ^ k0, b & LOW, ((a >> 32) & LOW) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    return torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], -1).reshape(-1, BLOCK).int()


def _to_8_bits(v, bits):
    """(what is stored, scales) of blocks [.., 256]: to nearest, or by 16 random bits."""
    top = v.abs().amax(-1, keepdim=True)
    top = torch.where(top >= 2.0 ** -100, top, torch.zeros_like(top))
    scale = top * (1.0 / 448.0)
    t = torch.where(top > 0, v * (torch.full_like(top, 448.0) / top), torch.zeros_like(v)).clamp(-448.0, 448.0)
    if bits is not None:
        fine = ((t.view(torch.int32) + (bits << 4)) & ~0xFFFFF).view(torch.float32)
        coarse = (((t * 2.0 ** 25).int() + bits) >> 16).float() / 512.0
        rounded = torch.where(t >= 2.0 ** -6, fine, coarse)
        t = torch.where(t > 0, rounded.clamp(min=2.0 ** -9), torch.zeros_like(t))
    return t.to(torch.float8_e4m3fn), scale


def _run_adam(s):
    (b1, b2), t, eight = BETAS, s["step"], s["bits"] == 8
    p = s["p"].view(-1, BLOCK)
    g = s["grad"].view(-1, BLOCK).double() * s["factors"][0].double()
    m, v = s["m"].view(-1, BLOCK).double(), s["v"].view(-1, BLOCK).double()
    if eight:
        m, v = m * s["scales"][:, :1].double(), (v * s["scales"][:, 1:].double()).square()
    m = (b1 * m + (1.0 - b1) * g).float()
    v = (b2 * v + (1.0 - b2) * g * g).float()
    r = v.double().sqrt().float()
    lr = LR * s["factors"][1].double()
    step = (lr / (1.0 - b1 ** t)).float() * m / (r * (1.0 / math.sqrt(1.0 - b2 ** t)) + ADAM_EPS)
    p.copy_(p - p * (lr * s["decay"]).float() - step)
    if eight:
        m, ms = _to_8_bits(m, None)
        v, rs = _to_8_bits(r, _philox(s["first"], t, s["seed"]))
        s["scales"].copy_(torch.cat([ms, rs], -1))
    s["m"].view(-1, BLOCK).copy_(m)
    s["v"].view(-1, BLOCK).copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(s["p"])
    return _adam_outputs(s)


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "adamw":
        return _run_adam(s)
    dt = s["x"].dtype
    f = {k: v.float() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    x = f["x"]
    if op == "linear_backward":
        return tuple(t.to(dt) for t in (f["grad_y"] @ f["w"], f["grad_y"].T @ x, f["grad_y"].sum(0)))
    if op in ("gated", "gated_train"):
        F = f["w"].shape[1]
        a, u = x @ f["w"][0].T + f["b"][0], x @ f["w"][1].T + f["b"][1]
        value, slope = _act(a, s["act"])
        h = (value * u).to(dt)
        if op == "gated":
            return h
        both = torch.cat([f["grad_h"] * u * slope, f["grad_h"] * value], -1)
        grads = (both @ f["w"].reshape(2 * F, -1), (both.T @ x).reshape(f["w"].shape), both.sum(0).reshape(2, F))
        return (h, *(t.to(dt) for t in grads))
    one = torch.ones((), device=x.device)
    gate = f["gate"][:, None, None] if "gate" in f else one
    if "gamma1" in f:
        unit1, rstd1 = _norm(x)
        b = unit1 * f["gamma1"] + f["beta1"]
    else:
        b = x
    z = (f["residual"] + gate * f["scale"] * b).to(dt)
    y = None
    if "gamma2" in f:
        unit2, rstd2 = _norm(z.float())
        y = (unit2 * f["gamma2"] + f["beta2"]).to(dt)
    if op == "end":
        return z, y
    grad, pixels = f["grad_z"], (0, 1)
    gamma1 = beta1 = gamma2 = beta2 = None
    if "gamma2" in f:
        grad = grad + _norm_backward(unit2, rstd2, f["grad_y"] * f["gamma2"])
        gamma2, beta2 = (f["grad_y"] * unit2).sum(pixels).to(dt), f["grad_y"].sum(pixels).to(dt)
    gb = grad * gate * f["scale"]
    grad_x = gb
    if "gamma1" in f:
        grad_x = _norm_backward(unit1, rstd1, gb * f["gamma1"])
        gamma1, beta1 = (gb * unit1).sum(pixels).to(dt), gb.sum(pixels).to(dt)
    return (z, y, grad_x.to(dt), grad.to(dt), (grad * gate * b).sum(pixels).to(dt), (grad * f["scale"] * b).sum((1, 2)), gamma1, beta1, gamma2, beta2)


def work(case):
    op, es = case["op"], ES[case["dtype"]]
    if op in ("gated", "gated_train"):
        P, K, F = case["P"], case["K"], case["F"]
        once, product = P * K + 2 * F * K + 2 * F, 4.0 * P * K * F
        if op == "gated":
            return {"bytes": float(es * (once + P * F)), "flops": product}
        # x, the weights, their gradients; h and its gradient.  The layer's products, and two as large of its gradient
        return {"bytes": float(es * (2 * once + 2 * P * F)), "flops": 3 * product}
    if op == "linear_backward":
        P, K, N = case["P"], case["K"], case["N"]
        return {"bytes": float(es * (2 * P * K + 2 * N * K + P * N + N)), "flops": 4.0 * P * K * N}
    if op in ("end", "end_train"):
        n, C, form = case["images"] * case["rows"] * case["C"], case["C"], case["form"]
        tensors = 3 if form == "post" else 4
        if op == "end_train":
            tensors += 3 if form == "post" else 4               # the gradients that come in and go out
        return {"bytes": float(es * (tensors * n + 10 * C)), "flops": float((20 if op == "end" else 60) * n)}
    n = sum(map(math.prod, _shapes(case)))
    states = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
    return {"bytes": n * (8.0 + es + states + (2.0 if es == 2 else 0.0)), "flops": 16.0 * n}


def _exact_adam(s):
    """The step from its definition in 64 bits, with numpy's words for the random numbers."""
    t, dev = s["step"], s["p"].device
    decayed = 1.0 - LR * float(s["factors"][1]) * s["decay"].double()
    grad = s["grad"].double().view(-1, BLOCK) * float(s["factors"][0])
    first, second = s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK)
    if s["bits"] == 8:
        first = first * s["scales"][:, 0].double().unsqueeze(-1)
        second = (second * s["scales"][:, 1].double().unsqueeze(-1)) ** 2
    first = first + (grad - first) * (1.0 - BETAS[0])
    second = second + (grad ** 2 - second) * (1.0 - BETAS[1])
    root = torch.sqrt(second)
    corrected = first / (1.0 - math.pow(BETAS[0], t)), root / math.sqrt(1.0 - math.pow(BETAS[1], t))
    p = s["p"].double().view(-1, BLOCK) * decayed - LR * float(s["factors"][1]) * corrected[0] / (corrected[1] + ADAM_EPS)
    p = p.reshape(-1)
    copy = None if s["copy"] is None else p
    if s["bits"] == 32:
        return p, first.reshape(-1), second.reshape(-1), None, copy
    number = (s["first"].cpu().numpy()[:, None] + np.arange(BLOCK // 8)).reshape(-1).astype(np.uint64)
    words = np.stack([number & np.uint64(LOW), number >> np.uint64(32), np.full_like(number, t & LOW), np.full_like(number, t >> 32)])
    key = np.array([s["seed"] & LOW, (s["seed"] >> 32) & LOW], dtype=np.uint64)
    for _ in range(10):
        even, odd = words[0] * np.uint64(M0), words[2] * np.uint64(M1)
        words = np.stack([(odd >> np.uint64(32)) ^ words[1] ^ key[0], odd & np.uint64(LOW),
                          (even >> np.uint64(32)) ^ words[3] ^ key[1], even & np.uint64(LOW)])
        key = (key + np.array([W0, W1], dtype=np.uint64)) & np.uint64(LOW)
    halves = np.ascontiguousarray(words.T.astype("<u4")).view("<u2").reshape(-1, BLOCK)
    part = torch.from_numpy(halves.astype(np.int32)).to(dev).double() / 65536.0

    def step_of(size):                                          # distance of the type's numbers around one of that size
        return torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3.0)

    def scaled(v):
        scale = v.abs().max(-1, keepdim=True).values / 448.0
        return torch.where(scale > 0, v / scale, torch.zeros_like(v)), scale

    a, sa = scaled(first)
    unit = step_of(a.abs())
    a = torch.round(a / unit) * unit
    r, sr = scaled(root)
    unit = step_of(r)
    # (random bits that are more than a number's missing part, by 16 bits, leave it below)
    up = torch.floor(r / unit * 65536.0) / 65536.0 + part
    stored = torch.minimum(torch.floor(up) * unit, torch.full_like(r, 448.0))
    stored = torch.where(r > 0, stored.clamp(min=2.0 ** -9), torch.zeros_like(r))
    return p, a.reshape(-1), stored.reshape(-1), torch.cat([sa, sr], -1), copy


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "adamw":
        return _exact_adam(s)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    x = d["x"]
    if op == "linear_backward":
        gy = d["grad_y"]
        return torch.mm(gy, d["w"]), torch.mm(x.T, gy).T, torch.mv(gy.T, torch.ones_like(gy[:, 0]))
    if op in ("gated", "gated_train"):
        (wg, wu), (bg, bu) = d["w"], d["b"]
        a, u = torch.addmm(bg, x, wg.T), torch.addmm(bu, x, wu.T)
        if s["act"] == "silu":
            gate = torch.sigmoid(a)
            value, slope = a * gate, gate + a * gate * torch.sigmoid(-a)
        else:
            tail = torch.special.erfc(-a / math.sqrt(2.0)) / 2.0
            value, slope = a * tail, tail + a * torch.exp(-a * a / 2.0) / math.sqrt(2.0 * math.pi)
        h = value * u
        if op == "gated":
            return h
        da, du = d["grad_h"] * u * slope, d["grad_h"] * value
        return h, torch.mm(da, wg) + torch.mm(du, wu), torch.stack([torch.mm(da.T, x), torch.mm(du.T, x)]), torch.stack([da.sum(0), du.sum(0)])

    n = x.shape[-1]

    def unit_of(v):
        centred = v - v.sum(-1, keepdim=True) / n
        sigma = torch.sqrt((centred * centred).sum(-1, keepdim=True) / n + NORM_EPS)
        return centred / sigma, sigma

    def through(g, unit, sigma):
        return (g - g.sum(-1, keepdim=True) / n - unit * ((g * unit).sum(-1, keepdim=True) / n)) / sigma

    first, second = "gamma1" in d, "gamma2" in d
    by = d["scale"] if s["gate"] is None else d["gate"].reshape(-1, 1, 1) * d["scale"]
    branch = x
    if first:
        unit1, sigma1 = unit_of(x)
        branch = d["beta1"] + d["gamma1"] * unit1
    z = branch * by + d["residual"]
    y = None
    if second:
        unit2, sigma2 = unit_of(z.to(s["x"].dtype).double())    # what the norm reads is the stored sum
        y = d["beta2"] + d["gamma2"] * unit2
    if op == "end":
        return z, y
    flat = lambda v: v.reshape(-1, n).sum(0)
    gz, sums1, sums2 = d["grad_z"], (None, None), (None, None)
    if second:
        gz = gz + through(d["gamma2"] * d["grad_y"], unit2, sigma2)
        sums2 = flat(d["grad_y"] * unit2), flat(d["grad_y"])
    gb = gz * by
    gx = gb
    if first:
        gx = through(gb * d["gamma1"], unit1, sigma1)
        sums1 = flat(gb * unit1), flat(gb)
    grad_scale = flat(gz * branch * d["gate"].reshape(-1, 1, 1))
    grad_gate = (gz * branch).sum(1) @ d["scale"]
    return (z, y, gx, gz, grad_scale, grad_gate, *sums1, *sums2)
