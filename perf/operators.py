"""The operators that a network built from the library's calls needs around its convolutions, and the sizes they are measured at.

A case is one call of a user's program ("op"):
  gn_fwd    group normalisation with its activation, channels last, and the statistics its gradient needs
  gn_bwd    its gradients by input, scale and shift, from those statistics
  logp      log probabilities of given labels over rows of logits, entropies and the `top` largest alternatives of each row
  logp_bwd  the gradient by the logits, for incoming gradients of the log probabilities and of the entropies
  adamw     one AdamW step of a whole network's parameters (a flat vector with a tensor table), moments in 32 or in 8 bits

The 8-bit moments: t(x) = (bits of fp32 |x|) >> 20 counts steps of an eighth of a binade.  256 consecutive elements of a tensor
(the last ones of a tensor may be fewer) share s = t(largest) + 1; m is kept as its sign and c = t - s + 127, v as c = t - s + 255,
0 for what lies below (v > 0: at least 1, so that no denominator vanishes).  Rounding is stochastic: t = (bits + 16 r + 8) >> 20
with a 16-bit random number r, the low (m) and high (v) half of a Philox4x32-10 word of the call's seed.  What is rounded are
the fp32 moments beta m + (1 - beta) g and beta v + (1 - beta) (g g), one rounding per operation.
"""
import math

import numpy as np
import torch

own = False

ACTS = {"none": 0, "relu": 1, "silu": 2}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GN_EPS = 1e-5
BLOCK = 256


def _f32(x):
    """The fp32 value that a C float argument of x has."""
    return float(np.float32(x))


BETA1, BETA2, EPS, LR, DECAY, STEP = _f32(0.9), _f32(0.999), _f32(1e-8), _f32(1e-3), _f32(0.01), 100


def listed():
    return [
        # one small image's last feature map: a single call's latency
        {"name": "gn_fwd_one_image", "op": "gn_fwd", "B": 1, "H": 8, "W": 8, "C": 512, "groups": 32, "dtype": "bf16", "act": "relu"},
        # an odd handful of odd-sized images through a wide network in fp32: five channels a group
        {"name": "gn_fwd_wide_b13_f32", "op": "gn_fwd", "B": 13, "H": 33, "W": 33, "C": 160, "groups": 32, "dtype": "f32", "act": "silu"},
        # the widest feature map of ImageNet training at batch 256
        {"name": "gn_fwd_imagenet_b256", "op": "gn_fwd", "B": 256, "H": 56, "W": 56, "C": 256, "groups": 32, "dtype": "bf16", "act": "relu"},
        # CIFAR training, first stage: two channels a group
        {"name": "gn_bwd_cifar_b512", "op": "gn_bwd", "B": 512, "H": 32, "W": 32, "C": 64, "groups": 32, "dtype": "bf16", "act": "relu"},
        # behind the ImageNet stem, 85 images: large maps of few channels
        {"name": "gn_bwd_stem_b85", "op": "gn_bwd", "B": 85, "H": 112, "W": 112, "C": 64, "groups": 16, "dtype": "bf16", "act": "silu"},
        # evaluation of an ImageNet batch: top-5
        {"name": "logp_imagenet_b256", "op": "logp", "N": 256, "V": 1000, "ld": 1000, "top": 5, "dtype": "f32", "mask": "none"},
        # three rows over a long list of classes: a single answer's latency
        {"name": "logp_long_b3", "op": "logp", "N": 3, "V": 131075, "ld": 131075, "top": 20, "dtype": "bf16", "mask": "none"},
        # many rows over many classes, rows padded to whole vectors, some classes masked
        {"name": "logp_many", "op": "logp", "N": 2039, "V": 50021, "ld": 50024, "top": 8, "dtype": "bf16", "mask": "inf"},
        # the training direction in fp32, rows that start at any element
        {"name": "logp_bwd_many_f32", "op": "logp_bwd", "N": 1021, "V": 32771, "ld": 32771, "dtype": "f32", "mask": "none", "dentropy": True},
        # the toy network's parameters: launch latency
        {"name": "adamw_tinycnn", "op": "adamw", "net": "tinycnn", "bits": 32, "grads": "f32", "copy": False},
        # the headline network with its bf16 compute copy, 8-bit moments
        {"name": "adamw_resnet50_8bit", "op": "adamw", "net": "resnet50", "bits": 8, "grads": "f32", "copy": True},
        # the largest network, 32-bit moments
        {"name": "adamw_wrn34_32bit", "op": "adamw", "net": "wrn34_10", "bits": 32, "grads": "f32", "copy": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gn_fwd", "gn_bwd", "logp", "logp_bwd", "adamw"])
    if op in ("gn_fwd", "gn_bwd"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice([16, 24, 35, 64, 64, 120, 128, 160, 256, 320, 512, 640, 1024, 2048])
        groups = rng.choice([g for g in (1, 2, 4, 5, 8, 16, 32, C) if C % g == 0])
        most = (50_000_000 if dtype == "bf16" else 25_000_000) if op == "gn_bwd" else (150_000_000 if dtype == "bf16" else 75_000_000)
        H = _log_int(rng, 1, 112)
        W = max(1, H + rng.choice([0, 0, 0, -1, 1, 3]))
        B = _log_int(rng, 1, max(1, min(512, most // (H * W * C))))
        return {"op": op, "B": B, "H": H, "W": W, "C": C, "groups": groups, "dtype": dtype, "act": rng.choice(["none", "relu", "relu", "silu"])}
    if op in ("logp", "logp_bwd"):
        dtype = rng.choice(["bf16", "f32"])
        V = rng.choice([10, 1000, _log_int(rng, 2, 262144), _log_int(rng, 2, 262144)])
        N = _log_int(rng, 1, max(1, min(16384, (40_000_000 if dtype == "bf16" else 20_000_000) // V)))
        ld = rng.choice([V, V, (V + 7) // 8 * 8, V + rng.randint(1, 40)])
        case = {"op": op, "N": N, "V": V, "ld": ld, "dtype": dtype, "mask": rng.choice(["none", "none", "inf", "lowest"])}
        case.update({"top": rng.choice([0, 1, 5, rng.randint(2, 32)])} if op == "logp" else {"dentropy": rng.random() < 0.5})
        return case
    return {"op": op, "net": rng.choice(["tinycnn", "resnet18", "wrn28_10", "resnet50", "ragged"]), "bits": rng.choice([8, 8, 32]),
            "grads": rng.choice(["f32", "f32", "bf16"]), "copy": rng.random() < 0.5, "shift": rng.randint(0, 99999)}


# ---- tensor tables ---------------------------------------------------------------------------------------------------
def _table(case):
    """(elements, decayed) of every parameter tensor, in the library's order: weights decay, scales, shifts and biases do not."""
    net, out = case["net"], []

    def conv(cin, cout, k, norm=True):
        out.append((cout * k * k * cin, True))
        out.extend([(cout, False)] * (2 if norm else 1))

    if net == "tinycnn":
        conv(3, 16, 3, False)
        conv(16, 32, 3, False)
        out.extend([(320, True), (10, False)])
    elif net == "resnet50":
        conv(3, 64, 7)
        c = 64
        for w, depth in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(depth):
                conv(c, w, 1)
                conv(w, w, 3)
                conv(w, 4 * w, 1)
                if b == 0:
                    conv(c, 4 * w, 1)
                c = 4 * w
        out.extend([(2048 * 1000, True), (1000, False)])
    elif net == "ragged":   # many small tensors of every length, as a table of scales, shifts and little layers
        rng = np.random.default_rng(case["shift"])
        out = [(int(n), bool(i % 2)) for i, n in enumerate(np.exp(rng.uniform(0, math.log(30000), 700)).astype(int))]
    else:
        c, widths, depth = (64, (64, 128, 256, 512), 2) if net == "resnet18" else (16, (160, 320, 640), 5 if net == "wrn34_10" else 4)
        conv(3, c, 3)
        for w in widths:
            for _ in range(depth):
                conv(c, w, 3)
                conv(w, w, 3)
                if c != w:
                    conv(c, w, 1)
                c = w
        out.extend([(c * 10, True), (10, False)])
    if case.get("shift") and net != "ragged":   # another first layer: every later offset ragged
        out[0] = (out[0][0] - case["shift"] % max(1, out[0][0] - 1), True)
    return out


# ---- inputs ----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    s = {"case": dict(case), "seed": int(seed)}

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    if op in ("gn_fwd", "gn_bwd"):
        B, H, W, C, G = case["B"], case["H"], case["W"], case["C"], case["groups"]
        dtype = DTYPES[case["dtype"]]
        # a convolution's output: every channel with its own mean and spread
        x = normal(B, H, W, C).mul_(torch.exp(0.5 * normal(C))).add_(0.5 * normal(C)).to(dtype)
        s.update(x=x, gamma=1 + 0.2 * normal(C), beta=0.2 * normal(C))
        if op == "gn_bwd":
            s.update(dy=normal(B, H, W, C).mul_(1e-3).to(dtype))
            s["mean"], s["rstd"] = _group_stats(x, G)
        return s
    if op in ("logp", "logp_bwd"):
        N, V, ld = case["N"], case["V"], case["ld"]
        dtype = DTYPES[case["dtype"]]
        rows = normal(N, ld).mul_(3.0)
        if case["mask"] != "none":   # a tenth of the classes is not allowed
            rows[torch.rand(N, ld, device="cuda", generator=g) < 0.1] = -math.inf if case["mask"] == "inf" else torch.finfo(dtype).min
        labels = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32, generator=g)
        rows[torch.arange(N, device="cuda"), labels.long()] = 2.0 * normal(N) + 4.0   # the given label is a likely one
        s.update(logits=rows.to(dtype)[:, :V], labels=labels)
        if op == "logp_bwd":
            s["lse"], s["entropy"] = _row_stats(s["logits"].float())
            s.update(dlogp=normal(N).mul_(1.0 / N))
            s["dentropy"] = normal(N).mul_(0.1 / N) if case["dentropy"] else None
        return s
    table = _table(case)
    sizes = np.array([n for n, _ in table], np.int64)
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    d = int(offsets[-1])
    s.update(offsets_host=offsets, offsets=torch.from_numpy(offsets).cuda(), decay=torch.tensor([DECAY if w else 0.0 for _, w in table], device="cuda"))
    tensor = torch.repeat_interleave(torch.arange(len(table), device="cuda"), torch.from_numpy(sizes).cuda())
    scale = torch.pow(10.0, -1.0 - 3.0 * torch.rand(len(table), device="cuda", generator=g))[tensor]   # gradients of very different size by layer
    s["theta"] = normal(d).mul_(0.05)
    spread = scale * torch.exp(normal(d))                                                           # and by element
    s["grads"] = (spread * normal(d)).to(DTYPES[case["grads"]])
    m, v = 0.3 * spread * normal(d), spread * spread * torch.exp(0.3 * normal(d))
    s["t"] = STEP
    s["copy"] = s["theta"].to(torch.bfloat16) if case["copy"] else None
    if case["bits"] == 32:
        s.update(m=m, v=v, scales=None)
        return s
    s["blocks"] = _blocks(offsets)
    s["slots"] = d // BLOCK + len(table)
    word = torch.zeros(d, dtype=torch.int64, device="cuda")
    s["m"], sm = _encode(m, word, s["blocks"], s["slots"], 127)
    s["v"], sv = _encode(v, word, s["blocks"], s["slots"], 255)
    s["scales"] = torch.stack([sm, sv], 1).to(torch.int16).contiguous()
    return s


# ---- plain forms: 32 bits, one rounding at the end --------------------------------------------------------------------
def _group_stats(x, G):
    """Mean and 1 / standard deviation of every image's groups, fp32 [B, G]."""
    xg = x.float().view(x.shape[0], -1, G, x.shape[3] // G)
    mean = xg.mean(dim=(1, 3))
    var = (xg - mean[:, None, :, None]).square().mean(dim=(1, 3))
    return mean, 1.0 / torch.sqrt(var + GN_EPS)


def _normalised(x, mean, rstd, gamma, beta):
    """xhat and z = xhat * gamma + beta, one rounding per operation."""
    B, G = mean.shape
    xg = x.float().view(B, -1, G, x.shape[3] // G)
    xhat = (xg - mean[:, None, :, None]) * rstd[:, None, :, None]
    return xhat, xhat * gamma.view(G, -1) + beta.view(G, -1)


def _plain_gn_fwd(s):
    x, act = s["x"], s["case"]["act"]
    mean, rstd = _group_stats(x, s["case"]["groups"])
    _, z = _normalised(x, mean, rstd, s["gamma"], s["beta"])
    if act == "relu":
        z = torch.clamp_min(z, 0.0)
    elif act == "silu":
        z = z / (1.0 + torch.exp(-z))
    return z.view(x.shape).to(x.dtype), mean, rstd


def _plain_gn_bwd(s):
    x, act, mean, rstd = s["x"], s["case"]["act"], s["mean"], s["rstd"]
    B, G = mean.shape
    xhat, z = _normalised(x, mean, rstd, s["gamma"], s["beta"])
    dz = s["dy"].float().view(xhat.shape)
    if act == "relu":
        dz = dz * (z > 0)
    elif act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    dgamma, dbeta = (dz * xhat).sum(dim=(0, 1)).view(-1), dz.sum(dim=(0, 1)).view(-1)
    h = dz * s["gamma"].view(G, -1)
    c1, c2 = h.mean(dim=(1, 3), keepdim=True), (h * xhat).mean(dim=(1, 3), keepdim=True)
    dx = (h - c1 - xhat * c2) * rstd[:, None, :, None]
    return dx.view(x.shape).to(x.dtype), dgamma, dbeta


def _row_stats(x):
    """log sum exp and entropy of every row."""
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1)
    weighted = torch.where(e > 0, (x - top) * e, 0.0).sum(dim=1)
    return top[:, 0] + torch.log(total), torch.log(total) - weighted / total


def _plain_logp(s):
    x, k = s["logits"].float(), s["case"]["top"]
    lse, entropy = _row_stats(x)
    logp = torch.gather(x, 1, s["labels"].long()[:, None])[:, 0] - lse
    if k == 0:
        return logp, entropy, lse
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k].to(torch.int32)
    index = torch.where(value > -math.inf, index, -1)
    value = value - lse[:, None]
    if k > x.shape[1]:   # fewer classes than asked for
        pad = (0, k - x.shape[1])
        value, index = torch.nn.functional.pad(value, pad, value=-math.inf), torch.nn.functional.pad(index, pad, value=-1)
    return logp, entropy, lse, value, index


def _plain_logp_bwd(s):
    x = s["logits"].float()
    logq = x - s["lse"][:, None]
    p = torch.exp(logq)
    onehot = torch.arange(x.shape[1], device=x.device)[None, :] == s["labels"][:, None]
    dx = s["dlogp"][:, None] * (onehot.float() - p)
    if s["dentropy"] is not None:
        dx = dx - s["dentropy"][:, None] * torch.where(p > 0, p * (logq + s["entropy"][:, None]), 0.0)
    return dx.to(s["logits"].dtype)


def _philox(block, seed, stream):
    """The four words of Philox4x32-10 for int64 counters `block`, key `seed`."""
    low = 0xFFFFFFFF

    def mul(a, c):   # 32 x 32 -> (high, low), by 16-bit halves: int64 has no unsigned 64-bit product
        p0, p1 = a * (c & 0xFFFF), a * (c >> 16)
        mid = (p0 >> 16) + p1
        return mid >> 16, ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)

    c0, c1 = block & low, block >> 32
    c2, c3 = torch.full_like(block, stream), torch.zeros_like(block)
    ka, kb = seed & low, (seed >> 32) & low
    for _ in range(10):
        h0, l0 = mul(c0, 0xD2511F53)
        h1, l1 = mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ ka, l1, h0 ^ c3 ^ kb, l0
        ka, kb = (ka + 0x9E3779B9) & low, (kb + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], 1)


def _blocks(offsets):
    """Of every element: its slot (tensor t's blocks are the slots from offsets[t] // 256 + t on) and its place in the block."""
    off = torch.from_numpy(offsets).cuda()
    sizes = off[1:] - off[:-1]
    t = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), sizes)
    local = torch.arange(int(offsets[-1]), device="cuda") - off[t]
    return (off[t] // BLOCK + t + local // BLOCK).to(torch.int32), (local % BLOCK).to(torch.int16)


def _random_words(s):
    """The random word of every element: word place % 4 of counter slot * 64 + place / 4, stream 2, key = the call's seed."""
    slot, place = s["blocks"]
    words = _philox(torch.arange(s["slots"] * (BLOCK // 4), device="cuda"), s["seed"] * 65536 + s["t"], 2).view(-1)
    return words[slot.long() * BLOCK + place]


def _encode(x, word16, blocks, slots, top):
    """Codes (uint8) and the blocks' s (int64)."""
    slot = blocks[0].long()
    bits = x.abs().view(torch.int32).long()
    largest = torch.zeros(slots, dtype=torch.int64, device=x.device).scatter_reduce(0, slot, bits, "amax")
    scale = (largest >> 20) + 1
    t = ((bits + 16 * word16 + 8) >> 20).clamp_max(0x7F7)
    c = (t - scale[slot] + top).clamp_min(0)
    if top == 255:
        c = torch.where(bits > 0, c.clamp_min(1), c)
    else:
        c = c | torch.where(x < 0, 128, 0)
    return c.to(torch.uint8), scale


def _decode(code, scale, blocks, top):
    c = code.long()
    sign = torch.where(c > top, -1.0, 1.0)
    c = c & top
    t = c + scale.long()[blocks[0].long()] - top
    bits = torch.where((c > 0) & (t > 0), t << 20, 0)
    return sign * bits.to(torch.int32).view(torch.float32)


def _plain_adamw(s):
    t, eight = s["t"], s["scales"] is not None
    g, theta = s["grads"].float(), s["theta"]
    m = _decode(s["m"], s["scales"][:, 0], s["blocks"], 127) if eight else s["m"]
    v = _decode(s["v"], s["scales"][:, 1], s["blocks"], 255) if eight else s["v"]
    m = BETA1 * m + _f32(1 - BETA1) * g
    v = BETA2 * v + _f32(1 - BETA2) * (g * g)
    u = (m * (1 / (1 - BETA1 ** t))) / (torch.sqrt(v * (1 / (1 - BETA2 ** t))) + EPS)
    decay = torch.repeat_interleave(s["decay"], s["offsets"][1:] - s["offsets"][:-1])
    theta.sub_(LR * (u + decay * theta))
    if s["copy"] is not None:
        s["copy"].copy_(theta)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return [x for x in (theta, s["m"], s["v"], s["copy"]) if x is not None]
    word = _random_words(s)
    s["m"], sm = _encode(m, word & 0xFFFF, s["blocks"], s["slots"], 127)
    s["v"], sv = _encode(v, word >> 16, s["blocks"], s["slots"], 255)
    s["scales"].copy_(torch.stack([sm, sv], 1))
    m, v = _decode(s["m"], sm, s["blocks"], 127), _decode(s["v"], sv, s["blocks"], 255)
    return [x for x in (theta, m, v, s["copy"]) if x is not None]


# ---- the framework's calls ---------------------------------------------------------------------------------------------
def _own(s):
    import paper_2206_06257_amd as dat
    case, op = s["case"], s["case"]["op"]
    if op == "gn_fwd":
        return dat.group_norm_forward(s["x"], s["gamma"], s["beta"], case["groups"], ACTS[case["act"]], eps=GN_EPS)
    if op == "gn_bwd":
        return dat.group_norm_backward(s["x"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], case["groups"], ACTS[case["act"]])
    if op == "logp":
        out = dat.log_probs(s["logits"], s["labels"], top=case["top"])
        return out if case["top"] else out[:3]
    if op == "logp_bwd":
        return dat.log_probs_backward(s["logits"], s["labels"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"])
    dat.adamw_update(s["theta"], s["grads"], s["m"], s["v"], s["offsets"], LR, s["t"], scales=s["scales"], seed=s["seed"] * 65536 + s["t"],
                     beta1=BETA1, beta2=BETA2, eps=EPS, decay=s["decay"], theta_bf16=s["copy"])
    m, v = (s["m"], s["v"]) if s["scales"] is None else dat.adamw_moments(s["m"], s["v"], s["scales"], s["offsets"])
    return [x for x in (s["theta"], m, v, s["copy"]) if x is not None]


PLAIN = {"gn_fwd": _plain_gn_fwd, "gn_bwd": _plain_gn_bwd, "logp": _plain_logp, "logp_bwd": _plain_logp_bwd, "adamw": _plain_adamw}


def run(s):
    s["t"] = s.get("t", 0) + 1
    if own:
        return _own(s)
    return PLAIN[s["case"]["op"]](s)


# ---- the least work of a case ------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    width = 2 if case.get("dtype") == "bf16" else 4
    if op in ("gn_fwd", "gn_bwd"):
        n, C, stats = case["B"] * case["H"] * case["W"] * case["C"], case["C"], 2 * case["B"] * case["groups"]
        if op == "gn_fwd":
            return {"bytes": 2 * width * n + 4 * (2 * C + stats), "flops": 9 * n}
        return {"bytes": 3 * width * n + 4 * (4 * C + stats), "flops": 18 * n}
    if op in ("logp", "logp_bwd"):
        n, N = case["N"] * case["V"], case["N"]
        if op == "logp":
            return {"bytes": width * n + 4 * N * (4 + 2 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * width * n + 4 * N * 5, "flops": 8 * n}
    sizes = [n for n, _ in _table(case)]
    d = sum(sizes)
    each = 8 + (4 if case["grads"] == "f32" else 2) + (2 if case["copy"] else 0) + (16 if case["bits"] == 32 else 4 + 8)   # 8 bit: and the values returned
    scales = 8 * sum((n + BLOCK - 1) // BLOCK for n in sizes) if case["bits"] == 8 else 0
    return {"bytes": each * d + scales + 12 * len(sizes), "flops": 16 * d}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def _kept(s):
    """Where the forward pass let values through: its z is the fp32 number ((x - mean) rstd) gamma + beta, one rounding per
    operation (products and sums of fp32 numbers in 64 bits, then rounded)."""
    G = s["case"]["groups"]
    mean, rstd = (torch.repeat_interleave(s[k], s["x"].shape[3] // G, dim=1)[:, None, None, :].double() for k in ("mean", "rstd"))
    z = (s["x"].double() - mean).float().double()
    z = (z * rstd).float().double()
    z = (z * s["gamma"].double()).float().double()
    return (z + s["beta"].double()).float() > 0


def _exact_gn(s, backward):
    case = s["case"]
    x = s["x"].double().requires_grad_(backward)
    gamma, beta = (s[k].double().requires_grad_(backward) for k in ("gamma", "beta"))
    B, H, W, C = x.shape
    with torch.set_grad_enabled(backward):
        rows = x.reshape(B, H * W, case["groups"], -1).transpose(1, 2).reshape(B, case["groups"], -1)
        var, mean = torch.var_mean(rows, dim=2, unbiased=False)
        rstd = (var + GN_EPS) ** -0.5
        z = ((rows - mean[..., None]) * rstd[..., None]).reshape(B, case["groups"], H * W, -1).transpose(1, 2).reshape(B, H, W, C) * gamma + beta
        y = z * (_kept(s) if backward else z > 0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
    if not backward:
        return y, mean, rstd
    return torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())


def _exact_logp(s, backward):
    x, k = s["logits"].double(), s["case"].get("top", 0)
    logq = x - torch.logsumexp(x, 1, keepdim=True)
    p = logq.exp()
    plogp = torch.where(p > 0, p * logq, 0.0)
    entropy = -plogp.sum(1)
    rows = torch.arange(x.shape[0], device=x.device)
    if backward:
        dx = -s["dlogp"].double()[:, None] * p
        dx[rows, s["labels"].long()] += s["dlogp"].double()
        if s["dentropy"] is not None:
            dx -= s["dentropy"].double()[:, None] * (plogp + p * entropy[:, None])
        return dx
    out = [logq[rows, s["labels"].long()], entropy, torch.logsumexp(x, 1)]
    if k:
        order = np.argsort(-x.cpu().numpy(), axis=1, kind="stable")[:, :k] if x.numel() < 20_000_000 else torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k].cpu().numpy()
        index = torch.from_numpy(np.ascontiguousarray(order)).cuda()
        value = torch.full((x.shape[0], k), -math.inf, dtype=torch.float64, device=x.device)
        value[:, :index.shape[1]] = torch.gather(logq, 1, index)
        whole = torch.full((x.shape[0], k), -1, dtype=torch.int32, device=x.device)
        whole[:, :index.shape[1]] = index.int()
        out += [value, torch.where(value > -math.inf, whole, -1)]
    return out


def _exact_code(x, r, block, slots, top):
    """The stored value of x >= 0 in 64 bits: steps of an eighth of a binade above 2^-127, rounded by r in [0, 1)."""
    mantissa, exponent = torch.frexp(x)          # mantissa in [0.5, 1)
    steps = torch.where(x > 0, 8.0 * (exponent.double() + 126.0) + 8.0 * (2.0 * mantissa - 1.0), 0.0)
    largest = torch.zeros(slots, dtype=torch.float64, device=x.device).index_reduce_(0, block, steps, "amax")
    s = torch.floor(largest[block]) + 1.0
    kept = torch.floor(steps + r)
    lowest = s - top + 1.0                       # code 1
    kept = torch.where(kept < lowest, torch.where(x > 0, lowest, 0.0) if top == 255 else torch.zeros_like(kept), kept)
    power = torch.floor(kept / 8.0)
    return torch.where((kept > 0) & (x > 0), torch.ldexp(1.0 + (kept / 8.0 - power), (power - 127.0).int()), 0.0)


def _exact_adamw(s):
    eight, t = s["scales"] is not None, s["t"] + 1
    lr, b1, b2, eps = (torch.tensor(v, dtype=torch.float64, device="cuda") for v in (LR, BETA1, BETA2, EPS))
    m = (_decode(s["m"], s["scales"][:, 0], s["blocks"], 127) if eight else s["m"]).double()
    v = (_decode(s["v"], s["scales"][:, 1], s["blocks"], 255) if eight else s["v"]).double()
    g, theta = s["grads"].double(), s["theta"].double()
    if eight:   # the code is that of the moment as an fp32 number, one rounding per operation: products and sums of fp32 numbers in 64 bits, then rounded
        c1, c2 = (torch.tensor(_f32(1 - b), dtype=torch.float64, device="cuda") for b in (BETA1, BETA2))
        m = ((b1 * m).float().double() + (c1 * g).float().double()).float().double()
        v = ((b2 * v).float().double() + (c2 * (g * g).float().double()).float().double()).float().double()
    else:
        m = torch.lerp(g, m, b1)
        v = torch.lerp(g ** 2, v, b2)
    step = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    table = torch.repeat_interleave(s["decay"].double(), torch.diff(s["offsets"]))
    theta = theta * (1 - lr * table) - lr * step
    if eight:
        s["t"] = t
        word, block = _random_words(s), s["blocks"][0].long()
        m = torch.sign(m) * _exact_code(m.abs(), ((word & 0xFFFF).double() + 0.5) / 65536.0, block, s["slots"], 127)
        v = _exact_code(v, ((word >> 16).double() + 0.5) / 65536.0, block, s["slots"], 255)
    return [theta, m, v] + ([theta] if s["copy"] is not None else [])


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("gn_fwd", "gn_bwd"):
        return _exact_gn(s, op == "gn_bwd")
    if op in ("logp", "logp_bwd"):
        return _exact_logp(s, op == "logp_bwd")
    return _exact_adamw(s)
