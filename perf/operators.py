"""Operators of a training step and its evaluation, as a user of `binding.py` calls them, each beside its plain form.

  group_norm  group normalisation of an NHWC activation with an activation function behind it: forward, backward, or both
  grad_norm   the 2-norm of all gradients of a network and the factor that clips it
  adamw       one AdamW step over all tensors of a network, its two states in 32 bits or as 8-bit floats with a scale per 256
  logprobs    log-probability of a given class per row, entropy, and the likeliest classes; with gradients where asked for

A network's tensors lie in one arena per kind (gradients, weights, states), each tensor from a multiple of 4096 elements on, with
zeros behind it; outputs are whole arenas.  Plain forms are elementary torch operations in 32 bits.
"""
import math

import torch

own = False

PAGE = 4096      # elements: where a tensor may begin in an arena
BLOCK = 256      # elements that share a scale of an 8-bit state
EPS = 1e-5       # of group norm
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=100, seed=20240607)
MAX_NORM = 1.0


def listed():
    return [
        # a late layer at the batch that 32-way strong scaling leaves, in inference: the smallest call, launches and latency
        dict(name="gn_fwd_14_512_n1", kind="group_norm", way="fwd", n=1, h=14, w=14, c=512, groups=32, dtype="bf16", act="relu"),
        # the first layers at the whole batch: the largest activation, groups of two channels
        dict(name="gn_fwd_224_64_n32", kind="group_norm", way="fwd", n=32, h=224, w=224, c=64, groups=32, dtype="bf16", act="relu"),
        # a middle layer at a middle batch that keeps its ReLU: the saved output masks the gradient
        dict(name="gn_bwd_28_512_n8", kind="group_norm", way="bwd", n=8, h=28, w=28, c=512, groups=32, dtype="bf16", act="relu"),
        # a residual stage at the whole batch, smooth activation
        dict(name="gn_bwd_56_256_n32", kind="group_norm", way="bwd", n=32, h=56, w=56, c=256, groups=32, dtype="bf16", act="silu"),
        # an image and groups of ten channels that no vector divides, reference precision, both directions
        dict(name="gn_both_73_80_n4_f32", kind="group_norm", way="both", n=4, h=73, w=73, c=80, groups=8, dtype="f32", act="silu"),
        # clipping the gradients of one residual block, and of a whole VGG-16
        dict(name="norm_block", kind="grad_norm", net="block", width=64, classes=0),
        dict(name="norm_vgg16", kind="grad_norm", net="vgg16", width=64, classes=1000),
        # optimizer step: one residual block, a whole VGG-16, and the 161 tensors of a ResNet-50 with states in 8 bits
        dict(name="adamw_block", kind="adamw", net="block", width=64, classes=0, bits=32),
        dict(name="adamw_vgg16", kind="adamw", net="vgg16", width=64, classes=1000, bits=32),
        dict(name="adamw8_resnet50", kind="adamw", net="resnet50", width=64, classes=1000, bits=8),
        # the next token of one sequence with its alternatives
        dict(name="logprobs_1x131072", kind="logprobs", rows=1, classes=131072, top=20, dtype="bf16", mask=False, grad=False),
        # scoring a batch of tokens in training: odd sizes, a padded vocabulary, gradients of log-probability and entropy
        dict(name="logprobs_2047x50001", kind="logprobs", rows=2047, classes=50001, top=5, dtype="bf16", mask=True, grad=True),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["group_norm", "group_norm", "grad_norm", "adamw", "adamw", "logprobs", "logprobs"])
    if kind == "group_norm":
        while True:
            per = rng.choice([1, 2, 4, 6, 8, 10, 12, 16, 20, 24, 32, 40, 64])
            groups = rng.choice([1, 2, 5, 8, 16, 32, 32, 32])
            h = _spread(rng, 1, 224)
            case = dict(kind=kind, way=rng.choice(["fwd", "bwd", "both"]), n=_spread(rng, 1, 32), h=h, w=max(1, h + rng.randint(-h // 8, h // 8)),
                        c=per * groups, groups=groups, dtype=rng.choice(["bf16", "bf16", "f32"]))
            # a pass of both directions masks by its own output; a smooth activation lets the two forms be compared there
            case["act"] = rng.choice(["none", "silu"] if case["way"] == "both" else ["none", "relu", "relu_front", "silu"])
            # a group of a few values has no gradient to compare: normalised, they hardly depend on their inputs
            if case["h"] * case["w"] * per >= 8 and case["n"] * case["h"] * case["w"] * case["c"] <= 50_000_000:
                return case
    if kind in ("grad_norm", "adamw"):
        net = rng.choice(["block", "block", "resnet50", "vgg16"])
        width = {"block": _spread(rng, 8, 512), "resnet50": _spread(rng, 8, 96), "vgg16": _spread(rng, 4, 60)}[net]
        case = dict(kind=kind, net=net, width=width, classes=0 if net == "block" else rng.choice([10, 100, 365, 1000]))
        if kind == "adamw":
            case["bits"] = rng.choice([32, 8])
        return case
    while True:
        case = dict(kind=kind, rows=_spread(rng, 1, 4096), classes=_spread(rng, 10, 140000), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    mask=rng.random() < 0.4, grad=rng.random() < 0.5)
        case["top"] = min(case["classes"], rng.choice([0, 1, 5, 5, 20, 64]))
        if case["rows"] * case["classes"] <= 90_000_000:
            return case


# ---- shapes -------------------------------------------------------------------------------------------------------

def _tensors(case):
    """[(elements, whether weight decay applies)] of a network's tensors in order: weights decay, biases and norms do not."""
    w, net, out = case["width"], case["net"], []

    def conv(c, k, r, norm):
        out.append((k * r * r * c, True))
        out.extend([(k, False)] * (2 if norm else 1))

    if net == "block":          # one residual block: 1x1, 3x3, 1x1 with group norms
        conv(4 * w, w, 1, True), conv(w, w, 3, True), conv(w, 4 * w, 1, True)
    elif net == "vgg16":        # 13 convolutions with bias, three dense layers
        c = 3
        for k in (1, 1, 2, 2, 4, 4, 4, 8, 8, 8, 8, 8, 8):
            conv(c, k * w, 3, False)
            c = k * w
        for i, o in ((49 * c, 64 * w), (64 * w, 64 * w), (64 * w, case["classes"])):
            out += [(i * o, True), (o, False)]
    else:                       # the residual network of 50 layers: stem, 3 + 4 + 6 + 3 blocks, one dense layer
        conv(3, w, 7, True)
        c = w
        for stage, blocks in enumerate((3, 4, 6, 3)):
            m = w << stage
            for b in range(blocks):
                conv(c, m, 1, True), conv(m, m, 3, True), conv(m, 4 * m, 1, True)
                if b == 0:
                    conv(c, 4 * m, 1, True)
                c = 4 * m
        out += [(c * case["classes"], True), (case["classes"], False)]
    return out


def _starts(tensors):
    at, total = [], 0
    for n, _ in tensors:
        at.append(total)
        total += -(-n // PAGE) * PAGE
    return at, total


# ---- inputs -------------------------------------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case.get("dtype") == "bf16" else torch.float32


class _Gen:
    def __init__(self, seed):
        self.dev = torch.device("cuda:0")
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.dev, dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev, dtype=torch.float32)

    def whole(self, below, *shape):
        return torch.randint(0, below, shape, generator=self.gen, device=self.dev, dtype=torch.int32)


def _inputs(case, seed):
    g = _Gen(seed)
    s = {"case": case}
    if case["kind"] == "group_norm":
        n, h, w, c, gr = (case[k] for k in ("n", "h", "w", "c", "groups"))
        # what a convolution gives: channels with an offset and a spread of their own
        x = g.normal(n, h, w, c)
        x.mul_(0.5 + g.uniform(c)).add_(g.normal(c) * 0.5)
        s["x"] = x.to(_type(case))
        s["gamma"], s["beta"] = 1 + 0.2 * g.normal(c), 0.2 * g.normal(c)
        if case["way"] != "fwd":
            dy = g.normal(n, h, w, c)
            if case["act"] == "relu_front":   # the layer behind has masked the gradient
                dy.mul_(g.uniform(n, h, w, c) < 0.5)
            s["dy"] = dy.to(_type(case))
            del dy
        if case["way"] == "bwd":              # kept from the forward pass
            xf = s["x"].float().view(n, h * w, gr, c // gr)
            s["mean"] = xf.mean(dim=(1, 3))
            s["rstd"] = 1 / torch.sqrt((xf - s["mean"].view(n, 1, gr, 1)).square().mean(dim=(1, 3)) + EPS)
            if case["act"] == "relu":
                u = ((xf - s["mean"].view(n, 1, gr, 1)) * s["rstd"].view(n, 1, gr, 1)).view(n, h, w, c) * s["gamma"] + s["beta"]
                s["y"] = torch.relu(u).to(_type(case))
    elif case["kind"] in ("grad_norm", "adamw"):
        tensors = _tensors(case)
        at, total = _starts(tensors)
        sizes = torch.tensor([n for n, _ in tensors], device=g.dev)
        pages = (sizes + PAGE - 1) // PAGE
        # gradients of a size of their own in every tensor; zeros behind each tensor's end
        page_scale = torch.repeat_interleave(1e-3 * torch.exp(g.normal(len(tensors))), pages)
        used = torch.ones(total, dtype=torch.bool, device=g.dev)
        for (n, _), a in zip(tensors, at):
            used[a + n:a + -(-n // PAGE) * PAGE] = False
        keep = used.view(-1, PAGE)
        s["g"] = ((g.normal(total).view(-1, PAGE) * page_scale[:, None]) * keep).view(-1)
        if case["kind"] == "adamw":
            s["w"] = (g.normal(total).view(-1, PAGE) * 0.05 * keep).view(-1)
            s["w16"] = s["w"].to(torch.bfloat16)
            m = (g.normal(total).view(-1, PAGE) * (0.3 * page_scale[:, None]) * keep).view(-1)
            v = ((0.02 + g.uniform(total)).view(-1, PAGE) * (0.1 * page_scale.square()[:, None]) * keep).view(-1)   # 100 steps at beta2 = 0.999
            if case["bits"] == 32:
                s["m"], s["v"] = m, v
            else:
                s["m"], s["ms"] = _to_8(m)
                s["v"], s["vs"] = _to_8(torch.sqrt(v))
            del m, v
            s["scale"] = torch.tensor([0.75], device=g.dev)
            s["decay"] = torch.repeat_interleave(torch.tensor([0.05 if d else 0.0 for _, d in tensors], device=g.dev), pages)
    else:
        r, c = case["rows"], case["classes"]
        z = g.normal(r, c).mul_(3.0)
        if case["mask"]:   # the end of a padded vocabulary, and a few forbidden classes of every row
            z[:, c - c // 50:] = -math.inf
            z.masked_fill_(g.uniform(r, c) < 0.01, -math.inf)
        s["z"] = z.to(_type(case))
        s["ids"] = g.whole(max(1, c - c // 50), r)
        if case["grad"]:
            s["dlogp"], s["dent"] = g.normal(r) / r, g.normal(r) * (0.01 / r)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps between its steps: descriptors, tables of its tensors, outputs and workspaces."""
    from paper_2112_10065_amd import binding as dp
    case, dev = s["case"], torch.device("cuda:0")
    s["dp"] = dp

    def empty(shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=dev)

    def workspace(nbytes):
        return empty(max(int(nbytes), 16), torch.uint8)

    io = dp.DP_BF16 if _type(case) == torch.bfloat16 else dp.DP_F32
    if case["kind"] == "group_norm":
        flags = {"none": 0, "relu": dp.DP_RELU, "relu_front": dp.DP_RELU, "silu": dp.DP_SILU}[case["act"]]
        s["desc"] = d = dp.group_norm_desc(case["n"], case["h"], case["w"], case["c"], case["groups"], io, flags, EPS)
        s["ws"] = workspace(max(dp.dp_group_norm_workspace_bytes(d, p) for p in (dp.DP_PASS_FWD, dp.DP_PASS_DGRAD)))
        if case["way"] != "bwd":
            s["y"] = torch.empty_like(s["x"])
            s["mean"], s["rstd"] = empty((case["n"], case["groups"])), empty((case["n"], case["groups"]))
        if case["way"] != "fwd":
            s["dx"], s["dgamma"], s["dbeta"] = torch.empty_like(s["x"]), empty(case["c"]), empty(case["c"])
    elif case["kind"] == "logprobs":
        r, k = case["rows"], case["top"]
        s["desc"] = d = dp.logprobs_desc(r, case["classes"], k, io)
        s["ws"] = workspace(dp.dp_logprobs_workspace_bytes(d))
        s["out"] = [empty(r), empty(r), empty(r), empty((r, k)), empty((r, k), torch.int32)]
        s["dz"] = torch.empty_like(s["z"]) if case["grad"] else None
    else:
        tensors = _tensors(case)
        at, _ = _starts(tensors)
        params = []
        for (n, decays), a in zip(tensors, at):
            p = dict(grad=s["g"][a:a + n])
            if case["kind"] == "adamw":
                p.update(w32=s["w"][a:a + n], w_bf16=s["w16"][a:a + n], m=s["m"][a:a + n], v=s["v"][a:a + n], weight_decay=0.05 if decays else 0.0)
                if case["bits"] == 8:
                    b = slice(a // BLOCK, a // BLOCK + -(-n // BLOCK))
                    p.update(m_scale=s["ms"][b], v_scale=s["vs"][b])
            params.append(p)
        s["params"] = dp.param_list(params, dp.DP_STATE_Q8 if case.get("bits") == 8 else dp.DP_STATE_F32)
        if case["kind"] == "grad_norm":
            s["norm"] = empty(2)
            s["ws"] = workspace(dp.dp_grad_norm_workspace_bytes(s["params"]))
        else:
            s["hyper"] = dp.adamw_hyper(**HYPER)


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    return {"group_norm": _own_group_norm, "grad_norm": _own_grad_norm, "adamw": _own_adamw, "logprobs": _own_logprobs}[s["case"]["kind"]](s) if own else \
        {"group_norm": _plain_group_norm, "grad_norm": _plain_grad_norm, "adamw": _plain_adamw, "logprobs": _plain_logprobs}[s["case"]["kind"]](s)


def _own_group_norm(s):
    dp, way, out = s["dp"], s["case"]["way"], []
    if way != "bwd":
        dp.dp_group_norm_fwd(s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], s["ws"])
        out += [s["y"], s["mean"], s["rstd"]]
    if way != "fwd":
        y_saved = s["y"] if s["case"]["act"] == "relu" else None
        dp.dp_group_norm_bwd(s["desc"], s["x"], s["dy"], y_saved, s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        out += [s["dx"], s["dgamma"], s["dbeta"]]
    return out


def _plain_group_norm(s):
    case, x, out = s["case"], s["x"].float(), []
    n, h, w, c, gr = (case[k] for k in ("n", "h", "w", "c", "groups"))
    act, shape, each = case["act"], (n, h, w, c), (n, 1, gr, 1)
    x = x.view(n, h * w, gr, c // gr)
    if case["way"] == "bwd":
        mean, rstd = s["mean"], s["rstd"]
    else:
        mean = x.mean(dim=(1, 3))
        rstd = 1 / torch.sqrt((x - mean.view(each)).square().mean(dim=(1, 3)) + EPS)
    xhat = (x - mean.view(each)) * rstd.view(each)
    u = xhat.view(shape) * s["gamma"] + s["beta"]
    if case["way"] != "bwd":
        y = torch.relu(u) if act in ("relu", "relu_front") else u / (1 + torch.exp(-u)) if act == "silu" else u
        out += [y.to(s["x"].dtype), mean, rstd]
    if case["way"] != "fwd":
        g = s["dy"].float()
        if act == "relu":
            g = g * (s["y"] > 0)
        elif act == "silu":
            q = 1 / (1 + torch.exp(-u))
            g = g * (q * (1 + u * (1 - q)))
        dgamma, dbeta = (g * xhat.view(shape)).sum(dim=(0, 1, 2)), g.sum(dim=(0, 1, 2))
        t = (g * s["gamma"]).view(n, h * w, gr, c // gr)
        dx = (t - t.mean(dim=(1, 3), keepdim=True) - xhat * (t * xhat).mean(dim=(1, 3), keepdim=True)) * rstd.view(each)
        out += [dx.view(shape).to(s["x"].dtype), dgamma, dbeta]
    return out


def _own_grad_norm(s):
    s["dp"].dp_grad_norm(s["params"], MAX_NORM, s["norm"], s["ws"])
    return s["norm"]


def _plain_grad_norm(s):
    norm = torch.sqrt(s["g"].square().sum())
    return torch.stack([norm, torch.clamp(MAX_NORM / norm, max=1.0)])


def _own_adamw(s):
    s["dp"].dp_adamw_step(s["params"], s["hyper"], s["scale"])
    return [s[k] for k in ("w", "w16", "m", "v", "ms", "vs") if k in s]


def _plain_adamw(s):
    h, q8 = HYPER, s["case"]["bits"] == 8
    g = s["g"] * s["scale"]
    m = _from_8(s["m"], s["ms"]) if q8 else s["m"]
    v = _from_8(s["v"], s["vs"]).square() if q8 else s["v"]
    m.mul_(h["beta1"]).add_(g * (1 - h["beta1"]))
    v.mul_(h["beta2"]).add_(g.square() * (1 - h["beta2"]))
    bc1, bc2 = 1 - h["beta1"] ** h["step"], 1 - h["beta2"] ** h["step"]
    root = torch.sqrt(v)
    update = m / (root * (1 / math.sqrt(bc2)) + h["eps"])
    w = s["w"].view(-1, PAGE)
    w.mul_(1 - h["lr"] * s["decay"][:, None])
    s["w"].sub_(update * (h["lr"] / bc1))
    s["w16"].copy_(s["w"])
    if q8:
        bits = _random16(s["g"].numel(), h["seed"], s["g"].device)
        _into_8(m, bits[0], s["m"], s["ms"], False)
        _into_8(root, bits[1], s["v"], s["vs"], True)
    return [s[k] for k in ("w", "w16", "m", "v", "ms", "vs") if k in s]


def _from_8(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _to_8(x):
    """Nearest 8-bit floats, the largest of each block at 448; and the blocks' scales."""
    scale = x.view(-1, BLOCK).abs().amax(dim=1) / 448
    r = torch.where(scale[:, None] > 0, x.view(-1, BLOCK) / scale[:, None], 0.0)
    return r.clamp_(-448, 448).view(-1).to(torch.float8_e4m3fn), scale


def _into_8(x, u, code, scale, positive):
    """The same with a random choice of the two nearest, up where the 16 random bits u say so; a positive value stays positive."""
    x = x.view(-1, BLOCK)
    most = x.abs().amax(dim=1)
    scale.copy_(most / 448)
    a = torch.where(most[:, None] > 0, x.abs() * (448 / most[:, None]), 0.0).view(-1)
    normal = ((a.view(torch.int32) + (u << 4)) >> 20) - 960
    small = torch.floor(a * 512 + u.float() * (1 / 65536)).int()
    c = torch.where(a < 2 ** -6, small, normal).clamp_(max=126)
    if positive:
        c = torch.where(a > 0, c.clamp_(min=1), c)
    else:
        c = torch.where(x.view(-1) < 0, c + 128, c)
    code.copy_(c.to(torch.uint8).view(torch.float8_e4m3fn))


def _random16(n, seed, device):
    """Two streams of 16 random bits for n elements: four fields of one 64-bit SplitMix64 output serve two elements."""
    k = torch.arange(1, n // 2 + 1, dtype=torch.int64, device=device) * -0x61C8864680B583EB + seed
    k = (k ^ ((k >> 30) & (2 ** 34 - 1))) * -0x40A7B892E31B1A47
    k = (k ^ ((k >> 27) & (2 ** 37 - 1))) * -0x6B2FB644ECCEEE15
    k = k ^ ((k >> 31) & (2 ** 33 - 1))
    f = torch.stack([k, k >> 16, k >> 32, k >> 48], dim=1).bitwise_and_(0xffff).int()
    return f[:, 0::2].reshape(-1), f[:, 1::2].reshape(-1)


def _own_logprobs(s):
    dp, (logp, ent, lse, top, ids) = s["dp"], s["out"]
    dp.dp_logprobs_fwd(s["desc"], s["z"], s["ids"], logp, ent, lse, top, ids, s["ws"])
    if not s["case"]["grad"]:
        return s["out"]
    dp.dp_logprobs_bwd(s["desc"], s["z"], s["ids"], lse, ent, s["dlogp"], s["dent"], s["dz"])
    return s["out"] + [s["dz"]]


def _plain_logprobs(s):
    case, z, ids = s["case"], s["z"].float(), s["ids"].long()[:, None]
    c, k = case["classes"], case["top"]
    most = z.amax(dim=1, keepdim=True)
    none = most == -math.inf          # a row whose classes are all forbidden: its log-probabilities are -inf, its entropy and gradient 0
    e = torch.where(none, 0.0, torch.exp(z - most))
    total = e.sum(dim=1, keepdim=True)
    lse = most + torch.log(total)
    ent = torch.where(none, 0.0, torch.log(total) - torch.where(e > 0, e * (z - most), 0.0).sum(dim=1, keepdim=True) / total)
    logp = torch.where(none, -math.inf, z.gather(1, ids) - lse)
    # the order of floats as whole numbers, equal ones by their index
    b = (z + 0.0).view(torch.int32)
    key = ((b ^ ((b >> 31) & 0x7fffffff)).long() << 32) | (c - 1 - torch.arange(c, device=z.device))
    at = (c - 1 - (key.topk(k, dim=1).values & 0xffffffff))
    out = [logp[:, 0], ent[:, 0], lse[:, 0], torch.where(none, -math.inf, z.gather(1, at) - lse), at.int()]
    if not case["grad"]:
        return out
    p = e / total
    dz = -p * s["dlogp"][:, None] - s["dent"][:, None] * torch.where(p > 0, p * (z - lse + ent), 0.0)
    dz.scatter_add_(1, ids, s["dlogp"][:, None])
    return out + [torch.where(none, 0.0, dz).to(s["z"].dtype)]


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "group_norm":
        n = case["n"] * case["h"] * case["w"] * case["c"]
        size = 2 if case["dtype"] == "bf16" else 4
        reads = {"fwd": 2, "bwd": 4 if case["act"] == "relu" else 3, "both": 4}[case["way"]]   # x y | x dy dx (y) | x dy y dx
        return {"bytes": size * n * reads + 16.0 * case["c"], "flops": {"fwd": 8, "bwd": 16, "both": 24}[case["way"]] * float(n)}
    if case["kind"] == "logprobs":
        n = case["rows"] * case["classes"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": float(size * n * (2 if case["grad"] else 1) + case["rows"] * (16 + 8 * case["top"])), "flops": (6.0 + (5 if case["grad"] else 0)) * n}
    n = sum(t[0] for t in _tensors(case))
    if case["kind"] == "grad_norm":
        return {"bytes": 4.0 * n, "flops": 2.0 * n}
    return {"bytes": n * (30.0 if case["bits"] == 32 else 18.0 + 16.0 / BLOCK), "flops": (14.0 if case["bits"] == 32 else 40.0) * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    f = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for k, t in s.items()}
    return {"group_norm": _exact_group_norm, "grad_norm": _exact_grad_norm, "adamw": _exact_adamw, "logprobs": _exact_logprobs}[case["kind"]](case, f)


def _exact_group_norm(case, f):
    n, gr, c = case["n"], case["groups"], case["c"]
    # [sample, group, pixels, channels of the group]
    part = lambda t: t.reshape(n, -1, gr, c // gr).transpose(1, 2).contiguous()                 # noqa: E731
    whole = lambda t: t.transpose(1, 2).reshape(n, case["h"], case["w"], c)                     # noqa: E731
    x, gamma, beta = part(f["x"]), f["gamma"].view(gr, 1, -1), f["beta"].view(gr, 1, -1)
    count = x.shape[2] * x.shape[3]
    mean = x.sum(dim=(2, 3)) / count
    centred = x - mean[..., None, None]
    rstd = (centred.pow(2).sum(dim=(2, 3)) / count + EPS).rsqrt()
    out = []
    if case["way"] != "bwd":
        u = centred * rstd[..., None, None] * gamma + beta
        y = u.clamp(min=0) if case["act"].startswith("relu") else u * torch.sigmoid(u) if case["act"] == "silu" else u
        out = [whole(y), mean, rstd]
    if case["way"] != "fwd":
        if case["way"] == "bwd":
            mean, rstd = f["mean"], f["rstd"]
        r = rstd[..., None, None]
        xhat = (x - mean[..., None, None]) * r
        g = part(f["dy"])
        if case["act"] == "relu":
            g = torch.where(part(f["y"]) > 0, g, torch.zeros_like(g))
        if case["act"] == "silu":
            u = xhat * gamma + beta
            g = g * (torch.sigmoid(u) + u * torch.sigmoid(u) * torch.sigmoid(-u))
        to_xhat = g * gamma
        s1, s2 = to_xhat.sum(dim=(2, 3), keepdim=True), (to_xhat * xhat).sum(dim=(2, 3), keepdim=True)
        dx = r / count * (count * to_xhat - s1 - xhat * s2)
        out += [whole(dx), (g * xhat).sum(dim=(0, 2)).reshape(c), g.sum(dim=(0, 2)).reshape(c)]
    return out


def _exact_grad_norm(case, f):
    norm = torch.linalg.vector_norm(f["g"])
    return torch.stack([norm, MAX_NORM / torch.clamp(norm, min=MAX_NORM)])


def _exact_adamw(case, f):
    h, blocks = HYPER, (-1, BLOCK)
    g = f["g"] * f["scale"]
    m, v = f["m"], f["v"]
    if case["bits"] == 8:
        m, v = (m.view(blocks) * f["ms"].view(-1, 1)).view(-1), (v.view(blocks) * f["vs"].view(-1, 1)).pow(2).view(-1)
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    mhat, vhat = m / (1 - h["beta1"] ** h["step"]), v / (1 - h["beta2"] ** h["step"])
    w = f["w"] - h["lr"] * (mhat / (vhat.sqrt() + h["eps"]) + f["decay"].repeat_interleave(PAGE) * f["w"])
    if case["bits"] == 32:
        return [w, w, m, v]
    # which of the two neighbouring 8-bit floats is taken is random: no value; the scales have one
    top = lambda t: t.abs().view(blocks).amax(dim=1) / 448                                      # noqa: E731
    return [w, w, None, None, top(m), top(v.sqrt())]


def _exact_logprobs(case, f):
    z, ids = f["z"], f["ids"].long()
    lse = torch.logsumexp(z, dim=1)
    logq = torch.where(torch.isneginf(z), -math.inf, z - lse[:, None])
    p = logq.exp()
    ent = -torch.special.xlogy(p, p).sum(dim=1)
    # equal values are taken by their index
    best = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["top"]]
    out = [logq.gather(1, ids[:, None])[:, 0], ent, lse, logq.gather(1, best), best.int()]
    if case["grad"]:
        # d logp / dz_j = [j = id] - p_j;  d entropy / dz_j = -p_j (log p_j + entropy)
        dz = -f["dent"][:, None] * (torch.special.xlogy(p, p) + p * ent[:, None]) - f["dlogp"][:, None] * p
        dz[torch.arange(len(ids), device=ids.device), ids] += f["dlogp"]
        dz[torch.isneginf(lse)] = 0
        out.append(dz)
    return out
