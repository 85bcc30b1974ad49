"""What a program calls beside the clustered layers when it runs and trains a low-bit model: microscaled 4-bit floating
point, and distillation from a teacher's stored top logits.

Three kinds of work:

* "quantize": activations or weights are smoothed and written as microscaled 4-bit numbers (blocks of 32 columns with a
  power of two each, elements of sign, two exponent bits and one mantissa bit), and read back as what they stand for.
* "linear": x of a layer to y: x is quantised like that and multiplied by a microscaled 4-bit weight matrix, which the
  program holds in the layout of a checkpoint: codes [N, 16 * blocks] bytes, scales [N, blocks] bytes, rows on 16 bytes.
* "distill": the loss of a student's logits against the k largest logits of a teacher, and its gradient.  `path` says how:
  "loss" (evaluation), "train" (loss and gradient in one call) or "two_step" (the loss first, the gradient when the step's
  weight of every token is known).

`own` says which arithmetic runs: the package's kernels or plain tensor operations.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def quantize(name, R, K, type, smooth):
    return dict(name=name, kind="quantize", R=R, K=K, type=type, smooth=smooth)


def linear(name, M, N, K, type, out, smooth):
    return dict(name=name, kind="linear", M=M, N=N, K=K, type=type, out=out, smooth=smooth)


def distill(name, path, T, V, k, type, *, tau=1.0, whole=False, masked=0.0, absent=0.0):
    return dict(name=name, kind="distill", path=path, T=T, V=V, k=k, type=type, tau=tau, whole=whole, masked=masked, absent=absent)


def listed():
    return [
        # one token's activations of a 7B-sized layer: latency
        quantize("quantize-1x4096", 1, 4096, "fp16", True),
        # master weights of a projection after an update, quantised and read back
        quantize("quantize-11008x4096-weights", 11008, 4096, "fp32", False),
        # a ragged prompt with rows of odd length
        quantize("quantize-333x5001", 333, 5001, "bf16", True),
        # single-stream decode, the smallest projection
        linear("linear-m1-4096x4096", 1, 4096, 4096, "fp16", "fp32", True),
        # batched decode, sixteen sequences
        linear("linear-m16-11008x4096", 16, 11008, 4096, "bf16", "bf16", True),
        # single-stream decode of a LLaMA-70B-shaped projection: bandwidth
        linear("linear-m1-28672x8192", 1, 28672, 8192, "fp16", "fp32", False),
        # a ragged prompt on a matrix whose sides are no multiple of anything
        linear("linear-m333-5003x5001", 333, 5003, 5001, "fp16", "fp32", True),
        # prompt processing of a LLaMA-13B-shaped projection: tensor cores
        linear("linear-m2048-13824x5120", 2048, 13824, 5120, "bf16", "bf16", False),
        # a short sequence's step on the fp32 logits that the package's layers return
        distill("distill-16x32000-train", "train", 16, 32000, 16, "fp32", tau=2.0),
        # evaluation of a batch
        distill("distill-2048x32000-loss", "loss", 2048, 32000, 64, "bf16"),
        # padded sequences, fewer stored entries for some tokens, an odd vocabulary, the gradient in a call of its own
        distill("distill-777x50021-two-step", "two_step", 777, 50021, 100, "fp16", tau=2.0, masked=0.2, absent=0.1),
        # the training step of a large vocabulary, against the teacher's whole distribution
        distill("distill-4096x128000-train", "train", 4096, 128000, 128, "bf16", whole=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, lo, hi):
    """A matrix side: a multiple of 256, of 32, or any number."""
    step = rng.choice((256, 32, 1))
    return max(lo, _log(rng, lo, hi) // step * step)


def draw(rng):
    pick = rng.random()
    type = rng.choice(("fp32", "fp16", "bf16"))
    if pick < 0.25:
        return dict(kind="quantize", R=_log(rng, 1, 11008), K=_side(rng, 256, 4096), type=type, smooth=rng.random() < 0.5)
    if pick < 0.65:
        M = rng.choice((1, _log(rng, 2, 16), _log(rng, 17, 2048)))
        return dict(kind="linear", M=M, N=_side(rng, 512, 13824), K=_side(rng, 512, 5120), type=type, out=rng.choice(("fp32", "fp32", "bf16", "fp16")), smooth=rng.random() < 0.5)
    T, V = _log(rng, 1, 4096), _side(rng, 8192, 128000)
    if type == "fp32":
        T = max(1, T // 2)
    path = rng.choice(("loss", "train", "train", "two_step"))
    if path == "two_step":
        T = max(1, T // 2)
    return dict(kind="distill", path=path, T=T, V=V, k=_log(rng, 4, 128), type=type, tau=rng.choice((1.0, 2.0, 0.7)), whole=rng.random() < 0.4,
                masked=rng.choice((0.0, 0.3)), absent=rng.choice((0.0, 0.2)))


# ------------------------------------------------------------------------------------------------- the inputs
def _activations(g, M, K, type):
    """N(0, 1) with one channel in a hundred fifty times larger, and factors that smooth them."""
    x = torch.randn(M, K, generator=g, device="cuda")
    factor = torch.ones(K, device="cuda")
    at = torch.randperm(K, generator=g, device="cuda")[: max(1, K // 100)]
    factor[at] = 50.0
    inv = torch.rsqrt(factor) * (0.5 + torch.rand(K, generator=g, device="cuda"))
    return (x * factor).to(TYPES[type]), inv


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["kind"] == "quantize":
        x, inv = _activations(g, case["R"], case["K"], case["type"])
        return dict(case, x=x, inv=inv if case["smooth"] else None)
    if case["kind"] == "linear":
        x, inv = _activations(g, case["M"], case["K"], case["type"])
        w = torch.randn(case["N"], case["K"], generator=g, device="cuda").mul_(0.02)
        if case["smooth"]:
            w.div_(inv)
        codes, scales = _checkpoint(w)
        return dict(case, x=x, inv=inv if case["smooth"] else None, codes=codes, scales=scales)
    T, V, k = case["T"], case["V"], case["k"]
    z = torch.randn(T, V, generator=g, device="cuda").mul_(2.5)
    teacher = z + torch.randn(T, V, generator=g, device="cuda")
    top, idx = teacher.topk(k, dim=1)
    lse = None
    if case["whole"]:
        lse = torch.logsumexp(teacher.div_(case["tau"]), dim=1)
    del teacher
    gone = torch.rand(T, k, generator=g, device="cuda") < case["absent"]
    idx = torch.where(gone, torch.full_like(idx, -1), idx).to(torch.int32)
    weight = (torch.rand(T, generator=g, device="cuda") >= case["masked"]).float() * (case["tau"] ** 2)
    weight[0] = case["tau"] ** 2
    return dict(case, z=z.to(TYPES[case["type"]]), idx=idx, top=top.half(), lse=lse, weight=weight)


# ------------------------------------------------------------------------------------------------- the plain form
def _blocks(x, inv):
    """fp32 [R, blocks, 32], smoothed, the last block filled with zeros."""
    t = x.float()
    if inv is not None:
        t = t * inv
    R, K = t.shape
    return torch.nn.functional.pad(t, (0, -K % 32)).view(R, -1, 32)


def _round_blocks(t):
    """Blocks' exponents (int32 [R, blocks]; 128 where a block is not finite) and elements (fp32, what the 4 bits stand for)."""
    top = t.abs().amax(dim=2)
    fine = torch.isfinite(top)
    _, e = torch.frexp(torch.where(fine, top, torch.ones_like(top)))
    e = torch.where(top == 0, torch.zeros_like(e), (e - 3).clamp(-127, 127))
    u = torch.where(fine[:, :, None], torch.ldexp(t, -e[:, :, None]), torch.zeros_like(t))
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.copysign((torch.round(a / step) * step).clamp(max=6.0), u)
    return torch.where(fine, e, torch.full_like(e, 128)), q


def _values(e, q, K):
    scale = torch.where(e == 128, torch.full_like(e, 0, dtype=torch.float32) / 0.0, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e))
    return (q * scale[:, :, None]).flatten(1)[:, :K]


def _checkpoint(w):
    """Codes and scales of a weight matrix as a checkpoint holds them; rows of scales start on 16 bytes."""
    e, q = _round_blocks(_blocks(w, None))
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = (code | (torch.signbit(q).to(torch.uint8) << 3)).flatten(1)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    blocks = e.shape[1]
    scales = torch.zeros(w.shape[0], -(-blocks // 16) * 16, dtype=torch.uint8, device="cuda")
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes, scales[:, :blocks]


def _read(codes, scales, K):
    code = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1).int()
    a = (code & 7).float()
    a = torch.where(a < 4, a / 2, torch.where(a < 6, a - 2, (a - 4) * 2))
    q = torch.where(code >= 8, -a, a).view(codes.shape[0], -1, 32)
    return _values(scales.int() - 127, q, K)


def _distill(s, gradient):
    z = s["z"].float() / s["tau"]
    V = z.shape[1]
    there = (s["idx"] >= 0) & (s["idx"] < V)
    at = torch.where(there, s["idx"], torch.zeros_like(s["idx"])).long()
    t = torch.where(there, s["top"].float() / s["tau"], torch.full(s["top"].shape, -math.inf, device="cuda"))
    if s["lse"] is None:
        high = t.amax(dim=1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
        norm = high + torch.log(torch.exp(t - high).sum(dim=1, keepdim=True))
    else:
        norm = s["lse"][:, None]
    p = torch.where(there, torch.exp(t - norm), torch.zeros_like(t))
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    logq = (z.gather(1, at) - top) - torch.log(total)
    w = s["weight"]
    loss = w * torch.where(p > 0, p * ((t - norm) - logq), torch.zeros_like(p)).sum(dim=1)
    if not gradient:
        return [loss]
    d = e.mul_(p.sum(dim=1, keepdim=True) / total).scatter_add_(1, at, -p)
    return [loss, d.mul_(w[:, None] / s["tau"]).to(s["z"].dtype)]


def _run_plain(s):
    if s["kind"] == "quantize":
        e, q = _round_blocks(_blocks(s["x"], s["inv"]))
        return [_values(e, q, s["K"])]
    if s["kind"] == "linear":
        e, q = _round_blocks(_blocks(s["x"], s["inv"]))
        return [(_values(e, q, s["K"]) @ _read(s["codes"], s["scales"], s["K"]).t()).to(TYPES[s["out"]])]
    return _distill(s, s["path"] != "loss")


def _run_own(s):
    import paper_2506_12038_b200 as lcd
    if s["kind"] == "quantize":
        codes, scales = lcd.mx_quantize(s["x"], s["inv"])
        return [lcd.mx_dequantize(codes, scales, s["K"])]
    if s["kind"] == "linear":
        return [lcd.mx_linear_fused(s["codes"], s["scales"], s["x"], s["inv"], dtype=TYPES[s["out"]])]
    teacher = dict(temperature=s["tau"], teacher_lse=s["lse"], weight=s["weight"])
    if s["path"] == "loss":
        return [lcd.distill_loss(s["z"], s["idx"], s["top"], **teacher)]
    if s["path"] == "train":
        return list(lcd.distill_loss(s["z"], s["idx"], s["top"], want_grad=True, **teacher))
    loss, stats = lcd.distill_loss(s["z"], s["idx"], s["top"], want_stats=True, **teacher)
    return [loss, lcd.distill_grad(s["z"], s["idx"], s["top"], stats, **teacher)]


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ------------------------------------------------------------------------------------------------- what it has to move
def work(case):
    size = {"fp32": 4, "fp16": 2, "bf16": 2}
    if case["kind"] == "quantize":
        n, blocks = case["R"] * case["K"], case["R"] * -(-case["K"] // 32)
        return {"bytes": n * size[case["type"]] + 17 * blocks + 4 * n + (4 * case["K"] if case["smooth"] else 0), "flops": 2 * n}
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 17 * N * -(-K // 32) + M * K * size[case["type"]] + M * N * size[case["out"]] + (4 * K if case["smooth"] else 0), "flops": 2 * M * N * K}
    T, V, k = case["T"], case["V"], case["k"]
    grads = 0 if case["path"] == "loss" else T * V * size[case["type"]]
    return {"bytes": T * V * size[case["type"]] + grads + T * (6 * k + 8 + (4 if case["whole"] else 0)), "flops": T * V * (4 if case["path"] == "loss" else 6)}


# ------------------------------------------------------------------------------------------------- the definition in 64 bits
def _nearest(t):
    """What blocks of 32 (float64) become: every element the nearest of the format's numbers times the block's power of two."""
    top = t.abs().amax(dim=2, keepdim=True)
    powers = torch.tensor([2.0 ** i for i in range(-150, 128)], dtype=torch.float64, device="cuda")
    power = powers[torch.bucketize(top, powers, right=True) - 1] / 4
    power = torch.where(top == 0, torch.ones_like(top), power.clamp(2.0 ** -127, 2.0 ** 127))
    a = t.abs() / power
    # the borders between neighbours; a tie goes to the one whose last bit is zero
    index = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5).int()
    numbers = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    return torch.sign(t) * numbers[index] * power


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("quantize", "linear"):
        t = s["x"].double()
        if s["inv"] is not None:
            t = (t * s["inv"].double()).float().double()        # the smoothed value is a binary32 number by definition
        R, K = t.shape
        values = _nearest(torch.cat([t, t.new_zeros(R, -K % 32)], dim=1).view(R, -1, 32)).reshape(R, -1)[:, :K]
        if case["kind"] == "quantize":
            return [values]
        numbers = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
        w = torch.empty(case["N"], s["codes"].shape[1] * 2, dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = numbers[(s["codes"] % 16).long()], numbers[(s["codes"] // 16).long()]
        powers = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [math.nan], dtype=torch.float64, device="cuda")
        w *= powers[s["scales"].long()].repeat_interleave(32, dim=1)
        return [values @ w[:, :K].t()]
    z = s["z"].double() / case["tau"]
    logq = torch.log_softmax(z, dim=1)
    there = (s["idx"] >= 0) & (s["idx"] < case["V"])
    t = s["top"].double() / case["tau"]
    lse = torch.logsumexp(t.masked_fill(~there, -math.inf), dim=1) if s["lse"] is None else s["lse"].double()
    logp = t - lse[:, None]
    p = torch.exp(logp).masked_fill(~there, 0.0)
    at = s["idx"].long().clamp(0, case["V"] - 1)
    w = s["weight"].double()
    loss = w * torch.nan_to_num(p * (logp - logq.gather(1, at))).sum(dim=1)
    if case["path"] == "loss":
        return [loss]
    grad = torch.exp(logq) * p.sum(dim=1, keepdim=True)
    grad.scatter_add_(1, at, -p)
    return [loss, grad * (w / case["tau"])[:, None]]
