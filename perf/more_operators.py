"""What a program calls where the rows of one batch go to different weights: layers of experts in microscaled 4-bit floating point, and
low-rank adapters of many requests beside a shared layer, in serving and in training.

Four kinds of work:

* "group": the plan of a batch: from the group of every row (an expert, an adapter, none) the rows' order by group.
* "experts": x of a layer of experts and every token's choices to y, one row for each pair of a token and a choice: plan, quantisation of
  x, product with the experts' microscaled 4-bit weights [G, N, 16 * blocks] as a checkpoint holds them.
* "adapters": what a shared layer gave, plus the adapter's part of every row: y = base + s_g (x a_g^T) b_g^T.  The plan is kept for
  all layers of a step, so the program has it in hand.
* "grad": the backward pass of the adapters, with t = x a_g^T kept from the forward pass: gradients of x, a and b.

`own` says which arithmetic runs: the package's kernels or plain tensor operations.
"""
import math

import numpy
import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def group(name, P, k, G, absent=0.0):
    return dict(name=name, kind="group", P=P, k=k, G=G, absent=absent)


def experts(name, T, k, G, N, K, type, out, *, smooth=False, absent=0.0):
    return dict(name=name, kind="experts", T=T, k=k, G=G, N=N, K=K, type=type, out=out, smooth=smooth, absent=absent)


def adapters(name, M, G, used, r, K, N, type, weights, out, *, absent=0.0):
    return dict(name=name, kind="adapters", M=M, G=G, used=used, r=r, K=K, N=N, type=type, weights=weights, out=out, absent=absent)


def grad(name, M, G, used, r, K, N, type, weights, *, absent=0.0):
    return dict(name=name, kind="grad", M=M, G=G, used=used, r=r, K=K, N=N, type=type, weights=weights, absent=absent)


def listed():
    return [
        # the choices of a decoding batch
        group("group-64x4-of-32", 256, 4, 32),
        # the choices of a long prompt, some of them experts that another GPU holds
        group("group-8192x8-of-128", 65536, 8, 128, absent=0.25),
        # one token of a layer of experts: latency, and the weights of four experts
        experts("experts-1x4-of-32", 1, 4, 32, 4096, 2048, "fp16", "fp32", smooth=True),
        # batched decode: every expert's weights for a few rows each
        experts("experts-48x2-of-8", 48, 2, 8, 11008, 4096, "bf16", "bf16"),
        # a ragged prompt, odd sides, choices that are left out
        experts("experts-333x3-of-13", 333, 3, 13, 1001, 2005, "fp32", "fp16", smooth=True, absent=0.2),
        # prompt processing: tensor cores
        experts("experts-2048x4-of-32", 2048, 4, 32, 4096, 2048, "bf16", "bf16"),
        # one request with an adapter beside a projection that returns fp32: latency
        adapters("adapters-1", 1, 8, 1, 16, 4096, 4096, "fp16", "fp16", "fp32"),
        # a decoding batch in which nearly every request has an adapter of its own
        adapters("adapters-64-of-48", 64, 64, 48, 16, 4096, 11008, "bf16", "bf16", "bf16"),
        # a ragged batch with odd sides and rank, some requests without adapter
        adapters("adapters-777-of-5", 777, 9, 5, 12, 5001, 5003, "fp16", "fp16", "fp32", absent=0.2),
        # the prompts of six requests beside a LLaMA-13B-shaped projection
        adapters("adapters-4096-of-6", 4096, 16, 6, 64, 5120, 13824, "bf16", "bf16", "bf16"),
        # a training step of one adapter beside a 4096 x 4096 projection, short sequences
        grad("grad-512", 512, 1, 1, 8, 4096, 4096, "fp16", "fp32"),
        # a training step of four adapters at once
        grad("grad-4096-of-4", 4096, 4, 4, 32, 5120, 5120, "bf16", "bf16"),
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
    absent = rng.choice((0.0, 0.0, 0.25))
    if pick < 0.1:
        k = rng.choice((1, 2, 4, 8))
        return dict(kind="group", P=k * _log(rng, 1, 8192), k=k, G=_log(rng, k, 256), absent=absent)
    if pick < 0.45:
        k, G = rng.choice((1, 2, 4)), _log(rng, 4, 32)
        T = rng.choice((1, _log(rng, 2, 64), _log(rng, 65, 2048)))
        return dict(kind="experts", T=T, k=k, G=G, N=_side(rng, 512, 4096), K=_side(rng, 512, 2048), type=type, out=rng.choice(("fp32", "fp16", "bf16")),
                    smooth=rng.random() < 0.5, absent=absent)
    M, G = rng.choice((1, _log(rng, 2, 64), _log(rng, 65, 4096))), _log(rng, 1, 64)
    shape = dict(M=M, G=G, used=_log(rng, 1, G), r=rng.choice((4, 8, 12, 16, 16, 32, 64, 50)), type=type, weights=rng.choice((type, type, "fp32")), absent=absent)
    if pick < 0.75:
        return dict(kind="adapters", K=_side(rng, 512, 5120), N=_side(rng, 512, 8192), out=rng.choice((type, "fp32")), **shape)
    return dict(kind="grad", K=_side(rng, 512, 5120), N=_side(rng, 512, 5120), **shape)


# ------------------------------------------------------------------------------------------------- the inputs
def _activations(g, M, K, type):
    """N(0, 1) with one channel in a hundred fifty times larger, and factors that smooth them."""
    x = torch.randn(M, K, generator=g, device="cuda")
    factor = torch.ones(K, device="cuda")
    at = torch.randperm(K, generator=g, device="cuda")[: max(1, K // 100)]
    factor[at] = 50.0
    inv = torch.rsqrt(factor) * (0.5 + torch.rand(K, generator=g, device="cuda"))
    return (x * factor).to(TYPES[type]), inv


def _choices(g, T, k, G, absent):
    """Every token's k experts, int32 [T, k]: different ones, some chosen more often than others, -1 where one is left out."""
    score = torch.rand(T, G, generator=g, device="cuda").log_().neg_().log_().neg_() + torch.randn(G, generator=g, device="cuda").mul_(0.7)
    top = score.topk(k, dim=1).indices.to(torch.int32)
    gone = torch.rand(T, k, generator=g, device="cuda") < absent
    return torch.where(gone, torch.full_like(top, -1), top)


def _requests(g, M, G, used, absent):
    """The adapter of every row, int32 [M]: requests of a few rows to many, one after the other, some without (-1)."""
    have = torch.randperm(G, generator=g, device="cuda")[:used]
    requests = max(used, M // 64)
    start = torch.rand(M, generator=g, device="cuda") < requests / M
    request = start.int().cumsum(0)
    pick = torch.randint(used, (M + 1,), generator=g, device="cuda")
    first = torch.randperm(used, generator=g, device="cuda")[: M + 1]
    pick[: len(first)] = first
    which = have[pick[request]]
    gone = (torch.rand(M + 1, generator=g, device="cuda") < absent)[request]
    return torch.where(gone, torch.full_like(which, -1), which).to(torch.int32)


def _plan(which, G):
    """Stable order of the rows by group, the group at every place of it (-1: none), the groups' offsets."""
    key = torch.where((which >= 0) & (which < G), which, torch.full_like(which, G))
    groups, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(groups, torch.arange(G + 1, device="cuda", dtype=groups.dtype))
    return order.to(torch.int32), torch.where(groups < G, groups, torch.full_like(groups, -1)).to(torch.int32), offsets.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["kind"] == "group":
        return dict(case, which=_choices(g, case["P"] // case["k"], case["k"], case["G"], case["absent"]))
    if case["kind"] == "experts":
        T, G, N, K = case["T"], case["G"], case["N"], case["K"]
        which = _choices(g, T, case["k"], G, case["absent"])
        x, inv = _activations(g, T, K, case["type"])
        made = []
        for _ in range(G):
            w = torch.randn(N, K, generator=g, device="cuda").mul_(0.02)
            if case["smooth"]:
                w.div_(inv)
            made.append(_checkpoint(w))
        codes, scales = torch.stack([c for c, _ in made]), torch.stack([s for _, s in made])
        blocks = -(-K // 32)
        key = torch.where(which >= 0, which, torch.full_like(which, G)).flatten()
        return dict(case, x=x, inv=inv if case["smooth"] else None, which=which, codes=codes, scales=scales[:, :, :blocks],
                    sizes=torch.bincount(key, minlength=G + 1).tolist())
    M, G, r, K, N = case["M"], case["G"], case["r"], case["K"], case["N"]
    which = _requests(g, M, G, case["used"], case["absent"])
    order, groups, offsets = _plan(which, G)
    bounds = offsets.tolist()
    x, _ = _activations(g, M, K, case["type"])
    weights = TYPES[case["weights"]]
    a = torch.randn(G, r, K, generator=g, device="cuda").mul_(K ** -0.5).to(weights)
    b = torch.randn(G, N, r, generator=g, device="cuda").mul_(0.05).to(weights)
    scale = 0.5 + torch.rand(G, generator=g, device="cuda")
    s = dict(case, x=x, a=a, b=b, scale=scale, order=order, groups=groups, offsets=offsets,
             present=[(e, bounds[e], bounds[e + 1]) for e in range(G) if bounds[e + 1] > bounds[e]])
    if case["kind"] == "adapters":
        return dict(s, base=torch.randn(M, N, generator=g, device="cuda").to(TYPES[case["out"]]))
    t = torch.zeros(M, r, device="cuda")
    for e, lo, hi in s["present"]:
        rows = order[lo:hi].long()
        t[rows] = x[rows].float() @ a[e].float().t()
    dy = torch.randn(M, N, generator=g, device="cuda").mul_(0.01).to(TYPES[case["type"]])
    return dict(s, t=t, dy=dy, base=torch.randn(M, K, generator=g, device="cuda").mul_(0.01).to(TYPES[case["type"]]))


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
    return codes, scales


def _read(codes, scales, K):
    code = torch.stack((codes & 15, codes >> 4), dim=2).flatten(1).int()
    a = (code & 7).float()
    a = torch.where(a < 4, a / 2, torch.where(a < 6, a - 2, (a - 4) * 2))
    q = torch.where(code >= 8, -a, a).view(codes.shape[0], -1, 32)
    return _values(scales.int() - 127, q, K)


def _run_plain(s):
    if s["kind"] == "group":
        return list(_plan(s["which"].flatten(), s["G"]))
    if s["kind"] == "experts":
        order, _, _ = _plan(s["which"].flatten(), s["G"])
        e, q = _round_blocks(_blocks(s["x"], s["inv"]))
        x = _values(e, q, s["K"])
        y = torch.zeros(s["T"] * s["k"], s["N"], device="cuda")
        at = 0
        for which, size in enumerate(s["sizes"][:-1]):
            if size:
                rows = order[at:at + size].long()
                y[rows] = x[rows // s["k"]] @ _read(s["codes"][which], s["scales"][which], s["K"]).t()
            at += size
        return [y.to(TYPES[s["out"]])]
    x, order, scale = s["x"].float(), s["order"].long(), s["scale"]
    few = s["M"] <= 64                    # a weight for every row in place of a product for every group
    if few:
        back = torch.empty_like(order).scatter_(0, order, torch.arange(s["M"], device="cuda"))
        which = s["groups"].long()[back]
        there = (which >= 0).float()[:, None]
        which = which.clamp(min=0)
        a, b, factor = s["a"][which].float(), s["b"][which].float(), scale[which][:, None] * there
    if s["kind"] == "adapters":
        y = s["base"].float()
        if few:
            t = torch.bmm(a, x[:, :, None])
            return [(y + factor * torch.bmm(b, t)[:, :, 0]).to(s["base"].dtype)]
        y = y.clone()
        for e, lo, hi in s["present"]:
            rows = order[lo:hi]
            y[rows] += scale[e] * ((x[rows] @ s["a"][e].float().t()) @ s["b"][e].float().t())
        return [y.to(s["base"].dtype)]
    dx, dy = s["base"].float().clone(), s["dy"].float()
    da, db = torch.zeros_like(s["a"], dtype=torch.float32), torch.zeros_like(s["b"], dtype=torch.float32)
    for e, lo, hi in s["present"]:
        rows = order[lo:hi]
        d = dy[rows] * scale[e]
        dt = d @ s["b"][e].float()
        dx[rows] += dt @ s["a"][e].float()
        da[e] = dt.t() @ x[rows]
        db[e] = d.t() @ s["t"][rows]
    return [dx.to(s["x"].dtype), da.to(s["a"].dtype), db.to(s["b"].dtype)]


def _run_own(s):
    import paper_2506_12038_b200 as lcd
    if s["kind"] == "group":
        return list(lcd.group_rows(s["which"], s["G"]))
    if s["kind"] == "experts":
        rows = lcd.group_rows(s["which"], s["G"])
        return [lcd.mx_linear_grouped(s["codes"], s["scales"], s["x"], rows, s["inv"], dtype=TYPES[s["out"]])]
    rows = lcd.RowGroups(s["order"], s["groups"], s["offsets"])
    if s["kind"] == "adapters":
        return [lcd.adapters(s["x"], s["a"], s["b"], rows, s["base"], scale=s["scale"])]
    return list(lcd.adapters_grad(s["dy"], s["x"], s["a"], s["b"], s["t"], rows, s["base"], scale=s["scale"]))


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ------------------------------------------------------------------------------------------------- what it has to move
def work(case):
    size = {"fp32": 4, "fp16": 2, "bf16": 2}
    if case["kind"] == "group":
        return {"bytes": 12 * case["P"] + 4 * (case["G"] + 1), "flops": case["P"]}
    if case["kind"] == "experts":
        T, k, G, N, K = (case[n] for n in ("T", "k", "G", "N", "K"))
        pairs = max(1, round(T * k * (1 - case["absent"])))
        read = G * (1 - (1 - 1 / G) ** pairs) if T > 1 else pairs           # experts that occur, about
        return {"bytes": int(read * 17 * N * -(-K // 32)) + T * K * size[case["type"]] + 4 * T * k + T * k * N * size[case["out"]], "flops": 2 * pairs * N * K}
    M, r, K, N = (case[n] for n in ("M", "r", "K", "N"))
    rows, present = max(1, round(M * (1 - case["absent"]))), min(case["used"], M)
    weights = present * r * (K + N) * size[case["weights"]]
    if case["kind"] == "adapters":
        return {"bytes": rows * K * size[case["type"]] + weights + 2 * M * N * size[case["out"]], "flops": 2 * rows * r * (K + N)}
    return {"bytes": (rows * (K + N) + 2 * M * K) * size[case["type"]] + weights + case["G"] * r * (K + N) * size[case["weights"]] + 4 * rows * r,
            "flops": 4 * rows * r * (K + N)}


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
    if case["kind"] == "group":
        which = s["which"].flatten().cpu().numpy()
        rows = [numpy.flatnonzero(which == e) for e in range(case["G"])]
        counts = [len(r) for r in rows]
        rest = numpy.flatnonzero((which < 0) | (which >= case["G"]))
        groups = numpy.concatenate([numpy.full(c, e) for e, c in enumerate(counts)] + [numpy.full(len(rest), -1)])
        whole = (numpy.concatenate(rows + [rest]), groups, numpy.concatenate([[0], numpy.cumsum(counts)]))
        return [torch.from_numpy(v.astype(numpy.int32)).cuda() for v in whole]
    if case["kind"] == "experts":
        t = s["x"].double()
        if s["inv"] is not None:
            t = (t * s["inv"].double()).float().double()        # the smoothed value is a binary32 number by definition
        T, K = t.shape
        values = _nearest(torch.cat([t, t.new_zeros(T, -K % 32)], dim=1).view(T, -1, 32)).reshape(T, -1)[:, :K]
        numbers = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
        powers = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [math.nan], dtype=torch.float64, device="cuda")
        y = torch.zeros(T, case["k"], case["N"], dtype=torch.float64, device="cuda")
        for e in range(case["G"]):
            token, choice = torch.nonzero(s["which"] == e, as_tuple=True)
            if len(token) == 0:
                continue
            codes = s["codes"][e]
            w = torch.empty(case["N"], codes.shape[1] * 2, dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = numbers[(codes % 16).long()], numbers[(codes // 16).long()]
            w *= powers[s["scales"][e].long()].repeat_interleave(32, dim=1)
            y[token, choice] = torch.matmul(values[token], w[:, :K].t())
        return [y.flatten(0, 1)]
    # the adapter of every row, from the plan
    which = torch.empty(case["M"], dtype=torch.int64, device="cuda")
    which[s["order"].long()] = s["groups"].long()
    x, base = s["x"].double(), s["base"].double()
    if case["kind"] == "adapters":
        y = base.clone()
        for e in which.unique().tolist():
            if e >= 0:
                mine = which == e
                t = torch.einsum("mk,rk->mr", x[mine], s["a"][e].double())
                y[mine] += float(s["scale"][e]) * torch.einsum("mr,nr->mn", t, s["b"][e].double())
        return [y]
    dx, da, db = base.clone(), torch.zeros_like(s["a"], dtype=torch.float64), torch.zeros_like(s["b"], dtype=torch.float64)
    for e in which.unique().tolist():
        if e < 0:
            continue
        mine, factor = which == e, float(s["scale"][e])
        dy, a, b = s["dy"][mine].double(), s["a"][e].double(), s["b"][e].double()
        dt = factor * torch.einsum("mn,nr->mr", dy, b)
        dx[mine] += torch.einsum("mr,rk->mk", dt, a)
        da[e] = torch.einsum("mr,mk->rk", dt, x[mine])
        db[e] = factor * torch.einsum("mn,mr->nr", dy, s["t"][mine].double())
    return [dx, da, db]
