"""The loss of a distillation call where a warp's teacher entries and the logits that it reads have nothing to do with each other:
vocabularies shorter than a CTA's words, rows masked to a few columns.  Bounds as derived at check()."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_distill_gpu import TYPES, check, every_path, host, make

pytestmark = pytest.mark.gpu


def every_loss(z, idx, top, **teacher):
    """Both forms of the loss (alone, with a gradient) and the gradient, each against the oracle."""
    loss, grad, stats = every_path(z, idx, top, **teacher)
    args = teacher.get("temperature", 1.0), teacher.get("teacher_lse"), teacher.get("weight")
    check(z, idx, top, *args, loss=loss, grad=grad, stats=stats)
    check(z, idx, top, *args, loss=lcd.distill_loss(z, idx, top, **teacher))


def whole_lse(teacher, tau):
    high = teacher.max(axis=1, keepdims=True)
    return torch.from_numpy(((high / tau)[:, 0] + np.log(np.exp((teacher - high) / tau).sum(axis=1))).astype(np.float32)).cuda()


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("tau", [0.7, 1.0, 2.0])
@pytest.mark.parametrize("T,V,k", [(2, 33, 33), (3, 100, 64), (5, 256, 128), (40, 20, 20), (4, 300, 300), (64, 500, 40), (700, 256, 64), (3, 700, 700),
                                   (1000, 130, 100)])
def test_vocabularies_shorter_than_the_words_of_a_block(T, V, k, tau, type):
    z, idx, top, teacher = make(T + V, T, V, k, type)
    every_loss(z, idx, top, temperature=tau)
    every_loss(z, idx, top, temperature=tau, teacher_lse=whole_lse(teacher, tau))


@pytest.mark.parametrize("k", [33, 64, 128, 300])
@pytest.mark.parametrize("left", [(0, 256), (31960, 32000), (17000, 17001)])
@pytest.mark.parametrize("T,tau,type,low", [(1, 0.7, "bf16", False), (64, 1.0, "fp32", True), (64, 0.7, "fp16", False), (300, 0.7, "bf16", True),
                                            (300, 2.0, "fp16", True), (1, 1.0, "fp32", True), (200, 0.7, "fp32", False)])
def test_rows_masked_to_a_few_columns(T, tau, type, low, left, k):
    # the teacher's entries lie among the columns that are left and take any place of the k; the others are absent, or the teacher
    # has masked them too (by -infinity, or by its type's lowest value: p = 0)
    V, n = 32000, left[1] - left[0]
    rng = np.random.default_rng(k + n)
    z = torch.full((T, V), torch.finfo(TYPES[type]).min if low else -float("inf"), dtype=TYPES[type], device="cuda")
    z[:, left[0]:left[1]] = torch.from_numpy(rng.normal(size=(T, n)) * 2.5).to(z.dtype).cuda()
    teacher = host(z[:, left[0]:left[1]]) + rng.normal(size=(T, n))
    idx, top = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    few = min(n, k)
    for t in range(T):
        place = rng.permutation(k)
        best = np.argsort(-teacher[t])[:few]
        idx[t, place[:few]], top[t, place[:few]] = left[0] + best, teacher[t, best]
        masked = place[few:few + 9]
        idx[t, masked], top[t, masked] = 1000 + np.arange(len(masked)), np.where(np.arange(len(masked)) % 2, -np.inf, -65504.0)
    idx, top = torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(top).half().cuda()
    every_loss(z, idx, top, temperature=tau)
    every_loss(z, idx, top, temperature=tau, teacher_lse=whole_lse(teacher, tau))


@pytest.mark.parametrize("T", [2, 64])
def test_the_student_rules_out_what_the_teacher_holds_likely(T):
    # at one entry of many, wherever in the row of entries it stands; and a token all of whose entries the student rules out
    z, idx, top, _ = make(T, T, 260, 130)
    for row, j in ((0, 0), (1, 129)):
        z[row, idx[row, j].long()] = -float("inf")
    loss, grad, _ = every_path(z, idx, top, temperature=0.7)
    assert (loss[:2] == float("inf")).all() and torch.isfinite(loss[2:]).all() and torch.isfinite(grad).all()
    z[0, idx[0].long()] = -float("inf")
    loss, grad, _ = every_path(z, idx, top, temperature=0.7)
    assert loss[0] == float("inf") and torch.isfinite(grad).all()


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("T,V,tau,whole", [(256, 32000, 2.0, True), (16, 33000, 2.0, True), (256, 5000, 2.0, True), (256, 32000, 1.0, False), (16, 33000, 1.0, True)])
def test_digits_of_the_loss(T, V, tau, whole, type):
    # log p and log q are each around ten times the loss: in 32 bits their roundings would be most of its error.  Held to the error of the
    # formula in 32-bit tensor operations, where they are rounded once an entry and in no common way (over 256 rows, root mean square)
    from oracle import train_oracle as O
    errors = [], []
    for seed in range(256 // T):
        z, idx, top, teacher = make(seed, T, V, 64, type)
        lse = whole_lse(teacher, tau) if whole else None
        want = O.distill(host(z), idx.cpu().numpy(), host(top), tau, None if lse is None else host(lse))[0]
        got = lcd.distill_loss(z, idx, top, temperature=tau, teacher_lse=lse)
        a = top.float() / tau
        logp = a - (torch.logsumexp(a, dim=1) if lse is None else lse)[:, None]
        x = z.float() / tau
        high = x.amax(dim=1, keepdim=True)
        logq = (x.gather(1, idx.long()) - high) - torch.log(torch.exp(x - high).sum(dim=1, keepdim=True))
        plain = (torch.exp(logp) * (logp - logq)).sum(dim=1)
        for e, v in zip(errors, (got, plain)):
            e.append((host(v) - want) / want)
    own, plain = (np.sqrt(np.mean(np.concatenate(e) ** 2)) for e in errors)
    assert own <= plain, (own, plain)


@pytest.mark.parametrize("tau", [0.7, 1.3])
@pytest.mark.parametrize("T,V,k", [(3, 3000, 10), (3, 40000, 300), (300, 700, 40)])
def test_large_teacher_logits_keep_their_differences(T, V, k, tau):
    # t / temperature is 11702 for t = 8192 and would be rounded to 2^-10
    z, idx, top, _ = make(T + k, T, V, k)
    top = (top.float() * 64).round() / 64 + 8192
    every_loss(z, idx, top, temperature=tau)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("T,V", [(3, 40000), (64, 700)])
def test_teacher_logits_whose_quotients_overflow(T, V, type):
    z, idx, top, _ = make(T, T, V, 40)
    high, low = torch.finfo(TYPES[type]).max, torch.finfo(TYPES[type]).min
    top = top.to(TYPES[type])
    top[0] = low                          # all alike, however low: 1 / k each
    top[1] = high
    top[2, 5:] = low                      # five entries are left
    loss, grad, stats = every_path(z, idx, top, temperature=0.5)
    even = lcd.distill_loss(z[:2], idx[:2], torch.zeros_like(top[:2]), temperature=0.5)
    # (the same formula on other numbers; 16 roundings of the loss's size)
    assert torch.isfinite(loss).all() and ((even - loss[:2]).abs() <= 2.0 ** -20 * even).all()
    short = lcd.distill_loss(z[2:3], idx[2:3, :5].contiguous(), top[2:3, :5].contiguous(), temperature=0.5)
    assert ((short - loss[2]).abs() <= 2.0 ** -20 * short).all()
    if T > 3:
        check(z[3:], idx[3:], top[3:], 0.5, loss=loss[3:], grad=grad[3:], stats=stats[3:])
