"""Rotary positions of several coordinates against 64 bits, the way back, and its use as the gradient."""
import pytest
import torch

from paper_2509_21354_amd import binding as kb
from tests import pages_ref as ref

pytestmark = pytest.mark.gpu


def _shape(L, B, H, Hkv, d, dtype):
    return kb.make_shape(L=L, B=B, H=H, H_kv=Hkv, d=d, T=0, T_cap=1, C=1, N_cap=0, W=0, d_sum=1, d_g=1, dtype=kb.F32 if dtype == torch.float32 else kb.BF16)


def _draw(seed, *size, dtype):
    return torch.randn(size, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _bound(want, x, dtype):
    """Sine and cosine in fp32 (within 2^-22 of a turn's rounding and their own), two products and a sum in fp32, one rounding."""
    size = x.double().abs().amax()
    return 2 * size * (2.0 ** -22 + 3 * 2.0 ** -24) + want.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)


CASES = [  # dtype, L, B, H, Hkv, d, Tq, sections, layout
    ("bf16", 1, 1, 1, 1, 128, 1, (64,), 0), ("bf16", 1, 2, 4, 2, 128, 5, (16, 24, 24), 0), ("f32", 1, 2, 4, 4, 64, 9, (10, 11, 11), 0),
    ("bf16", 2, 1, 8, 1, 64, 33, (8, 8, 16), 1), ("f32", 2, 2, 3, 1, 128, 40, (16, 16, 16, 16), 1), ("bf16", 1, 3, 2, 2, 128, 70, (7, 9, 10), 0),
    ("f32", 1, 1, 5, 5, 64, 17, (1, 2), 1), ("bf16", 1, 1, 2, 1, 64, 300, (0, 32), 0), ("bf16", 1, 2, 4, 4, 128, 3, (1,), 1), ("f32", 1, 1, 2, 2, 128, 2, (3, 0, 2), 0),
    ("bf16", 1, 2, 3, 1, 128, 37, (20, 20, 21), 0), ("f32", 2, 1, 3, 1, 64, 21, (10, 10, 11), 0), ("bf16", 1, 1, 1, 1, 64, 1, (31,), 0), ("f32", 1, 1, 1, 1, 64, 2, (31,), 0),
    ("bf16", 1, 3, 5, 5, 64, 50, (1,), 0), ("f32", 1, 2, 9, 3, 128, 130, (20, 21, 22), 0), ("bf16", 2, 3, 12, 4, 128, 300, (3, 5, 9), 0),
    ("bf16", 3, 1, 40, 8, 128, 1, (24, 20, 20), 1), ("f32", 1, 2, 2, 2, 64, 31, (4, 4, 4, 4), 0)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
@pytest.mark.parametrize("inverse", [0, 1])
def test_rotary(case, inverse):
    name, L, B, H, Hkv, d, Tq, sections, layout = case
    dtype = torch.float32 if name == "f32" else torch.bfloat16
    P = sum(sections)
    g = torch.Generator().manual_seed(P)
    freq = torch.pow(torch.tensor(1e4), -torch.arange(P) / P).float()
    pos = torch.randint(-1000, 2 ** 20, (len(sections), B, Tq), generator=g).to(torch.int32)
    pos[:, :, 0] = 0
    pos[0, 0, -1] = 2 ** 24 + 1
    Q, K = _draw(1, L, B, H, Tq, d, dtype=dtype), _draw(2, L, B, Hkv, Tq, d, dtype=dtype)
    sh, axes = _shape(L, B, H, Hkv, d, dtype), kb.make_rotary_axes(sections, layout)
    q, k = Q.cuda(), K.cuda()
    qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    args = (sh, axes, freq.cuda(), pos.cuda(), Tq)
    kb.kvev_rotary(*args, q, k, qo, ko, inverse)
    for x, y in ((Q, qo), (K, ko)):
        want = ref.rotary(x.double(), pos, freq, sections, layout == kb.ROTARY_PAIRS, inverse)
        err = (y.cpu().double() - want).abs()
        assert (err <= _bound(want, x, dtype)).all(), float(err.max())
        assert torch.equal(y.cpu()[..., 2 * P:], x[..., 2 * P:])
    # one of the two alone, and in place: the same bits
    only = torch.full_like(k, 9.0)
    kb.kvev_rotary(*args, None, k, None, only, inverse)
    assert torch.equal(only, ko)
    kb.kvev_rotary(*args, q, None, q, None, inverse)
    assert torch.equal(q, qo)


@pytest.mark.parametrize("sections,layout", [((16, 24, 24), 0), ((7, 9, 10), 0), ((7, 9, 10), 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_that_are_not_finite_stay_in_their_pairs(dtype, sections, layout):
    P, d, Tq = sum(sections), 128, 6
    x = _draw(1, 1, 1, 2, Tq, d, dtype=dtype)
    bad = x.clone()
    for t, e in ((0, 0), (1, P - 1), (2, P), (3, 2 * P - 1), (4, d - 1), (5, 40)):
        bad[..., t, e] = float("inf") if t % 2 else float("nan")
    pos = torch.arange(1, 3 * Tq + 1, dtype=torch.int32).view(3, 1, Tq)
    args = (_shape(1, 1, 2, 2, d, dtype), kb.make_rotary_axes(sections, layout), torch.linspace(0.1, 1, P).cuda(), pos.cuda(), Tq)
    y, z = (torch.empty_like(x, device="cuda") for _ in range(2))
    kb.kvev_rotary(*args, x.cuda(), None, y, None)
    kb.kvev_rotary(*args, bad.cuda(), None, z, None)
    y, z = y.cpu(), z.cpu()
    pair = lambda e: (e,) if e >= 2 * P else (e, e ^ 1) if layout else (e, e + P if e < P else e - P)
    for t, e in ((0, 0), (1, P - 1), (2, P), (3, 2 * P - 1), (4, d - 1), (5, 40)):
        hit = torch.zeros(d, dtype=torch.bool)
        hit[list(pair(e))] = True
        assert not torch.isfinite(z[0, 0, :, t, hit]).any() and torch.equal(z[0, 0, :, t, ~hit], y[0, 0, :, t, ~hit])


@pytest.mark.parametrize("layout", [0, 1])
def test_rotary_far_positions(layout):
    """The largest positions, turned by frequency 1: the angle's fraction of a turn is what 64 bits leave of it."""
    pos = torch.tensor([[[2 ** 31 - 1, -2 ** 31, 10 ** 9, 12345678]]], dtype=torch.int32)
    x = _draw(1, 1, 1, 1, 4, 64, dtype=torch.float32)
    y = torch.empty_like(x, device="cuda")
    kb.kvev_rotary(_shape(1, 1, 1, 1, 64, torch.float32), kb.make_rotary_axes((32,), layout), torch.ones(32, device="cuda"), pos.cuda(), 4, x.cuda(), None, y, None)
    want = ref.rotary(x.double(), pos, torch.ones(32), (32,), layout == 1, False)
    # 2^31 / (2 pi) turns in 53 bits: an error of 2^-24 turns or so
    assert (y.cpu().double() - want).abs().max() <= 2 * x.abs().max() * (2.0 ** -22 * 6.3 + 2.0 ** -22)


@pytest.mark.parametrize("layout,sections", [(0, (10, 11, 11)), (1, (3, 4))])
def test_inverse_is_the_gradient(layout, sections):
    L, B, H, Tq, d = 1, 2, 3, 11, 64
    sh, axes, P = _shape(L, B, H, H, d, torch.float32), kb.make_rotary_axes(sections, layout), sum(sections)
    freq = torch.pow(torch.tensor(1e4), -torch.arange(P) / P).float().cuda()
    pos = torch.randint(0, 500, (len(sections), B, Tq), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    x, g, u = (_draw(s, L, B, H, Tq, d, dtype=torch.float32).cuda() for s in (1, 2, 3))

    def turn(t, inverse=0):
        out = torch.empty_like(t)
        kb.kvev_rotary(sh, axes, freq, pos, Tq, t, None, out, None, inverse)
        return out
    grad = turn(g, 1)
    # of the formula
    y = x.cpu().double().requires_grad_()
    ref.rotary(y, pos.cpu(), freq.cpu(), sections, layout == 1, False).backward(g.cpu().double())
    assert (grad.cpu().double() - y.grad).abs().max() <= 2 * g.abs().max() * (2.0 ** -22 + 4 * 2.0 ** -24)
    # of differences: the map is linear, so a step of any size will do; 6 roundings of values up to 8 or so
    diff = ((turn(x + u) - turn(x - u)).double() / 2 * g.double()).sum()
    size = (g.double().abs() * 8).sum()
    assert abs(float(diff - (grad.double() * u.double()).sum())) <= float(size) * 16 * 2.0 ** -24
    assert (turn(turn(x), 1) - x).abs().max() <= 4 * x.abs().max() * (2.0 ** -22 + 4 * 2.0 ** -24)
