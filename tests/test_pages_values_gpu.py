"""Values of a paged cache and of the kept summaries beside it that are out of the ordinary: infinities, mantissas that are hard to
cut into terms, the largest numbers."""
import numpy as np
import pytest
import torch

from paper_2509_21354_amd import binding as kb
from tests import pages_ref as ref
from tests.test_pages_gpu import I32, cache_of, fill, frames, ints, normal, pairs, shape_of      # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def formula(Q, K, V, scale):
    """Q [R, d], K, V [n, d] float64 -> the outputs, whatever the values are."""
    with np.errstate(invalid="ignore"):
        x = (Q[:, None, :] * K[None]).sum(2) * scale
        w = np.exp(x - x.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        return (w[:, :, None] * V[None]).sum(1)


def infinite_summaries(dtype, d, L, B, Hkv, G, Tq, T, form):
    """Keys of -inf take their row out (or spoil a query that is zero or negative there), values of +-inf reach their element of
    every query, with the sign that they have; NaN where the formula gives it."""
    n, kept = T if T > 1000 else min(T, 100), 70
    sh = shape_of(L, B, Hkv * G, Hkv, d, dtype, T)
    c = cache_of(sh, 32, [n] * B, Tq=Tq, max_pages=-(-T // 32))
    assert kb.kvev_debug_page_form(sh, c.pages, Tq) == form
    pk, pv = fill(c, [n] * B, dtype)
    Kc, Vc = normal(8, L, B, Hkv, kept, d, dtype=dtype), normal(9, L, B, Hkv, kept, d, dtype=dtype)
    Q = normal(7, L, B, Hkv * G, Tq, d, dtype=dtype)
    Q[..., 3] = Q[..., 3].abs() + 1
    if G * Tq > 2:                                           # (one query sees the key of -inf with a zero, one with the other sign)
        flat = Q.view(L, B, Hkv, G * Tq, d)
        flat[:, :, :, 0, 3], flat[:, :, :, -1, 3] = 0, -1
    Q[:, ::2] = Q[:, ::2].bfloat16().to(dtype)               # (fp32: lower terms that are zero, and such that are not)
    Kc[..., 2, 3] = Kc[..., 66, 3] = -INF
    Vc[..., 0, 5], Vc[..., 65, 6], Vc[..., 1, 7], Vc[..., 69, 7], Vc[..., 64, 8] = INF, -INF, INF, -INF, NAN
    count = torch.full((L, B, Hkv), kept, dtype=I32, device="cuda")
    O = torch.full_like(Q, 9.0)
    kb.kvev_page_attention(sh, c.pages, Q, Tq, c.pool, c.table, c.length, O, c.ws_attn, Kc=Kc, Vc=Vc, count=count, k_cap=kept)
    k, v = torch.empty_like(pk), torch.empty_like(pv)
    c.read(ints([0] * B), None, n, k, v)
    for l, b, h in {(0, 0, 0), (L - 1, B - 1, Hkv - 1), (L // 2, B // 2, Hkv // 2)}:
        K, V = (torch.cat((x[l, b, h], y[l, b, h])).cpu().double().numpy() for x, y in ((Kc, k), (Vc, v)))
        q, got = (x[l, b, h * G:(h + 1) * G].reshape(G * Tq, d).cpu().double().numpy() for x in (Q, O))
        want = formula(q, K, V, d ** -0.5)
        plain = np.isfinite(want)
        assert (np.isnan(got) == np.isnan(want)).all() and (got[np.isinf(want)] == want[np.isinf(want)]).all(), (l, b, h, got[0, :10], want[0, :10])
        assert plain.any() and np.isposinf(want[:, 5]).any() and np.isneginf(want[:, 6]).any() and np.isnan(want[:, 7:9]).all()
        # the bound of the same rows without those of -inf, which weigh nothing, and without the infinite values
        rows = [i for i in range(K.shape[0]) if i not in (2, 66)]
        o, E, S = ref.attention(q, K[rows], np.where(np.isfinite(V[rows]), V[rows], 0), np.ones((G * Tq, len(rows)), bool), d ** -0.5)
        bound = ref.attention_bound(o, E, S, K.shape[0], d, dtype, form[0] > 32)
        assert (np.abs(got[plain] - want[plain]) <= bound[plain]).all()


@pytest.mark.parametrize("dtype,d,L,B,Hkv,G,Tq,T,form", [
    (torch.float32, 64, 1, 2, 2, 2, 3, 100, (16, 8, 1)), (torch.float32, 128, 1, 2, 2, 1, 1, 3000, (16, 8, 6)), (torch.float32, 64, 16, 12, 8, 1, 1, 150, (16, 1, 1)),
    (torch.bfloat16, 128, 1, 2, 2, 2, 1, 3000, (16, 8, 6)), (torch.bfloat16, 64, 16, 12, 8, 1, 2, 150, (16, 1, 1)), (torch.bfloat16, 64, 4, 24, 8, 1, 1, 600, (16, 4, 1))])
def test_infinite_summaries(dtype, d, L, B, Hkv, G, Tq, T, form):
    infinite_summaries(dtype, d, L, B, Hkv, G, Tq, T, form)


@pytest.mark.parametrize("d,L,B,Hkv,G,Tq,T,form", [(128, 1, 2, 2, 1, 30, 100, (32, 4, 1)), (64, 24, 16, 8, 1, 20, 100, (32, 1, 1))])
def test_infinite_summaries_of_pairs_of_tiles(d, L, B, Hkv, G, Tq, T, form, pairs):
    infinite_summaries(torch.bfloat16, d, L, B, Hkv, G, Tq, T, form)


@pytest.mark.parametrize("d,G,Tq,T,form", [(128, 1, 60, 100, (128, 4, 1)), (64, 2, 40, 100, (128, 4, 1)), (128, 2, 100, 100, (256, 8, 1))])
def test_infinite_summaries_of_frames(d, G, Tq, T, form, frames):
    infinite_summaries(torch.bfloat16, d, 1, 2, 2, G, Tq, T, form)


@pytest.mark.parametrize("dtype,Tq", [(torch.float32, 3), (torch.bfloat16, 3), (torch.bfloat16, 50)])
def test_query_whose_scores_are_all_minus_infinity(dtype, Tq, frames):
    """... counts as one that sees no row."""
    sh = shape_of(1, 2, 2, 1, 64, dtype)
    c = kb.PagedCache(sh, 16, 1, 1, Tq)
    Kc, Vc, Q = normal(1, 1, 2, 1, 5, 64, dtype=dtype), normal(2, 1, 2, 1, 5, 64, dtype=dtype), normal(3, 1, 2, 2, Tq, 64, dtype=dtype)
    Kc[..., 9], Q[..., 9] = -INF, Q[..., 9].abs() + 1
    O = torch.full_like(Q, 9.0)
    c.attend(Q, Tq, O, Kc=Kc, Vc=Vc, count=ints([[[5], [0]]]), k_cap=5)
    assert (O == 0).all()


def test_fp32_summaries_whose_terms_are_hard_to_cut():
    """Two summaries with one element each, whose scores of 2^16 differ by less than 1: keys that bf16 terms of full size make up, and
    bf16 keys beside them.  One product has three roundings in fp32 at most (a sum of the terms rounds at its last step, by a unit of 2^-24 or, cut
    off, two; products that are left out come to one), the other key's two; scaling and the difference are rounded at its own size."""
    B, Tq, d = 64, 16, 64
    sh = shape_of(1, B, 1, 1, d, torch.float32)
    c = kb.PagedCache(sh, 16, 1, 1, Tq)
    rng = np.random.default_rng(5)
    low = np.where(np.arange(B) % 2, 0xFFFF, rng.integers(0xFF00, 0x10000, B))
    kA = ((0x3F800000 | (rng.integers(0, 0x80, B) << 16) | low).astype(np.uint32)).view(np.float32)
    kB = torch.from_numpy(kA).bfloat16().float().numpy()
    q = ((0x3F800000 | (rng.integers(0, 0x80, (B, Tq)) << 16) | np.where(np.arange(Tq) % 2, 0xFFFF, rng.integers(0, 0x10000, (B, Tq)))).astype(np.uint32)).view(np.float32)
    kA[0], kB[0], q[0, 0] = np.uint32(0x3F80FFFF).view(np.float32), 1.0078125, np.uint32(0x3F80FFFF).view(np.float32)
    assert (np.abs(kA.astype(np.float64) - kB) <= 2.0 ** -15).all()
    Kc, Vc, Q = torch.zeros(1, B, 1, 2, d), torch.zeros(1, B, 1, 2, d), torch.zeros(1, B, 1, Tq, d)
    Kc[0, :, 0, 0, 0], Kc[0, :, 0, 1, 0] = torch.from_numpy(kA) * 2 ** 9, torch.from_numpy(kB) * 2 ** 9
    Vc[..., 0, 0], Vc[..., 1, 0] = 1, -1
    Q[0, :, 0, :, 0] = torch.from_numpy(q) * 2 ** 10
    O = torch.empty_like(Q, device="cuda")
    kb.kvev_page_attention(sh, c.pages, Q.cuda(), Tq, c.pool, c.table, c.length, O, c.ws_attn, Kc=Kc.cuda(), Vc=Vc.cuda(),
                           count=torch.full((1, B, 1), 2, dtype=I32, device="cuda"), k_cap=2)
    a, b = (q.astype(np.float64) * k[:, None] * 2.0 ** 19 / 8 for k in (kA.astype(np.float64), kB.astype(np.float64)))
    err = np.abs(O[0, :, 0, :, 0].cpu().double().numpy() - np.tanh((a - b) / 2))
    # the weights' difference moves by half of the scores'; its own roundings, exp2's and the division's are a few units
    print("largest error, in units of 2^-24 of the score:", float((err / (a * 2.0 ** -25)).max()))
    assert (err <= 5 * 2.0 ** -24 * a / 2 + 16 * 2.0 ** -24).all(), float((err / (a * 2.0 ** -25)).max())


def test_fp32_summaries_of_the_largest_values():
    """Rounded to bf16 they would be infinite.  One row, weight 1: its values come out, off by the output's rounding and the products' two."""
    sh = shape_of(1, 1, 1, 1, 64, torch.float32)
    c = kb.PagedCache(sh, 16, 1, 1)
    top = torch.tensor([0x7F7FFFFF, 0x7F7F8000, 0x7F7F7FFF, 0x7F7F8001]).to(I32).view(torch.float32)
    Kc, Vc, Q = torch.zeros(1, 1, 1, 1, 64), torch.zeros(1, 1, 1, 1, 64), torch.zeros(1, 1, 1, 1, 64)
    Kc[..., :4], Q[..., :4] = top, 2.0 ** -100
    Vc[..., :4], Vc[..., 60:] = top, -top
    O = torch.full_like(Q, 9.0, device="cuda")
    Q[..., 8:12] = top
    c.attend(Q.cuda(), 1, O, Kc=Kc.cuda(), Vc=Vc.cuda(), count=ints([[[1]]]), k_cap=1)
    assert ((O.cpu().double() - Vc.double()).abs() <= 3 * 2.0 ** -24 * Vc.double().abs()).all()


@pytest.mark.parametrize("dtype,Tq,kept", [(torch.float32, 3, 0), (torch.float32, 20, 40), (torch.bfloat16, 3, 40), (torch.bfloat16, 60, 40)])
def test_queries_that_are_not_finite_keep_to_themselves(dtype, Tq, kept, frames):
    sh = shape_of(1, 2, 4, 2, 64, dtype)
    c = cache_of(sh, 16, [130, 130], Tq=Tq)
    fill(c, [130, 130], dtype)
    Q = normal(7, 1, 2, 4, Tq, 64, dtype=dtype)
    store = (normal(8, 1, 2, 2, 40, 64, dtype=dtype), normal(9, 1, 2, 2, 40, 64, dtype=dtype), torch.full((1, 2, 2), kept, dtype=I32, device="cuda"))
    O, P = torch.empty_like(Q), torch.empty_like(Q)
    c.attend(Q, Tq, O, None, False, *store, 40)
    bad = Q.clone()
    bad[0, 0, 1, 1, 5], bad[0, 1, 2, 0, 0], bad[0, 1, 3, Tq - 1, 63] = NAN, INF, -INF
    c.attend(bad, Tq, P, None, False, *store, 40)
    hit = torch.zeros(1, 2, 4, Tq, dtype=torch.bool, device="cuda")
    hit[0, 0, 1, 1] = hit[0, 1, 2, 0] = hit[0, 1, 3, Tq - 1] = True
    assert torch.isnan(P[hit]).all() and torch.equal(P[~hit], O[~hit]) and torch.isfinite(O).all()
