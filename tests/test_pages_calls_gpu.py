"""Paged calls and rotary positions: signs of zeros, calls on a stream of their own, copies of many pages, elements each against its own
pair."""
import random

import numpy as np
import pytest
import torch

from paper_2509_21354_amd import binding as kb
from tests import pages_ref as ref
from tests.test_pages_gpu import cache_of, edge_blocks, ints, normal, shape_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_signs_of_rows(dtype, d):
    """Zeros, and what is rounded to zero, keep their sign."""
    per, blocks = d // 32, edge_blocks(dtype)
    n = blocks.shape[0] // per
    x = blocks[:n * per].reshape(1, 1, 1, n, d).contiguous()
    c = cache_of(shape_of(H=1, d=d, dtype=dtype), 32, [n])
    K, V = x.cuda(), -x.cuda()
    k, v = torch.empty_like(K), torch.empty_like(V)
    c.start.zero_()
    c.append(K, V, n)
    c.read(c.start, None, n, k, v)
    want = ref.cache_values(x)
    there = ~np.isnan(want)
    assert ((want == 0) & (x.double().numpy() < 0) & there).any() and ((want == 0) & np.signbit(x.double().numpy()) & (x.double().numpy() == 0)).any()
    for got, sign in ((k, np.signbit(want)), (v, ~np.signbit(want))):
        got = got.cpu().double().numpy()
        assert np.array_equal(np.signbit(got)[there], sign[there]), np.argwhere(there & (np.signbit(got) != sign))[:5]


def test_every_call_keeps_to_its_stream():
    """The calls of a cache's life on a stream that has other work first, their inputs made behind that work: a call that ran on another
    stream, or before what stands in front of it, would meet zeros, empty tables and rows that are not there yet."""
    sh, page = shape_of(L=2, B=3, H=4, H_kv=2, d=64), 16
    axes, freq, to = kb.make_rotary_axes((32,)), torch.linspace(1, 0.1, 32).cuda(), kb.make_pages(page, 30, 8)
    Tn = 40
    src = dict(Q=normal(1, 2, 3, 4, Tn, 64), K=normal(2, 2, 3, 2, Tn, 64), V=normal(3, 2, 3, 2, Tn, 64), pos=torch.arange(Tn).repeat(1, 3, 1).to(torch.int32).cuda(),
               new=ints([40, 17, 0]), one=ints([0]), two=ints([2]), keep=ints([25, 9, 30]), first=ints([0, 0, 16]), pair=ints([29]))
    busy = torch.randn(4096, 4096, device="cuda")

    def life(on):
        c = kb.PagedCache(sh, page, 30, 8, Tn)
        c.pool.zero_()
        t = {k: torch.zeros_like(v) for k, v in src.items()}
        O, k, v, start = torch.zeros_like(src["Q"]), torch.zeros_like(src["K"]), torch.zeros_like(src["V"]), ints([0] * 3)
        pool, table, refs = torch.zeros(kb.page_pool_bytes(sh, to), dtype=torch.uint8, device="cuda"), ints([[-9] * 8] * 3), ints([-9] * 30)
        ws = kb.alloc_workspace(kb.page_workspace_bytes(kb.OP_PAGES_COMPACT, sh, c.pages, 0))
        torch.cuda.synchronize()
        with torch.cuda.stream(on):
            if on != torch.cuda.default_stream():
                for _ in range(30):                              # some tens of milliseconds
                    busy @ busy
            for name in src:
                t[name].copy_(src[name])
            kb.kvev_rotary(sh, axes, freq, t["pos"], Tn, t["Q"], t["K"], t["Q"], t["K"])
            c.reserve(t["new"])
            c.append(t["K"], t["V"], Tn, t["new"])
            c.fork(t["one"], t["two"], 1)
            c.trim(None, 3, None, t["keep"])
            c.reserve(t["new"])                                  # (row 0 goes on in a shared page)
            c.attend(t["Q"], Tn, O, t["first"], True)
            c.read(start, c.length, Tn, k, v)
            kb.kvev_pages_copy(sh, c.pages, c.pool, t["one"], t["pair"], 1, c.status)
            kb.kvev_pages_compact(sh, c.pages, c.pool, c.table, c.refs, to, pool, table, refs, c.status, ws)
        on.synchronize()
        return [x.clone() for x in (t["Q"], t["K"], O, k, v, c.pool, c.table, c.length, c.refs, c.status, pool, table, refs)]
    want = life(torch.cuda.default_stream())
    assert want[2].any() and want[3].any() and (want[11] >= 0).any() and want[7].tolist() == [65, 26, 30] and int(want[9]) == 0
    for x, y in zip(want, life(torch.cuda.Stream())):
        assert torch.equal(x, y)


@pytest.mark.parametrize("L,n_pages,n", [(1, 40, 40), (3, 700, 300), (2, 6000, 5000)])
def test_copies_of_many_pages(L, n_pages, n):
    """Pairs of which some are refused: twice the same destination, chains, places outside; more of them than workgroups."""
    rng = random.Random(n)
    sh = shape_of(L=L, B=1, H=1, d=64)
    c = kb.PagedCache(sh, 16, n_pages, 2)
    c.pool.random_(0, 256)
    before = c.pool.view(L, n_pages, -1).clone()
    src, dst = [rng.randrange(n_pages // 2) for _ in range(n)], rng.sample(range(n_pages // 2, n_pages), min(n, n_pages // 2)) + [rng.randrange(n_pages) for _ in range(n - n_pages // 2)]
    rng.shuffle(dst)
    for i in rng.sample(range(n), n // 20):
        (src if rng.random() < 0.5 else dst)[i] = rng.choice((-1, n_pages, 2 ** 31 - 1, -2 ** 31, rng.randrange(n_pages)))
    assert len(dst) == n
    want, written, seen, refused = before.clone(), set(dst), set(), 0
    for s, d in zip(src, dst):
        if 0 <= s < n_pages and 0 <= d < n_pages and d not in seen and s not in written:
            want[:, d] = before[:, s]
        else:
            refused += 1
        seen.add(d)
    assert 0 < refused < n
    kb.kvev_pages_copy(sh, c.pages, c.pool, ints(src), ints(dst), n, c.status)
    assert torch.equal(c.pool.view(L, n_pages, -1), want) and int(c.status) == kb.PAGES_BAD_PAIR


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,sections,layout", [(128, (16, 24, 24), 0), (64, (7, 9, 10), 0), (128, (20, 21), 1)])
def test_rotary_elements_against_their_own_pair(dtype, d, sections, layout):
    """Pairs of sizes from 1 to 1e-6 side by side.  The turn is rounded once, by 2^-26 of a turn at most, 1.6 units of 2^-24 as an angle;
    sine and cosine are within 2 units of their own; together 3.6, on both elements of a pair of length r at most 5.1 r; two products
    and a sum add 2 r.  bf16: half a step of the output as well."""
    P, L, B, H, Tq = sum(sections), 1, 2, 3, 60
    g = torch.Generator().manual_seed(P)
    freq = torch.pow(torch.tensor(1e4), -torch.arange(P) / P).float()
    pos = torch.randint(-1000, 2 ** 20, (len(sections), B, Tq), generator=g).to(torch.int32)
    x = torch.randn(L, B, H, Tq, d, generator=g)
    a, b = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout else (slice(0, P), slice(P, 2 * P))
    size = 10.0 ** -(torch.arange(P) % 7).float()
    x[..., a], x[..., b] = x[..., a] * size, x[..., b] * size
    x = x.to(dtype)
    y = torch.empty_like(x, device="cuda")
    sh = kb.make_shape(L=L, B=B, H=H, H_kv=H, d=d, T=0, T_cap=1, C=1, N_cap=0, W=0, d_sum=1, d_g=1, dtype=kb.F32 if dtype == torch.float32 else kb.BF16)
    kb.kvev_rotary(sh, kb.make_rotary_axes(sections, layout), freq.cuda(), pos.cuda(), Tq, x.cuda(), None, y, None)
    want, y = ref.rotary(x.double(), pos, freq, sections, layout == kb.ROTARY_PAIRS, 0), y.cpu().double()
    r = torch.hypot(x[..., a].double(), x[..., b].double())
    for e in (a, b):
        bound = 8 * 2.0 ** -24 * r + (want[..., e].abs() * 2.0 ** -8 if dtype == torch.bfloat16 else 0)
        err = (y[..., e] - want[..., e]).abs()
        assert (err <= bound).all(), float((err / bound).max())
