"""Operators on a cache kept in pages against plain 64-bit forms, through the public entry points."""
import math

import numpy as np
import pytest
import torch

from paged_helpers import Case

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def fl():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2305_13484_amd as m
    m.load_library()
    return m


def check_attention(fl, c, plan=None, q=None):
    print("attention", c.dtype, c.n_head, c.n_kv, c.d, c.page, c.new, c.lens, c.window, c.sinks, flush=True)
    plan = plan or c.plan(fl)
    out, lse = fl.k_paged_attention(plan, c.q.cuda() if q is None else q, c.k.cuda(), c.v.cuda(), lse=True)
    ref, z, ob, lb = c.attention()
    err, lerr = (out.cpu().double() - ref).abs(), (lse.cpu().double() - z).abs()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(out.cpu()), fine)
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(ref))
    assert torch.all(err[fine] <= ob[fine]), float((err[fine] / ob[fine]).max())
    assert torch.all(lerr <= lb), float((lerr / lb).max())
    return out, lse


SHAPES = [(4, 4, 64), (8, 2, 128), (6, 2, 64), (16, 1, 128), (5, 5, 128), (24, 2, 64)]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n_head,n_kv,d", SHAPES)
def test_attention_of_single_tokens(fl, dtype, n_head, n_kv, d):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257, 700]
    check_attention(fl, Case(dtype, n_head, n_kv, d, 16, [1] * len(lens), lens, seed=d + n_head))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n_head,n_kv,d", SHAPES)
def test_attention_of_chunks(fl, dtype, n_head, n_kv, d):
    new = [1, 0, 17, 64, 3, 130, 40, 0, 1]
    lens = [1, 0, 17, 200, 90, 130, 333, 50, 64]
    check_attention(fl, Case(dtype, n_head, n_kv, d, 48, new, lens, seed=d))


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 4), (33, 40), (64, 0), (100, 17), (500, 4), (5000, 2)])
def test_attention_in_a_window(fl, dtype, d, window, sinks):
    new = [1, 1, 1, 50, 129, 5]
    lens = [1, 300, 64, 260, 129, 420]
    check_attention(fl, Case(dtype, 8, 4, d, 32, new, lens, window, sinks, seed=window))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_head,n_kv,d", [(40, 1, 128), (64, 1, 64), (34, 2, 64)])
def test_many_heads_on_one_key_head(fl, dtype, n_head, n_kv, d):
    """More than 16 rows from a single token; groups that do not divide a tile."""
    c = Case(dtype, n_head, n_kv, d, 16, [1, 1, 1, 7], [1, 40, 700, 130], seed=d)
    check_attention(fl, c)
    check_weights(fl, c, 0.5)
    check_attention(fl, Case(dtype, n_head, n_kv, d, 16, [1, 5], [300, 77], 50, 3, seed=d))


@pytest.mark.parametrize("page,lens", [(1, [1, 1, 0]), (7, [7, 3]), (16, [16])])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_smallest_pages(fl, dtype, page, lens):
    for new in ([min(n, 1) for n in lens], lens):
        c = Case(dtype, 4, 2, 64, page, new, lens, seed=page)
        check_attention(fl, c)
        check_weights(fl, c, 1.0)


def test_nothing_new_ages_the_weights_alone(fl):
    c = Case(BF, 4, 2, 64, 16, [0, 0], [40, 17], seed=1)
    w = torch.rand(2, 2, 50, device="cuda")
    ref = w.clone()
    ref[0, :, :40] *= 0.5
    ref[1, :, :17] *= 0.5
    none = torch.zeros(0, 4, 64, dtype=BF, device="cuda")
    plan = c.plan(fl)
    assert torch.equal(fl.k_paged_weights(plan, none, c.k.cuda(), torch.zeros(0, 4, device="cuda"), w, decay=0.5), ref)
    assert fl.k_paged_attention(plan, none, c.k.cuda(), c.v.cuda()).shape == (0, 4, 64)


def test_a_page_twice_in_one_sequence(fl):
    """Read, it is the same rows twice; writing to it is refused."""
    c = Case(BF, 4, 2, 64, 16, [1], [64], seed=1)
    c.table[0][2] = c.table[0][1]
    check_attention(fl, c)
    with pytest.raises(fl.FloverError, match="in use twice"):
        fl.k_paged_evict(c.plan(fl), c.k.cuda(), c.v.cuda(), torch.rand(1, 2, 64, device="cuda"), 30)
    c.table[0][3] = c.table[0][0]
    k = torch.randn(1, 2, 64, device="cuda").to(BF)
    with pytest.raises(fl.FloverError, match="another sequence"):
        fl.k_paged_append(c.plan(fl), k, k, c.k.cuda(), c.v.cuda())


def test_a_window_longer_than_any_sequence_is_none(fl):
    c = Case(BF, 8, 2, 64, 16, [1, 40], [300, 90], seed=2)
    q, k, v, lse = c.q.cuda(), c.k.cuda(), c.v.cuda(), c.attention()[1].float().cuda()
    w = torch.zeros(2, 2, 300, device="cuda")
    plans = [c.plan(fl), c.plan(fl, window=300, sinks=7), c.plan(fl, window=2 ** 31 - 1, sinks=2 ** 31 - 1)]
    outs = [(fl.k_paged_attention(p, q, k, v), fl.k_paged_weights(p, q, k, lse, w.clone())) for p in plans]
    for a, b in outs[1:]:
        assert torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1])


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("page,lens", [(16, [160]), (700, [700, 33, 1]), (333, [100, 333]), (256, [1000, 257]), (112, [500, 113])])
def test_page_sizes(fl, dtype, page, lens):
    for new in ([1] * len(lens), [min(n, 37) for n in lens]):
        check_attention(fl, Case(dtype, 4, 2, 128, page, new, lens, seed=page))


@pytest.mark.parametrize("dtype,new,length", [(BF, 1, 9000), (HF, 3, 5001), (BF, 300, 3000), (HF, 700, 700), (F32, 1, 4000), (F32, 70, 1500)])
def test_attention_of_one_long_sequence(fl, dtype, new, length):
    """Few rows over many keys: the keys are shared out and the parts joined."""
    check_attention(fl, Case(dtype, 4, 2, 128, 64, [new], [length], seed=new))
    check_attention(fl, Case(dtype, 4, 2, 64, 16, [new], [length], 1000, 5, seed=new))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("new", [1, 2, 40, 200])
def test_what_a_token_does_not_see_does_not_reach_it(fl, dtype, new):
    """Infinities and NaN in K and V of rows that only some tokens see, and of rows outside every window."""
    for window, sinks in ((0, 0), (30, 3)):
        c = Case(dtype, 8, 2, 64, 16, [new, 1], [260, 90], window, sinks, seed=new)
        for b in range(2):
            for p, x in ((c.lens[b] - 1, math.nan), (c.lens[b] - min(new, 20), math.inf), (c.lens[b] - 50, -math.inf), (5, math.nan)):
                pg = c.table[b][p // 16]
                if (p + b) % 2:
                    c.v[pg, :, p % 16, 3:9] = x
                else:
                    c.k[pg, :, p % 16, 2] = x if not math.isinf(x) else math.nan
        out, lse = fl.k_paged_attention(c.plan(fl), c.q.cuda(), c.k.cuda(), c.v.cuda(), lse=True)
        ref, z, ob, _ = c.attention()
        got, fine = out.cpu().double(), torch.isfinite(ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isinf(got), torch.isinf(ref))
        assert torch.all((got - ref).abs()[fine] <= ob[fine])
        assert torch.equal(torch.isnan(lse.cpu()), torch.isnan(z))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_large_scores(fl, dtype):
    """Scores of some hundreds: weights of one row alone, sums that must not overflow."""
    c = Case(dtype, 4, 2, 128, 16, [1, 40, 7], [100, 200, 7], seed=3)
    c.q = (c.q * 60).to(dtype)
    check_attention(fl, c)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
def test_rows_of_a_packed_projection_and_rows_off_the_grid(fl, dtype, d):
    c = Case(dtype, 8, 2, d, 16, [30, 1, 5], [30, 77, 40], seed=8)
    plan = c.plan(fl)
    ref = fl.k_paged_attention(plan, c.q.cuda(), c.k.cuda(), c.v.cuda())
    packed = torch.zeros((c.T, 12, d), dtype=dtype, device="cuda")
    packed[:, :8] = c.q.cuda()
    flat = torch.zeros(c.T * 8 * d + 1, dtype=dtype, device="cuda")
    flat[1:] = c.q.cuda().reshape(-1)
    turned = c.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    for q in (packed[:, :8], flat[1:].view(c.T, 8, d), turned):
        assert torch.equal(fl.k_paged_attention(plan, q, c.k.cuda(), c.v.cuda()), ref)
    k, v = torch.randn(c.T, 2, d).to(dtype), torch.randn(c.T, 2, d).to(dtype)
    packed[:, 8:10], packed[:, 10:] = k.cuda(), v.cuda()
    a = fl.k_paged_append(plan, k.cuda(), v.cuda(), c.k.cuda(), c.v.cuda())
    b = fl.k_paged_append(plan, packed[:, 8:10], packed[:, 10:], c.k.cuda(), c.v.cuda())
    for x, y in zip(a, b):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_sequences_that_share_pages(fl):
    """A common prefix read by three sequences; writing to it is refused, in every form."""
    c = Case(BF, 8, 2, 128, 16, [1, 5, 20], [70, 100, 100], seed=4, share=((1, 0, 4), (2, 0, 2)))
    plan = c.plan(fl)
    check_attention(fl, c, plan)
    w = torch.rand(3, 2, 100, device="cuda")
    with pytest.raises(fl.FloverError, match="in use twice"):
        fl.k_paged_evict(plan, c.k.cuda(), c.v.cuda(), w, 50)
    k = torch.randn(26, 2, 128, device="cuda").to(BF)
    kc, vc = fl.k_paged_append(plan, k, k, c.k.cuda(), c.v.cuda())       # the new rows lie in pages of their own
    assert torch.isfinite(kc[c.table[0][4], :, 5].float()).all()
    shared = Case(BF, 8, 2, 128, 16, [1, 1], [70, 70], seed=4, share=((1, 0, 5),))
    k = torch.randn(2, 2, 128, device="cuda").to(BF)
    with pytest.raises(fl.FloverError, match="another sequence"):
        fl.k_paged_append(shared.plan(fl), k, k, shared.k.cuda(), shared.v.cuda())


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n_kv,d,page", [(1, 64, 16), (5, 128, 48), (8, 64, 256)])
def test_append(fl, dtype, n_kv, d, page):
    print("append", dtype, n_kv, d, page, flush=True)
    c = Case(dtype, n_kv, n_kv, d, page, [1, 0, 40, 3, 200], [1, 30, 40, 50, 333], seed=d, stale=0.5)
    k, v = torch.randn(c.T, n_kv, d).to(dtype), torch.randn(c.T, n_kv, d).to(dtype)
    kc, vc = c.k.clone(), c.v.clone()
    t = 0
    for b, n in enumerate(c.new):
        for p in range(c.lens[b] - n, c.lens[b]):
            kc[c.table[b][p // page], :, p % page], vc[c.table[b][p // page], :, p % page] = k[t], v[t]
            t += 1
    got = fl.k_paged_append(c.plan(fl), k.cuda(), v.cuda(), c.k.cuda(), c.v.cuda())
    assert torch.equal(got[0].cpu(), kc) and torch.equal(got[1].cpu(), vc)


def check_weights(fl, c, decay):
    print("weights", c.dtype, c.n_head, c.n_kv, c.d, c.page, c.new, c.lens, c.window, c.sinks, flush=True)
    lse = c.attention()[1].float()
    g = torch.Generator().manual_seed(1)
    old = torch.rand((len(c.new), c.n_kv, max(c.lens) + 3), generator=g)
    ref, bound = c.weights(lse, old, decay)
    got = fl.k_paged_weights(c.plan(fl), c.q.cuda(), c.k.cuda(), lse.cuda(), old.cuda(), decay=decay).cpu()
    for b, n in enumerate(c.lens):
        assert torch.equal(got[b, :, n:], old[b, :, n:])
        assert torch.all((got[b, :, :n].double() - ref[b, :, :n]).abs() <= bound[b, :, :n])
    return got


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n_head,n_kv,d", SHAPES)
def test_weights(fl, dtype, n_head, n_kv, d):
    check_weights(fl, Case(dtype, n_head, n_kv, d, 16, [1] * 6, [1, 16, 33, 65, 257, 600], seed=d), 1.0)
    check_weights(fl, Case(dtype, n_head, n_kv, d, 48, [1, 0, 17, 64, 130, 0, 40], [1, 0, 17, 200, 130, 9, 333], seed=d), 0.5)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (33, 40), (100, 17), (500, 4)])
def test_weights_in_a_window(fl, dtype, d, window, sinks):
    check_weights(fl, Case(dtype, 8, 4, d, 32, [1, 1, 50, 129, 5, 300], [1, 300, 260, 129, 420, 700], window, sinks, seed=window), 0.0)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64), (F32, 128), (F32, 64)])
def test_weights_of_many_blocks(fl, dtype, d):
    """More than 128 blocks of 128 positions (the waves of a block share the rows), more than 1024 of 512 (longer blocks of the streaming kernel)."""
    check_weights(fl, Case(dtype, 16, 8, d, 64, [70, 130, 0], [1500, 1000, 30], seed=d), 0.9)
    check_weights(fl, Case(dtype, 6, 6, d, 16, [90, 200], [1700, 1200], 300, 40, seed=d), 0.9)
    check_weights(fl, Case(dtype, 8, 8, d, 16, [1] * 132, [5 + 3 * i for i in range(132)], seed=d), 0.9)


def test_weights_without_decay_overwrite_whatever_was_there(fl):
    c = Case(BF, 4, 2, 64, 16, [1, 2], [40, 30], seed=1)
    lse = c.attention()[1].float().cuda()
    args = (c.plan(fl), c.q.cuda(), c.k.cuda(), lse)
    clean = fl.k_paged_weights(*args, torch.zeros(2, 2, 40, device="cuda"), decay=0.0)
    dirty = fl.k_paged_weights(*args, torch.full((2, 2, 40), math.nan, device="cuda"), decay=0.0)
    assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1, :, :30], dirty[1, :, :30]) and torch.isnan(dirty[1, :, 30:]).all()


def test_weights_of_all_tokens_sum_to_their_number(fl):
    """Every new token gives one unit per head in all."""
    c = Case(BF, 8, 2, 128, 16, [40, 1], [200, 3000], seed=1)
    plan = c.plan(fl)
    q, k = c.q.cuda(), c.k.cuda()
    _, lse = fl.k_paged_attention(plan, q, k, c.v.cuda(), lse=True)
    w = fl.k_paged_weights(plan, q, k, lse, torch.zeros(2, 2, 3000, device="cuda"))
    assert torch.allclose(w.sum(2).cpu(), torch.tensor([[160.0, 160.0], [4.0, 4.0]]), rtol=1e-5)


def check_evict(fl, c, weights, budget, first, recent, in_place):
    print("evict", c.dtype, c.n_kv, c.d, c.page, c.lens, budget, first, recent, in_place, flush=True)
    k, v, kept = c.evicted(weights, budget, first, recent)
    kc, vc, w = c.k.cuda(), c.v.cuda(), weights.cuda()
    out = None if in_place else torch.full((len(c.lens), c.n_kv, min(budget, max(c.lens)) + 2), -7.0, device="cuda")
    got = fl.k_paged_evict(c.plan(fl), kc, vc, w, budget, first, recent, weights_out=out).cpu()
    assert torch.equal(kc.cpu().nan_to_num(9.0), k.nan_to_num(9.0)) and torch.equal(vc.cpu().nan_to_num(9.0), v.nan_to_num(9.0))
    rest = weights if in_place else torch.full_like(out, -7.0).cpu()
    out = (w if in_place else out).cpu()
    for b in range(len(c.lens)):
        for h in range(c.n_kv):
            keep = kept[b][h]
            n = len(keep)
            assert got[b, h].tolist() == keep + [-1] * (budget - n)
            assert torch.equal(out[b, h, :n].nan_to_num(5.0), weights[b, h, keep].nan_to_num(5.0))
            assert torch.equal(out[b, h, n:].nan_to_num(5.0), rest[b, h, n:].nan_to_num(5.0))


@pytest.mark.parametrize("dtype,n_kv,d,page", [(BF, 2, 128, 16), (HF, 3, 64, 48), (F32, 1, 128, 256)])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 4, 16), (100, 50, 50), (300, 0, 299), (1000, 3, 0), (2000, 4, 100)])
def test_evict(fl, dtype, n_kv, d, page, budget, first, recent):
    lens = [0, 1, 64, 65, 300, 301, 1025, 2500]
    c = Case(dtype, n_kv, n_kv, d, page, [0] * len(lens), lens, seed=budget)
    g = torch.Generator().manual_seed(budget)
    w = torch.exp(2 * torch.randn((len(lens), n_kv, max(lens)), generator=g))
    check_evict(fl, c, w, budget, first, recent, in_place=budget % 2 == 0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_evict_many_sequences(fl, dtype):
    """Enough sequences for the wider pieces of a row."""
    lens = [20 + 11 * i for i in range(40)]
    c = Case(dtype, 4, 4, 128, 32, [0] * len(lens), lens, seed=3)
    check_evict(fl, c, torch.rand((len(lens), 4, max(lens)), generator=torch.Generator().manual_seed(3)), 150, 3, 40, in_place=False)


def test_evict_from_a_long_sequence(fl):
    """More positions than a block holds in LDS, ties across that border."""
    c = Case(HF, 1, 1, 64, 256, [0, 0], [21000, 19000], seed=3)
    w = torch.rand((2, 1, 21000), generator=torch.Generator().manual_seed(3))
    w[1] = (w[1] * 40).floor()
    check_evict(fl, c, w, 9000, 3, 40, in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_ties_zeros_and_weights_that_are_no_numbers(fl, in_place):
    c = Case(BF, 2, 2, 64, 16, [0] * 4, [700, 1500, 40, 2100], seed=6)
    g = torch.Generator().manual_seed(2)
    w = torch.randint(-2, 3, (4, 2, 2100), generator=g).float()          # many ties, some below zero
    w[0, 0] = 1.0
    w[1, 0, ::3] = -0.0
    w[1, 1, ::5] = math.nan
    w[3, 0, ::7], w[3, 0, 1::7], w[3, 1] = math.inf, -math.inf, math.nan
    for budget, first, recent in ((300, 0, 0), (39, 5, 5), (1000, 4, 64)):
        check_evict(fl, c, w, budget, first, recent, in_place)


def test_a_decode_loop_with_appends_windows_and_evictions(fl):
    """A chunk, then single tokens, weights accumulated, the cache cut back whenever it outgrows its budget: every step against the same
    loop in 64 bits, which takes over the rows that the library kept."""
    torch.manual_seed(0)
    n_head, n_kv, d, page, budget, pages = 8, 2, 64, 16, 48, 40
    group = n_head // n_kv
    table = np.random.default_rng(0).permutation(pages).reshape(2, -1)[:, :20]
    kc = torch.full((pages, n_kv, page, d), math.nan, dtype=BF, device="cuda")
    vc = kc.clone()
    weights = torch.zeros(2, n_kv, 20 * page, device="cuda")
    held = [[[] for _ in range(n_kv)] for _ in range(2)]          # rows (k, v, weight) per sequence and key head
    lens, plan = [0, 0], None
    for step in range(40):
        new = [30, 41] if step == 0 else [1, 1 if step % 3 else 0]
        lens = [a + b for a, b in zip(lens, new)]
        if plan is None:
            plan = fl.PagedPlan(BF, n_head, n_kv, d, page, pages, new, lens, table)
        else:
            plan.update(new, lens, table)
        t = sum(new)
        q, k, v = (torch.randn(t, h, d).to(BF) for h in (n_head, n_kv, n_kv))
        fl.k_paged_append(plan, k.cuda(), v.cuda(), kc, vc)
        out, lse = fl.k_paged_attention(plan, q.cuda(), kc, vc, lse=True)
        fl.k_paged_weights(plan, q.cuda(), kc, lse, weights, decay=0.9)
        out, at = out.cpu().double(), 0
        for b in range(2):
            for h in range(n_kv):
                rows = held[b][h]
                for r in rows:
                    r[2] *= 0.9
                rows += [[k[at + i, h].double(), v[at + i, h].double(), 0.0] for i in range(new[b])]
                for i in range(new[b]):
                    seen = rows[:lens[b] - new[b] + i + 1]
                    keys, vals = torch.stack([r[0] for r in seen]), torch.stack([r[1] for r in seen])
                    for x in range(group):
                        p = torch.softmax(keys @ q[at + i, h * group + x].double() / math.sqrt(d), 0)
                        err = (out[at + i, h * group + x] - p @ vals).abs()
                        assert torch.all(err <= 2.0 ** -8 * 1.01 * (p @ vals).abs() + (2.0 ** -8 + 1e-5) * (p @ vals.abs()))
                        for r, w in zip(seen, p.tolist()):
                            r[2] += w
            at += new[b]
        got = weights.cpu()
        for b in range(2):
            for h in range(n_kv):
                ref = torch.tensor([r[2] for r in held[b][h]], dtype=torch.float64)
                assert torch.allclose(got[b, h, :lens[b]].double(), ref, rtol=1e-5, atol=1e-6)
        if max(lens) > budget + 8:
            kept = fl.k_paged_evict(plan, kc, vc, weights, budget, first=2, recent=10).cpu()
            for b in range(2):
                for h in range(n_kv):
                    keep = [p for p in kept[b, h].tolist() if p >= 0]
                    assert len(keep) == min(lens[b], budget)
                    if lens[b] > budget:
                        lightest = min(held[b][h][p][2] for p in keep[2:-10])
                        gone = [held[b][h][p][2] for p in range(lens[b]) if p not in keep]
                        assert max(gone) <= lightest * (1 + 1e-4)
                    held[b][h] = [held[b][h][p] for p in keep]
            lens = [min(n, budget) for n in lens]


def test_the_cache_of_the_fused_step_is_one_of_single_pages(fl):
    """A context of the framework: its slots are pages, and its rows are attended to where they lie."""
    import flover_synth as synth
    cfg = synth.small_llama16(synth.DT_BF16)
    gpu = fl.Flover(cfg, {k: v.cuda() for k, v in synth.make_weights(cfg, 1).items()})
    g = torch.Generator().manual_seed(4)
    for rid, n in ((5, 33), (6, 70), (7, 12)):
        gpu.add_request(rid, torch.randint(0, cfg.V, (n,), generator=g).tolist(), 10)
    gpu.step()
    st = gpu.state()
    slots = [int(i) for i in range(cfg.C) if st["state"][i] == 2]
    lens = [int(st["len"][i]) for i in slots]
    k, v = gpu.kv_cache()[1]
    q = torch.randn(len(slots), cfg.nh, cfg.d, generator=g).to(BF).cuda()
    plan = fl.PagedPlan(BF, cfg.nh, cfg.nh, cfg.d, cfg.S, cfg.C, [1] * len(slots), lens, [[s] for s in slots])
    got = fl.k_paged_attention(plan, q, k, v).float()
    ref = fl.k_decode_attention(q, k, v, slots, lens).float()
    assert len(slots) == 3 and torch.all((got - ref).abs() <= 2.0 ** -7 * (1 + ref.abs()))
    gpu.close()


def test_rows_beyond_four_gigabytes(fl):
    """Pages at the far end of caches of 5 GB and more, among them the last."""
    n_pages, n_kv, page, d = 21000, 8, 128, 128                         # 5.5 GB each
    k = torch.zeros((n_pages, n_kv, page, d), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    far = [n_pages - 1, n_pages - 7, 20001, 3]
    small = Case(BF, 16, 8, d, page, [9, 1], [300, 100], seed=5, stale=0.0)
    table, at = [], 0
    for row in small.table:
        table.append(far[at:at + len(row)])
        at += len(row)
        for a, b in zip(table[-1], row):
            k[a], v[a] = small.k[b].cuda(), small.v[b].cuda()
    plan = fl.PagedPlan(BF, 16, 8, d, page, n_pages, small.new, small.lens, table)
    ref_plan, q = small.plan(fl), small.q.cuda()
    out, lse = fl.k_paged_attention(plan, q, k, v, lse=True)
    ref, z = fl.k_paged_attention(ref_plan, q, small.k.cuda(), small.v.cuda(), lse=True)
    assert torch.equal(out, ref) and torch.equal(lse, z)
    w = torch.rand(2, 8, 300, device="cuda")
    assert torch.equal(fl.k_paged_weights(plan, q, k, lse, w.clone()), fl.k_paged_weights(ref_plan, q, small.k.cuda(), lse, w.clone()))
    x = torch.randn(10, 8, d, device="cuda").to(BF)
    fl.k_paged_append(plan, x, x, k, v)
    assert torch.equal(k[table[0][-1], :, 299 % page], x[8])
    rk, rv = small.k.cuda(), small.v.cuda()
    fl.k_paged_append(ref_plan, x, x, rk, rv)
    assert torch.equal(fl.k_paged_evict(plan, k, v, w.clone(), 50), fl.k_paged_evict(ref_plan, rk, rv, w.clone(), 50))
    for a, b in zip(sum(table, []), sum(small.table, [])):
        assert torch.equal(k[a], rk[b]) and torch.equal(v[a], rv[b])


def test_streams_plans_and_repeated_calls(fl):
    """The same bits on another stream, from a plan set again, and beside another plan's calls."""
    a, b = Case(BF, 8, 2, 128, 16, [1, 60], [3000, 90], seed=1), Case(HF, 4, 4, 64, 32, [1], [5000], 100, 4, seed=2)
    pa, pb = a.plan(fl), b.plan(fl)
    qa, ka, va, qb, kb, vb = (t.cuda() for t in (a.q, a.k, a.v, b.q, b.k, b.v))
    ra, rb = fl.k_paged_attention(pa, qa, ka, va), fl.k_paged_attention(pb, qb, kb, vb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(sa):
            xa = fl.k_paged_attention(pa, qa, ka, va)
        with torch.cuda.stream(sb):
            xb = fl.k_paged_attention(pb, qb, kb, vb)
            fresh = b.plan(fl)                        # set on this stream, used on the other
        torch.cuda.current_stream().wait_stream(sb)
        xc = fl.k_paged_attention(fresh, qb, kb, vb)
        torch.cuda.synchronize()
        assert torch.equal(xa, ra) and torch.equal(xb, rb) and torch.equal(xc, rb)
    pa.update([1], [40], [a.table[0]])
    assert torch.equal(fl.k_paged_attention(pa, qa[:1].contiguous(), ka, va),
                       fl.k_paged_attention(fl.PagedPlan(BF, 8, 2, 128, 16, a.n_pages, [1], [40], [a.table[0]]), qa[:1].contiguous(), ka, va))
    pa.update(a.new, a.lens, a.table)
    assert torch.equal(fl.k_paged_attention(pa, qa, ka, va), ra)


def test_captured_calls(fl):
    """Append, attention and weights in a graph, replayed among eager work, two graphs with plans of their own."""
    cases = [Case(BF, 8, 2, 128, 16, [1, 70], [2500, 90], seed=1, stale=0.0), Case(BF, 8, 2, 128, 16, [1, 1, 20], [700, 1, 50], 64, 4, seed=2, stale=0.0)]
    runs = []
    for c in cases:
        plan = c.plan(fl)
        t = dict(q=c.q.cuda(), k=torch.randn(c.T, 2, 128, device="cuda").to(BF), v=torch.randn(c.T, 2, 128, device="cuda").to(BF), kc=c.k.cuda(), vc=c.v.cuda(),
                 w=torch.zeros(len(c.new), 2, max(c.lens), device="cuda"))
        def call(plan=plan, t=t):
            fl.k_paged_append(plan, t["k"], t["v"], t["kc"], t["vc"])
            out, lse = fl.k_paged_attention(plan, t["q"], t["kc"], t["vc"], lse=True)
            return out, lse, fl.k_paged_weights(plan, t["q"], t["kc"], lse, t["w"], decay=0.0)
        ref = [x.clone() for x in call()]
        for b, n in enumerate(c.lens):
            ref[2][b, :, n:] = 3.0                    # behind a sequence stays what is put there below
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = call()
        runs.append((graph, outs, ref, call, t))
    for _ in range(3):
        for graph, outs, ref, call, t in runs:
            outs[0].zero_()
            t["w"].fill_(3.0)
            graph.replay()
            for x, y in zip(outs, ref):
                assert torch.equal(x, y)
            call()
    torch.cuda.synchronize()
    plan = cases[0].plan(fl)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(fl.FloverError, match="captured"):
        with torch.cuda.graph(graph):
            plan.update(cases[0].new, cases[0].lens, cases[0].table)


def test_refusals_of_the_calls(fl):
    c = Case(BF, 8, 2, 64, 16, [1, 3], [20, 30], seed=1, stale=0.0)
    plan, q, k, v = c.plan(fl), c.q.cuda(), c.k.cuda(), c.v.cuda()
    w, lse = torch.zeros(2, 2, 30, device="cuda"), torch.zeros(4, 8, device="cuda")
    new = torch.zeros(4, 2, 64, dtype=BF, device="cuda")
    bad = [lambda: fl.k_paged_attention(plan, q[:3], k, v), lambda: fl.k_paged_attention(plan, q.half(), k, v),
           lambda: fl.k_paged_attention(plan, q, k[:1], v), lambda: fl.k_paged_attention(plan, q, k, v.transpose(1, 2)),
           lambda: fl.k_paged_attention(plan, q, k, v, out=q), lambda: fl.k_paged_attention(plan, q, k, v, out=torch.empty_like(q)[:3]),
           lambda: fl.k_paged_attention(plan, q, k, v, lse=lse.double()), lambda: fl.k_paged_attention(plan, q, k.cpu(), v),
           lambda: fl.k_paged_append(plan, new, new, k, k), lambda: fl.k_paged_append(plan, new[:, :1], new, k, v),
           lambda: fl.k_paged_weights(plan, q, k, lse, w[:, :, :29]), lambda: fl.k_paged_weights(plan, q, k, lse, w.half()),
           lambda: fl.k_paged_evict(plan, k, v, w, 0), lambda: fl.k_paged_evict(plan, k, v, w, 10, 6, 5),
           lambda: fl.k_paged_evict(plan, k, k, w, 10), lambda: fl.k_paged_evict(plan, k, v, w, 10, -1, 0),
           lambda: fl.k_paged_evict(plan, k, v, w, 10, weights_out=w[:, :, 5:15]),
           lambda: fl.k_paged_evict(plan, k, v, w, 10, weights_out=torch.zeros(2, 2, 9, device="cuda")),
           lambda: fl.k_paged_evict(plan, k, v, w, 10, kept=torch.zeros(2, 2, 10, device="cuda"))]
    for i, f in enumerate(bad):
        with pytest.raises(fl.FloverError):
            f()
            print("call", i, "was not refused")
    empty = fl.PagedPlan(BF, 8, 2, 64, 16, 4, [], [], [])
    none = torch.zeros(0, 8, 64, dtype=BF, device="cuda")
    assert fl.k_paged_attention(empty, none, torch.zeros(4, 2, 16, 64, dtype=BF, device="cuda"), torch.zeros(4, 2, 16, 64, dtype=BF, device="cuda")).shape == (0, 8, 64)
    assert fl.k_paged_attention(plan, q, k, v).shape == q.shape           # and it still works after the refused calls
