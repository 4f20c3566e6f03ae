"""Attention over the cache held in 4 bits, in each of its forms (few rows of 16 and of 32, many rows with and without splits, one or
several segments of 512 pages), against the definition in fp64 with bounds that follow the weights."""
import numpy as np
import pytest
import torch

import paper_2605_25475_amd as im
from helpers import f64
from packed_model import close
from test_packed_gpu import DEV, Pair

pytestmark = pytest.mark.gpu

# queries per sequence that the handle is made for, queries, heads
FORMS = {"16 rows": (1, 4, (4, 2)), "32 rows": (64, 16, (4, 2)), "2 x 32 rows": (64, 30, (4, 2)), "many": (1, 40, (4, 2)),
         "many, few rows": (1, 20, (4, 2)), "many, in splits": (128, 40, (4, 2)), "many, 3 tiles in splits": (128, 70, (4, 1))}


def expect(p, q, q_pos=None, lost=None):
    """(output, tolerance, NaN outputs) of q [B, n_q, H, 128]; lost [B, Hk, C]: entries that are not there.

    A weight is off by the error of its logit (fp32 sums of exact products, exp2, its argument: below 2^-17 of the sum of |q k| scale)
    and by its rounding: two bf16 parts (2^-17) up to 64 rows a unit on a handle that is made for them, else one fp16 value: half a step
    of 2^-11, or 2^-32 of the largest weight where it is below 2^-21 of it.  fp32 sums of n terms, 16 in a product: (n / 16 + 64)
    roundings of 2^-24.  The output is a quotient: twice that, of the weighted sum of |v|.  The readout is off by 2^-15 of the sum of its
    terms, the output by half a step of its rounding, 2^-8 of it, and by 2^-122 where the scales go to their end."""
    r, g = p.ref, p.H // p.Hk
    B, n_q = q.shape[:2]
    out, tol, nan = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape, bool)
    fp16 = n_q * g > 16 and (n_q * g > 64 or p.cfg.max_queries < n_q)
    for b in range(B):
        for h in range(p.Hk):
            n = int(r.len[b, h])
            K, V = r.K[b, h, :n], r.V[b, h, :n]
            x = q[b, :, h * g:(h + 1) * g].reshape(n_q * g, 128)
            seen = np.ones((n_q, n), bool) if q_pos is None else r.pos[b, h, :n][None] <= np.asarray(q_pos)[b][:, None]
            if lost is not None:
                seen = seen & ~lost[b, h, :n]
            seen = seen.repeat(g, 0)
            bad = seen.astype(float) @ np.isnan(V) + (seen.astype(float) @ np.isnan(K).any(1, keepdims=True)) > 0
            K, V = np.nan_to_num(K), np.nan_to_num(V)
            logit = np.where(seen, x @ K.T * r.cfg.softmax_scale, -np.inf)
            top = logit.max(1, keepdims=True, initial=-1e300)
            w = np.exp(logit - top)
            total = w.sum(1, keepdims=True)
            w = w / np.where(total > 0, total, 1)
            size = np.where(seen, np.abs(x) @ np.abs(K).T * r.cfg.softmax_scale, 0).max(1, keepdims=True, initial=0)
            eps = (2.0 ** -12 if fp16 else 0) + 2.0 ** -16 + 2.0 ** -17 * size + (n / 16 + 64) * 2.0 ** -24
            t = 2 * eps * (w @ np.abs(V)) + (2.0 ** -31 * (seen @ np.abs(V)) if fp16 else 0)
            phi = x @ r.p.Wtheta.T
            den = ((phi * phi) @ r.b[b, h] + r.cfg.mem_eps)[:, None]
            gate = 1 / (1 + np.exp(-(x @ r.p.wg + r.p.cg)))[:, None]
            o = w @ V + gate * (phi @ r.M[b, h]) / den
            t = t + 2.0 ** -15 * gate * (np.abs(phi) @ np.abs(r.M[b, h])) / den + 2.0 ** -8 * np.abs(o) + 2.0 ** -122
            sl = (b, slice(None), slice(h * g, (h + 1) * g))
            out[sl], tol[sl], nan[sl] = (a.reshape(n_q, g, 128) for a in (o, t, bad))
    return out, tol, nan


def check(p, q, q_pos=None, lost=None, status=0):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    qp = None if q_pos is None else torch.tensor(np.ascontiguousarray(q_pos), dtype=torch.int32, device=DEV)
    im.im_attn_packed_with_readout(p.h, p.p, p.st, q.cuda(), out, qp)
    assert im.im_query_status(p.h) == status
    want, tol, nan = expect(p, f64(q), q_pos, lost)
    close(f64(out), np.where(nan, np.nan, want), tol)


def make(form, capacity, seed=0):
    max_queries, n_q, heads = FORMS[form]
    return Pair(batch=1, heads=heads, capacity=capacity, max_queries=max_queries, seed=seed), n_q


def positions(n_q, n, seed=1):
    """From nothing seen to everything."""
    q_pos = np.random.default_rng(seed).integers(0, n, (1, n_q))
    q_pos[0, :4] = -1, n - 1, n // 3, 0
    return q_pos


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_flat_and_peaked_softmax(form, scale):
    p, n_q = make(form, 700)
    p.append(690, pos=torch.randperm(690, generator=p.g).int()[None])
    p.memory()
    q = p.bf(1, n_q, p.H, 128, scale=scale)
    check(p, q)
    check(p, q, positions(n_q, 690))


@pytest.mark.parametrize("form", list(FORMS))
def test_nan_reaches_the_queries_that_see_it_and_no_others(form):
    p, n_q = make(form, 400)
    k, v = p.bf(1, p.Hk, 390, 128), p.bf(1, p.Hk, 390, 128)
    v[0, 0, 100, 40] = float("nan")
    v[0, 0, 270, 127] = float("inf")
    v[0, 0, 388, 0] = float("nan")
    k[0, p.Hk - 1, 330, 3] = float("-inf")
    p.append(390, k, v, pos=torch.arange(390, dtype=torch.int32)[None])
    p.memory()
    q_pos = positions(n_q, 390)
    q_pos[0, :4] = 50, 150, 389, 99
    q = p.bf(1, n_q, p.H, 128)
    check(p, q, q_pos)
    check(p, q, np.full((1, n_q), 99))
    check(p, q)


@pytest.mark.parametrize("form", list(FORMS))
def test_a_table_entry_that_names_no_page_is_skipped(form):
    p, n_q = make(form, 500)
    p.append(490)
    p.memory()
    lost = np.zeros((1, p.Hk, 500), bool)
    p.st.table[0, p.Hk - 1, 2] = -1
    p.st.table[0, 0, 5] = 1 << 30
    lost[0, p.Hk - 1, 128:192] = True
    lost[0, 0, 320:384] = True
    q = p.bf(1, n_q, p.H, 128)
    check(p, q, lost=lost, status=im.IM_STATUS_BAD_PAGE)
    check(p, q, positions(n_q, 490), lost=lost, status=im.IM_STATUS_BAD_PAGE)


@pytest.mark.parametrize("form", list(FORMS))
def test_empty_units_and_units_of_one_entry(form):
    p, n_q = make(form, 200)
    p.append(130)
    p.memory()
    q = p.bf(1, n_q, p.H, 128)
    for n in ([[0, 130], [1, 0], [64, 65]] if p.Hk == 2 else [[0], [1], [64]]):
        p.set_len(torch.tensor([n]))
        check(p, q)
        check(p, q, positions(n_q, 130))


@pytest.mark.parametrize("form", list(FORMS))
def test_entries_beyond_the_promised_length_are_not_looked_at(form):
    p, n_q = make(form, 400)
    p.append(390)
    p.memory()
    im.im_set_max_live(p.h, 150)
    p.ref.len[:] = 150
    q = p.bf(1, n_q, p.H, 128)
    check(p, q, status=im.IM_STATUS_LIVE_EXCEEDED)
    check(p, q, positions(n_q, 390), status=im.IM_STATUS_LIVE_EXCEEDED)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("power", [10, 26, 45, 70, 110, 180])
@pytest.mark.parametrize("large_first", [False, True])
def test_values_of_very_different_size(form, power, large_first):
    """Queries that see the small values alone get them as exactly as if there were no others."""
    p, n_q = make(form, 400)
    v = p.bf(1, p.Hk, 390, 128).float()
    small = torch.arange(390) < 200
    v[:, :, ~small if large_first else small] *= 2.0 ** -min(power, 100)
    if power > 100:
        v[:, :, small if large_first else ~small] *= 2.0 ** (power - 100)
    v[:, :, 30, 32:64] *= 2.0 ** -4
    pos = torch.arange(390, dtype=torch.int32)
    p.append(390, v=v.bfloat16(), pos=(389 - pos if large_first else pos)[None].contiguous())
    q = p.bf(1, n_q, p.H, 128)
    first = 189 if large_first else 199        # (the last position of the small values)
    check(p, q, np.full((1, n_q), first))
    check(p, q, np.linspace(0, 389, n_q).astype(int)[None])
    check(p, q)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("size", [2.0 ** 11, 2.0 ** 13, 2.0 ** 55, -2.0 ** 13, -2.0 ** 55])
def test_logits_far_from_zero(form, size):
    """Logits of 10^7 to 10^34 and of both signs (whole multiples of one number): the largest of them share the weight."""
    p, n_q = make(form, 400)
    k = torch.full((1, p.Hk, 390, 128), size)
    first = torch.arange(390) % 5 == 0
    k[:, :, ~first if size < 0 else first] *= 1.5
    v = p.bf(1, p.Hk, 390, 128)
    p.append(390, k=k.bfloat16(), v=v)
    q = (abs(size) * (1 + torch.arange(n_q) / 128)[None, :, None, None]).expand(1, n_q, p.H, 128).bfloat16()
    for n in (390, 1):
        q_pos = None if n == 390 else np.zeros((1, n_q), int)
        out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
        im.im_attn_packed_with_readout(p.h, p.p, p.st, q.cuda(), out, None if n == 390 else torch.zeros((1, n_q), dtype=torch.int32, device=DEV))
        rows = p.ref.V[0, :, :n][:, first.numpy()[:n]]
        want = np.broadcast_to(rows.mean(1).repeat(p.H // p.Hk, 0)[None, None], q.shape)   # (no memory: the readout is 0)
        close(f64(out), want, 2.0 ** -11 * np.abs(rows).mean() + 2.0 ** -8 * np.abs(want))


# ---- more than one segment of 512 pages in one split -------------------------------------------------------------
def long_cache(n, values, pos, seed=0):
    """One head, and a number of queries (128 rows and more) for which a handle made for one query has records of one split: (layer, queries)."""
    p = Pair(batch=1, heads=(1, 1), capacity=n, n_pages=(n + 63) // 64, seed=seed)
    for i in range(0, n, 1 << 14):
        m = min(1 << 14, n - i)
        p.append(m, v=values[i:i + m].bfloat16()[None, None], pos=torch.as_tensor(pos[i:i + m], dtype=torch.int32)[None])
    return p, (n + 127) // 128 // 2 + 1


@pytest.mark.parametrize("n", [257 * 64, 300 * 64 - 5, 511 * 64 + 1, 513 * 64 - 63, 513 * 64, 700 * 64 + 9, 1031 * 64 + 1])
def test_more_pages_than_a_wave_knows_and_than_a_segment_holds(n):
    g = torch.Generator().manual_seed(n)
    v = torch.randn(n, 128, generator=g)
    order = torch.randperm((n + 63) // 64, generator=g)
    pos = (order.repeat_interleave(64)[:n] * 64 + torch.arange(n) % 64).numpy()   # pages in no order: a mask drops some, in odd numbers
    p, n_q = long_cache(n, v, pos, seed=n)
    p.memory()
    q = p.bf(1, n_q, 1, 128)
    check(p, q)
    check(p, q, positions(n_q, n))
    check(p, q, np.random.default_rng(n).integers(0, 64 * 9, (1, n_q)))


@pytest.mark.parametrize("powers", [(0, -40), (0, -100), (0, -104), (0, -110), (0, -123), (-123, 0), (-60, 40), (40, -123, 0), (90, -30)])
def test_segments_of_very_different_size(powers):
    """A segment after another whose values are far larger or smaller: the sums over the first stay, and queries that see the second
    alone get it exactly."""
    n = 512 * 64 * len(powers) - 64 * 511 - 63    # the last segment has one entry
    at = torch.arange(n) // (512 * 64)
    v = torch.ones(n, 128) * 2.0 ** torch.tensor(powers, dtype=torch.float64)[at].float()[:, None]
    v[:, 32:64] *= 1.5 * (1 - 2 * (torch.arange(n) % 3 == 0).float())[:, None]
    v[:, 64:96] = torch.where(at[:, None] == len(powers) - 1, v[:, 64:96], torch.zeros(1))
    p, n_q = long_cache(n, v, (n - 1 - torch.arange(n)).numpy())
    q = p.bf(1, n_q, 1, 128, scale=1e-2)
    check(p, q)
    check(p, q, np.zeros((1, n_q), int))
    q_pos = np.linspace(0, n - 1, n_q).astype(int)[None]
    q_pos[0, 1] = 1
    check(p, q, q_pos)


def test_bands_within_and_between_segments():
    """Small and large values side by side in the first segment, the large ones alone in the second, the small ones alone in the third."""
    n = 1024 * 64 + 70
    g = torch.Generator().manual_seed(5)
    v = torch.randn(n, 128, generator=g)
    i = torch.arange(n)
    small = ((i < 32768) & (i % 3 == 0)) | (i >= 65536)
    v = torch.where(small[:, None], v * 2.0 ** -90, v)
    v[17, :] *= 2.0 ** 60
    pos = torch.where(small, i, i + n)
    p, n_q = long_cache(n, v, pos.numpy())
    q = p.bf(1, n_q, 1, 128)
    check(p, q)
    check(p, q, np.full((1, n_q), n - 1))
    check(p, q, np.linspace(0, 2 * n, n_q).astype(int)[None])


# ---- an event that finds no pages ---------------------------------------------------------------------------------
def test_an_event_without_pages_for_a_units_copies_leaves_its_memory_alone():
    """Sequences share pages and the pool is full: the unit that cannot be compacted keeps its entries, and its memory has not taken
    them; the other unit's event happens."""
    p = Pair(batch=2, heads=(1, 1), capacity=200, n_pages=4, max_queries=2, n_sink=2)
    p.append(100)                           # two pages each
    p.memory()
    p.fork([0, 0])                          # two shared pages, two free ones
    p.check()
    lay, r, lam, eta = p.gpu, p.ref, float(np.float32(0.9)), 0.5
    p.st.refs[3] = p.ref.refs[3] = 1        # and one of these another user's
    before = f64(p.st.M), f64(p.st.b)
    q = p.bf(2, 2, 1, 128)
    x, pos = q.reshape(2, 2, -1), np.tile(np.arange(98, 100), (2, 1))
    lay.compress(q.cuda(), x.cuda(), torch.tensor(pos, dtype=torch.int32, device=DEV), 60, lam, eta)
    kept, gone = r.topb_select(r.index_score(f64(q), f64(x), pos), 60)
    needs = [len({int(s) // 64 for s in gone[b][0] if s < 60}) for b in range(2)]
    assert needs == [1, 1]                  # (each has holes in its first page alone: the first gets the free page)
    r.memory_update([gone[0], [gone[1][0][:0]]], lam, eta)
    r.compact_kv(kept, gone)
    p.check(status=im.IM_STATUS_OUT_OF_PAGES)
    assert p.ref.len.ravel().tolist() == [60, 100]
    for name, was in zip(("M", "b"), before):
        got, want = f64(getattr(p.st, name)), getattr(r, name)
        assert np.array_equal(got[1], was[1])
        assert np.abs(got[0] - want[0]).max() <= 1e-4 * np.sqrt((want[0] ** 2).mean())
    # with pages, the next event takes them, once
    p.st.refs[3] = p.ref.refs[3] = 0
    r.status = 0
    lay.compress(q.cuda(), x.cuda(), torch.tensor(pos, dtype=torch.int32, device=DEV), 60, lam, eta)
    kept, gone = r.topb_select(r.index_score(f64(q), f64(x), pos), 60)
    r.memory_update(gone, lam, eta)
    r.compact_kv(kept, gone)
    p.check()
    for name in ("M", "b"):
        got, want = f64(getattr(p.st, name)), getattr(r, name)
        assert np.abs(got - want).max() <= 1e-4 * np.sqrt((want ** 2).mean())


# ---- indexer keys -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_new", [3, 20, 70])
def test_an_infinite_projection_weight_makes_nan_of_its_own_column_alone(n_new):
    """The norm is infinite: what is finite becomes 0, as the quotient has it, however many rows a call projects."""
    p = Pair(heads=(4, 2), capacity=100)
    for row, dim, w in ((5, 7, np.inf), (9, 100, -np.inf)):
        p.p.Uk[row, dim] = p.ref.p.Uk[row, dim] = w
    p.append(n_new)
    p.check()
    assert np.isnan(p.ref.Kidx[0, :, :n_new][..., [5, 9]]).all() and (p.ref.Kidx[0, :, :n_new, :5] == 0).all()
