"""The cache held in 4 bits, in pages, against a plain fp64 model: rounding, page tables, attention, compaction, forks, and all of them
together as a serving program runs them."""
import numpy as np
import pytest
import torch

import paper_2605_25475_amd as im
from helpers import f64
from oracle import indexmem_oracle as O
from packed_model import PackedModel, close, quantise

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Pair:
    """A layer on the GPU and its model, over the same inputs."""

    def __init__(self, batch=1, heads=(4, 2), capacity=200, n_pages=None, max_queries=1, seed=0, n_sink=0, first_pages_taken=0):
        H, Hk = heads
        self.B, self.H, self.Hk, self.C = batch, H, Hk, capacity
        self.g = torch.Generator().manual_seed(1000 + seed)
        hi = max(1, H // 4)
        T = (capacity + 63) // 64
        n_pages = n_pages or batch * Hk * T * 2 + first_pages_taken
        w = {k: self.bf(*s, scale=f) for k, s, f in (("Uq", (hi * 64, H * 128), 0.02), ("G", (hi, H * 128), 0.02), ("Uk", (64, 128), 0.1),
                                                      ("Wtheta", (128, 128), 0.1), ("wg", (128,), 0.1))}
        w["nq"], w["nk"] = (torch.ones(64) + self.randn(64) * 0.1).bfloat16(), (torch.ones(64) + self.randn(64) * 0.1).bfloat16()
        self.cfg = im.Config(batch=batch, n_q_heads=H, n_kv_heads=Hk, capacity=capacity, n_idx_heads=hi, n_sink=n_sink, max_queries=max_queries)
        c = {k: v.cuda() for k, v in w.items()}
        self.h = im.Handle(self.cfg, DEV)
        self.p = im.Params(c["Uq"], c["G"], c["Uk"], c["Wtheta"], c["wg"], 0.25, c["nq"], c["nk"])
        self.gpu = im.PackedLayer(self.h, self.p, n_pages)
        self.st = self.gpu.st
        self.st.pages.random_(0, 256)           # what nobody has written to holds anything
        self.st.pos.random_(0, 1 << 30)
        if first_pages_taken:
            self.st.refs[:first_pages_taken] = 1
        cfg = O.OracleConfig(batch=batch, n_q_heads=H, n_kv_heads=Hk, capacity=capacity, n_idx_heads=hi, n_sink=n_sink,
                             rms_eps=float(np.float32(1e-6)), mem_eps=float(np.float32(1e-6)), softmax_scale=float(np.float32(128 ** -0.5)))
        self.ref = PackedModel(cfg, O.OracleParams(*(f64(w[k]) for k in ("Uq", "G", "Uk", "nq", "nk", "Wtheta", "wg")), 0.25), n_pages)
        self.ref.refs[:first_pages_taken] = 1
        self.ref.pos[:] = self.st.pos.cpu().numpy()
        self.next = 0

    def randn(self, *s):
        return torch.randn(s, generator=self.g)

    def bf(self, *s, scale=1.0):
        return (self.randn(*s) * scale).bfloat16()

    def append(self, n_new, k=None, v=None, pos=None):
        k = self.bf(self.B, self.Hk, n_new, 128) if k is None else k
        v = self.bf(self.B, self.Hk, n_new, 128) if v is None else v
        pos = (self.next + torch.arange(n_new, dtype=torch.int32)).repeat(self.B, 1) if pos is None else pos
        self.next += n_new
        self.gpu.append(k.cuda(), v.cuda(), pos.cuda())
        self.ref.append_kv(f64(k), f64(v), pos.numpy())

    def memory(self):
        """A memory state with something in it, the same on both sides."""
        M, b = self.randn(self.B, self.Hk, 128, 128) * 0.3, self.randn(self.B, self.Hk, 128).abs() + 0.5
        self.st.M.copy_(M), self.st.b.copy_(b)
        self.ref.M[:], self.ref.b[:] = f64(M), f64(b)

    def set_len(self, n):
        """The program drops entries behind the n-th of each unit."""
        n = torch.as_tensor(n, dtype=torch.int32).expand(self.B, self.Hk).contiguous()
        self.st.len.copy_(n), self.st.n_projected.copy_(n)
        self.ref.len[:], self.ref.n_projected[:] = n.numpy(), n.numpy()

    def compact(self, keep_n, seed=1):
        """Random keep / evict lists: keep_n [B, Hk] (or a number) of each unit's entries stay."""
        r = np.random.default_rng(seed)
        keep_n = np.broadcast_to(np.asarray(keep_n), (self.B, self.Hk))
        lists = [torch.zeros((self.B, self.Hk, self.C), dtype=torch.int32) for _ in range(2)]
        counts = [torch.zeros((self.B, self.Hk), dtype=torch.int32) for _ in range(2)]
        keep, evict = ([[None] * self.Hk for _ in range(self.B)] for _ in range(2))
        for b in range(self.B):
            for h in range(self.Hk):
                n = int(self.ref.len[b, h])
                order = r.permutation(n)
                parts = np.sort(order[:keep_n[b, h]]), np.sort(order[keep_n[b, h]:])
                keep[b][h], evict[b][h] = parts
                for i in range(2):
                    lists[i][b, h, :len(parts[i])] = torch.from_numpy(parts[i].astype(np.int32))
                    counts[i][b, h] = len(parts[i])
        im.im_compact_packed(self.h, self.st, lists[0].cuda(), counts[0].cuda(), lists[1].cuda(), counts[1].cuda())
        self.ref.compact_kv(keep, evict)

    def fork(self, src_of):
        im.im_fork_packed(self.h, self.st, torch.tensor(src_of, dtype=torch.int32, device=DEV))
        self.ref.fork(list(src_of))

    def check(self, status=0):
        """Every part of the state that the library keeps, exactly."""
        torch.cuda.synchronize()
        st, ref = self.st, self.ref
        assert im.im_query_status(self.h) == status == ref.status
        ref.status = 0
        for name in ("table", "refs", "len", "n_projected", "pos"):
            assert np.array_equal(getattr(st, name).cpu().numpy(), getattr(ref, name)), name
        users = np.bincount(ref.table[ref.table >= 0].ravel(), minlength=ref.refs.size)
        assert (users <= ref.refs).all()
        K, V = (torch.full((self.B, self.Hk, self.C, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        im.im_unpack_kv(self.h, st, K, V)
        for b in range(self.B):
            for h in range(self.Hk):
                n = int(ref.len[b, h])
                assert np.array_equal(f64(K[b, h, :n]), ref.K[b, h, :n], equal_nan=True)
                assert np.array_equal(f64(V[b, h, :n]), ref.V[b, h, :n], equal_nan=True)
                assert bool((K[b, h, n:] == 7).all()) and bool((V[b, h, n:] == 7).all())   # rows behind the last entry: as they were
                assert np.array_equal(f64(st.Kidx[b, h, :n]), ref.Kidx[b, h, :n], equal_nan=True)

    def attend(self, n_q, q_pos=None, q=None, scale=1.0):
        q = self.bf(self.B, n_q, self.H, 128, scale=scale) if q is None else q
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
        res = torch.full(q.shape, float("nan"), device=DEV)
        qp = None if q_pos is None else torch.as_tensor(q_pos, dtype=torch.int32)
        im.im_attn_packed_with_readout(self.h, self.p, self.st, q.cuda(), out, None if qp is None else qp.cuda().contiguous(), res)
        torch.cuda.synchronize()
        want, r, t_out, t_res = self.ref.attend(f64(q), None if qp is None else qp.numpy())
        close(f64(res), r, t_res)
        close(f64(out), want, t_out)
        return out


# ---- rounding and appending ------------------------------------------------------------------------------------
def test_every_bf16_value_is_rounded_to_the_nearest_code():
    # all finite bf16 patterns, 32 neighbours to a block, and again in blocks whose largest value differs
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    finite = bits[torch.isfinite(bits.float())]
    finite = finite[:finite.numel() // 128 * 128].view(-1, 128)
    mixed = finite.clone()
    mixed[:, ::32] = (finite[:, 1::32].float() * 3.7).clamp(-3e38, 3e38).bfloat16()
    rows = torch.cat([finite, mixed])
    p = Pair(heads=(1, 1), capacity=rows.shape[0])
    p.append(rows.shape[0], k=rows.view(1, 1, -1, 128), v=rows.flip(0).view(1, 1, -1, 128).contiguous())
    K, V = (torch.zeros((1, 1, p.C, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    im.im_unpack_kv(p.h, p.st, K, V)
    assert np.array_equal(f64(K)[0, 0], quantise(f64(rows)))
    assert np.array_equal(f64(V)[0, 0], quantise(f64(rows.flip(0))))


def test_blocks_with_infinities_and_nan_read_as_nan_and_their_neighbours_do_not():
    p = Pair(capacity=100)
    k, v = p.bf(1, 2, 70, 128), p.bf(1, 2, 70, 128)
    k[0, 0, 3, 5], k[0, 1, 66, 127], v[0, 0, 64, 32], v[0, 1, 0, 0] = float("inf"), float("nan"), float("-inf"), float("nan")
    p.append(70, k, v)
    # (the indexer keys of rows with infinities or NaN are not compared: RMSNorm of them is the model's business alone)
    for h, r in ((0, 3), (1, 66)):
        p.st.Kidx[0, h, r] = 0
        p.ref.Kidx[0, h, r] = 0
    p.check()


@pytest.mark.parametrize("n_new", [1, 2, 4, 5, 17, 63, 64, 65, 130])
@pytest.mark.parametrize("before", [0, 1, 63, 64, 66])
def test_append(n_new, before):
    p = Pair(batch=2, heads=(6, 3), capacity=before + n_new + 3, seed=n_new)
    if before:
        p.append(before)
    p.append(n_new)
    p.check()


def test_append_of_ragged_units_and_of_units_that_are_full():
    p = Pair(batch=3, heads=(2, 2), capacity=150, seed=5)
    p.append(100)
    p.set_len(torch.tensor([[0, 100], [99, 1], [64, 63]]))
    p.append(51)          # the unit of 100 has no room
    p.check(status=1)
    p.append(3)           # and now that of 99 + 51 has none
    p.check(status=1)


def test_an_append_without_pages_leaves_the_unit_as_it_was():
    p = Pair(batch=2, heads=(2, 2), capacity=300, n_pages=9)
    p.append(60)          # 4 pages
    p.append(100)         # 2 more each: the first two units get theirs
    p.check(status=16)
    p.append(4)           # the first two have room in their pages; the others fill the first page
    p.check()
    p.fork([0, -1])       # three are free
    p.append(64)          # one for each unit: the last gets none
    p.check(status=16)


def test_tokens_that_are_dropped_leave_their_pages_with_the_unit():
    p = Pair(batch=1, heads=(2, 2), capacity=300)
    p.append(130)
    p.set_len(40)
    p.append(30)
    p.check()
    p.append(100)
    p.check()
    p.compact(10)
    p.check()


def test_pages_beyond_four_gigabytes():
    n = (1 << 32) // 8704 + 40
    p = Pair(batch=1, heads=(2, 2), capacity=140, n_pages=n, first_pages_taken=n - 8)
    p.append(130)
    p.memory()
    p.check()
    p.attend(1)
    p.attend(20, np.arange(110, 130)[None])
    p.compact(60)
    p.check()


# ---- reading back ----------------------------------------------------------------------------------------------
def test_unpack_of_listed_slots_writes_those_rows_alone():
    p = Pair(batch=2, heads=(2, 2), capacity=150)
    p.append(140)
    idx = torch.full((2, 2, 150), 99999, dtype=torch.int32)
    n = torch.tensor([[3, 0], [5, 1]], dtype=torch.int32)
    idx[0, 0, :3] = torch.tensor([7, 7, 139])                 # the same one twice
    idx[1, 0, :5] = torch.tensor([139, 140, -1, 64, 149])     # some that hold nothing
    idx[1, 1, :1] = 0
    K, V = (torch.full((2, 2, 150, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    im.im_unpack_kv(p.h, p.st, K, V, idx.cuda(), n.cuda())
    want = np.full((2, 2, 150, 128), 7.0), np.full((2, 2, 150, 128), 7.0)
    for b, h, s in ((0, 0, 7), (0, 0, 139), (1, 0, 139), (1, 0, 64), (1, 1, 0)):
        want[0][b, h, s], want[1][b, h, s] = p.ref.K[b, h, s], p.ref.V[b, h, s]
    assert np.array_equal(f64(K), want[0]) and np.array_equal(f64(V), want[1])
    assert im.im_query_status(p.h) == 0


# ---- attention -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (6, 2), (8, 2), (5, 1), (12, 2), (7, 1), (8, 1)])
@pytest.mark.parametrize("n", [1, 15, 64, 65, 200, 700])
def test_one_query(heads, n):
    p = Pair(batch=2, heads=heads, capacity=n + 2, seed=n)
    p.append(n)
    p.memory()
    p.attend(1)
    p.attend(1, q_pos=[[n // 2], [0]])


@pytest.mark.parametrize("heads,n_q", [((4, 2), 2), ((4, 2), 8), ((4, 2), 9), ((6, 2), 5), ((6, 2), 6), ((2, 2), 16), ((2, 2), 17),
                                       ((8, 1), 40), ((4, 1), 129), ((7, 1), 61), ((4, 2), 64), ((4, 2), 65)])
@pytest.mark.parametrize("n,max_queries", [(1, 1), (70, 128), (333, 1), (1100, 256)])
def test_several_queries(heads, n_q, n, max_queries):
    p = Pair(batch=2, heads=heads, capacity=n + 1, max_queries=max_queries, seed=n + n_q)
    p.append(n, pos=torch.stack([torch.randperm(n, generator=p.g).int() for _ in range(2)]))
    p.set_len(torch.tensor([n, n // 2]).repeat((2, 1))[:, :p.Hk] if p.Hk > 1 else torch.tensor([[n], [n // 2]]))
    p.memory()
    r = np.random.default_rng(n_q)
    p.attend(n_q)                                                        # everything is seen
    p.attend(n_q, q_pos=r.integers(-1, n + 1, (2, n_q)))                 # some see nothing, some all
    p.attend(n_q, q_pos=np.full((2, n_q), -5))                           # nothing is seen: the readout alone
    p.attend(n_q, q_pos=np.full((2, n_q), 2 ** 31 - 1))


def test_a_prompt_chunk_sees_the_entries_before_it_and_itself():
    p = Pair(batch=1, heads=(4, 1), capacity=800, max_queries=300)
    p.append(400, pos=torch.randperm(400, generator=p.g).int()[None])
    p.compact(300)
    p.append(300)
    p.memory()
    p.attend(300, q_pos=400 + np.arange(300)[None])
    p.check()


@pytest.mark.parametrize("n_q", [1, 20, 50])
def test_an_empty_cache_gives_the_readout_alone(n_q):
    p = Pair(batch=2, heads=(4, 2), capacity=70)
    p.append(5)
    p.set_len(torch.tensor([[0, 5], [0, 0]]))
    p.memory()
    p.attend(n_q)
    p.attend(n_q, q_pos=np.full((2, n_q), 3))


@pytest.mark.parametrize("scale", [1e-3, 30.0])
@pytest.mark.parametrize("n_q", [1, 10, 33])
def test_flat_and_peaked_softmax(n_q, scale):
    p = Pair(batch=1, heads=(4, 2), capacity=400)
    p.append(390)
    p.memory()
    p.attend(n_q, scale=scale)


@pytest.mark.parametrize("n_q", [1, 20, 40])
def test_a_long_flat_tail_under_one_large_weight(n_q):
    """2^16 entries whose weights are 2^-16, 2^-22, 2^-25 or less of the largest: together they count, each by itself hardly."""
    p = Pair(batch=1, heads=(2, 1), capacity=1 << 16)
    for i in range(4):
        k, v = (torch.zeros(1, 1, 1 << 14, 128).bfloat16() for _ in range(2))
        v[...] = 1.0
        if i == 1:
            k[0, 0, 777], v[0, 0, 777] = 1.5, 0.0
        p.append(1 << 14, k, v)
    q = torch.ones(1, n_q, 2, 128) * torch.tensor([0.65, 0.9, 1.03, 1.25])[torch.arange(n_q) % 4][None, :, None, None]   # (logits of 11 to 21)
    p.attend(n_q, q=q.bfloat16())


@pytest.mark.parametrize("n_q", [3, 20, 40])
def test_nan_reaches_the_queries_that_see_it_and_no_others(n_q):
    p = Pair(batch=1, heads=(4, 2), capacity=300)
    k, v = p.bf(1, 2, 280, 128), p.bf(1, 2, 280, 128)
    v[0, 0, 100, 40] = float("nan")      # one block of one head's values
    v[0, 0, 270, 127] = float("inf")
    k[0, 1, 200, 3] = float("-inf")      # a key of the other head
    p.append(280, k, v)
    p.memory()
    q_pos = np.sort(np.random.default_rng(1).integers(0, 280, (1, n_q)), axis=1)
    q_pos[0, :3] = 50, 150, 279
    q = p.bf(1, n_q, 4, 128)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    im.im_attn_packed_with_readout(p.h, p.p, p.st, q.cuda(), out, torch.tensor(q_pos, dtype=torch.int32, device=DEV))
    got = f64(out)
    # the model's sums over the rows that are seen; a row of weight > 0 with NaN in a block makes NaN of that block
    want, _, tol, _ = p.ref.attend(f64(q), q_pos)
    nan = np.zeros(q.shape, bool)
    for s in range(n_q):
        nan[0, s, :2, 32:64] = q_pos[0, s] >= 100
        nan[0, s, :2, 96:] = q_pos[0, s] >= 270
        nan[0, s, 2:] = q_pos[0, s] >= 200
    assert np.array_equal(np.isnan(got), nan)
    close(np.where(nan, 0, got), np.where(nan, 0, np.nan_to_num(want)), np.where(nan, 1, np.nan_to_num(tol, nan=1.0) + 2.0 ** -13 * 6))


def test_entries_beyond_the_promised_length_are_not_looked_at():
    p = Pair(batch=1, heads=(4, 2), capacity=300)
    p.append(290)
    p.memory()
    im.im_set_max_live(p.h, 100)
    q = p.bf(1, 1, 4, 128)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    for n_q in (1, 30, 50):
        x = q.expand(1, n_q, 4, 128).contiguous()
        out = torch.zeros(x.shape, dtype=torch.bfloat16, device=DEV)
        im.im_attn_packed_with_readout(p.h, p.p, p.st, x.cuda(), out)
        assert im.im_query_status(p.h) == im.IM_STATUS_LIVE_EXCEEDED
        p.ref.len[:] = 100
        want, _, tol, _ = p.ref.attend(f64(x))
        close(f64(out), want, tol)
    p.ref.len[:] = 290
    keep = torch.arange(300, dtype=torch.int32, device=DEV).repeat(1, 2, 1).contiguous()
    n = torch.full((1, 2), 50, dtype=torch.int32, device=DEV)
    im.im_compact_packed(p.h, p.st, keep, n, keep, n * 5 - 10)
    p.ref.status = im.IM_STATUS_LIVE_EXCEEDED
    im.im_set_max_live(p.h, 300)
    p.check(status=im.IM_STATUS_LIVE_EXCEEDED)


@pytest.mark.parametrize("n_q", [1, 30, 50])
def test_a_table_entry_that_names_no_page_is_skipped(n_q):
    p = Pair(batch=1, heads=(4, 2), capacity=300)
    p.append(290)
    p.memory()
    p.st.table[0, 1, 2] = -1
    p.st.table[0, 0, 1] = 1 << 30
    q = p.bf(1, n_q, 4, 128)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    im.im_attn_packed_with_readout(p.h, p.p, p.st, q.cuda(), out)
    assert im.im_query_status(p.h) == im.IM_STATUS_BAD_PAGE
    p.ref.pos[:] = 0
    p.ref.pos[0, 1, 128:192] = p.ref.pos[0, 0, 64:128] = 9
    want, _, tol, _ = p.ref.attend(f64(q), np.zeros((1, n_q), int))
    close(f64(out), want, tol)


# ---- compaction and forks ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,keep", [(1, 0), (1, 1), (64, 63), (65, 64), (65, 1), (200, 199), (200, 128), (200, 100), (300, 7), (130, 0)])
def test_compact(n, keep):
    p = Pair(batch=2, heads=(2, 2), capacity=n + 5, seed=n)
    p.append(n)
    p.compact(keep, seed=keep)
    p.check()
    if n >= 3:
        p.append(3)
        p.check()


def test_compaction_of_some_units_and_lists_that_do_not_fit():
    p = Pair(batch=2, heads=(2, 2), capacity=200)
    p.append(190)
    p.compact([[190, 20], [65, 189]])
    p.check()
    idx = torch.zeros((2, 2, 200), dtype=torch.int32, device=DEV)
    bad = torch.tensor([[5, -1], [1 << 30, 0]], dtype=torch.int32, device=DEV)
    im.im_compact_packed(p.h, p.st, idx, bad, idx, bad)
    p.ref.status = im.IM_STATUS_BAD_LISTS
    p.check(status=im.IM_STATUS_BAD_LISTS)


def test_forks_share_pages_until_one_of_them_writes():
    p = Pair(batch=4, heads=(4, 2), capacity=250, n_pages=64)
    p.append(150)
    p.memory()
    p.fork([0, 0, -1, 0])
    p.check()
    assert int(p.st.refs.max()) == 3
    p.attend(1)
    p.append(1)                      # the third page is copied by each of the three
    p.check()
    p.append(70)
    p.check()
    p.compact([[200, 150], [221, 100], [71, 20], [1, 221]])
    p.check()
    p.fork([3, 1, 1, 3])             # 0 becomes 3's copy, 2 becomes 1's
    p.check()
    p.compact([[1, 150], [150, 64], [221, 99], [0, 200]])
    p.check()
    p.attend(1)
    p.fork([-1, -1, -1, -1])
    p.check()
    assert int(p.st.refs.sum()) == 0


def test_many_units_and_pages():
    """More (unit, page) pairs than one pass of a plan takes, and than its notes in LDS hold."""
    p = Pair(batch=8, heads=(8, 8), capacity=4480, n_pages=3000)
    p.append(1030)
    p.check()
    p.fork([0, 0, 2, 2, -1, 5, 5, -1])
    p.append(70)
    p.compact(np.random.default_rng(3).integers(0, 71, (8, 8)))
    p.check()
    p.append(5)
    p.check()


def test_many_units_with_too_few_pages_and_lists_that_do_not_fit():
    p = Pair(batch=8, heads=(8, 8), capacity=4480, n_pages=1200)
    p.append(140)
    p.fork([0, 0, 2, 2, 2, -1, 6, 6])       # 64 units of 3 pages, 8 of them empty: 72 pages in use
    p.st.refs[172:] = 1                     # 100 are free, the rest another user's
    p.ref.refs[172:] = 1
    keep = np.random.default_rng(4).integers(70, 100, (8, 8))
    keep[5] = 0
    p.compact(keep)                         # 56 units with holes in two shared pages each: the last ones go without
    p.check(status=16)
    len0 = p.st.len.clone()
    idx = torch.zeros((8, 8, 4480), dtype=torch.int32, device=DEV)
    n_keep, n_evict = len0.clone(), torch.zeros_like(len0)
    n_keep[3, 2], n_evict[3, 2] = -1, 141   # lists that do not fit, some of them with the right sum
    n_keep[4, 1] += 1
    im.im_compact_packed(p.h, p.st, idx, n_keep, idx, n_evict)
    p.ref.status = im.IM_STATUS_BAD_LISTS
    p.check(status=im.IM_STATUS_BAD_LISTS)


def test_two_handles_take_pages_of_one_pool():
    """Two layers' tables over one pool of pages, their calls one after another."""
    a, b = Pair(batch=1, heads=(2, 2), capacity=200, n_pages=12), Pair(batch=1, heads=(2, 2), capacity=200, n_pages=12, seed=1)
    b.st.pages, b.st.refs = a.st.pages, a.st.refs
    b.st.pk = im.binding.ImPacked(a.st.pages.data_ptr(), a.st.refs.data_ptr(), b.st.table.data_ptr(), 12)
    b.ref.refs = a.ref.refs
    for p in (a, b, a, b):
        p.append(60)
        p.check()
    a.compact(10)
    b.append(70)
    b.check()
    a.check()


@pytest.mark.parametrize("n_pages,free", [(37, 37), (37, 9), (1063, 40), (17000, 40)])
def test_counts_that_start_on_any_integer(n_pages, free):
    """Pools of any size, the free pages their last ones, their counts 4 bytes behind a 16-byte boundary."""
    p = Pair(batch=1, heads=(2, 2), capacity=600, n_pages=n_pages)
    p.st.refs = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV)[1:]
    p.st.pk = im.binding.ImPacked(p.st.pages.data_ptr(), p.st.refs.data_ptr(), p.st.table.data_ptr(), n_pages)
    p.st.refs[:n_pages - free] = 1
    p.ref.refs[:n_pages - free] = 1
    p.append(200)
    p.check()
    p.append(63)
    p.append(100)
    p.check(status=16 if free < 12 else 0)
    p.compact(70)
    p.check()


def test_forks_that_are_refused_leave_their_sequences_as_they_were():
    p = Pair(batch=4, heads=(2, 2), capacity=100)
    p.append(90)
    p.fork([1, 0, 7, -2])            # a swap, a sequence there is none of, no sequence
    p.check(status=32)
    p.fork([1, 1, 0, 3])             # 2 wants to be a copy of one that changes
    p.check(status=32)


def test_a_compaction_without_pages_for_its_copies_leaves_the_unit_as_it_was():
    p = Pair(batch=2, heads=(1, 1), capacity=200, n_pages=4)
    p.append(1)
    p.fork([0, -1])
    p.append(100, k=p.bf(2, 1, 100, 128))   # two pages each, the pool is full
    p.fork([0, 0])                          # two are free
    p.compact([[60], [80]])                 # the first has holes in one shared page, the second in two: there are two
    p.check(status=16)
    p.compact([[59], [100]])
    p.check()


# ---- together ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads", [(8, 2), (7, 1)])
def test_a_prompt_in_chunks_then_decoding_with_candidates(heads):
    """Chunks of a prompt enter, attend and are cut back to the budget; the second sequence ends and becomes a copy of the first; both
    decode, one entry leaving per token; the evicted rows go to the memory.  Every decision, every state and every output."""
    p = Pair(batch=2, heads=heads, capacity=260, max_queries=90, n_sink=4, seed=3)
    lam, eta, budget, r = float(np.float32(0.99)), 0.5, 150, p.ref
    lay = p.gpu

    def event(n_new, keep):
        q = p.bf(2, n_new, p.H, 128)
        pos = np.tile(p.next - n_new + np.arange(n_new), (2, 1))
        x = q.reshape(2, n_new, -1)
        qp = torch.tensor(pos, dtype=torch.int32, device=DEV)
        lay.compress(q.cuda(), x.cuda(), qp, keep, lam, eta)
        scores = r.index_score(f64(q), f64(x), pos)
        kept, gone = r.topb_select(scores, keep)
        for u in r.units():
            assert np.array_equal(lay.evict_idx[u][:len(gone[u[0]][u[1]])].cpu().numpy(), gone[u[0]][u[1]])
        r.memory_update(gone, lam, eta)
        r.compact_kv(kept, gone)
        p.check()
        for name in ("M", "b"):   # (fp32 sums over parts of 16 bits: the library's bar for its memory state)
            got, want = f64(getattr(p.st, name)), getattr(r, name)
            assert np.abs(got - want).max() <= 1e-4 * np.sqrt((want ** 2).mean())

    for n_new in (90, 90, 61):
        p.append(n_new)
        p.attend(n_new, q_pos=np.tile(p.next - n_new + np.arange(n_new), (2, 1)))
        event(n_new, budget)
    p.fork([0, 0])
    p.check()
    for step in range(3):
        p.append(1)
        event(1, budget)
        p.attend(1)
    p.fork([0, -1])
    p.check()


def test_a_captured_step_is_replayed():
    """A decode step with forks in it, captured once and replayed between eager work, against the same calls made eagerly."""
    def make():
        p = Pair(batch=2, heads=(4, 2), capacity=300, max_queries=1, n_sink=2, seed=9)
        p.append(200)
        p.memory()
        return p

    a, e = make(), make()
    e.st.pages.copy_(a.st.pages), e.st.pos.copy_(a.st.pos)
    g = torch.Generator(device=DEV).manual_seed(4)
    k, v = (torch.randn((2, 2, 1, 128), generator=g, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn((2, 1, 4, 128), generator=g, device=DEV).bfloat16()
    pos = torch.full((2, 1), 200, dtype=torch.int32, device=DEV)
    src = torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    outs = [torch.zeros((2, 1, 4, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    wide = torch.randn((2, 24, 4, 128), generator=g, device=DEV).bfloat16()
    wpos = torch.randint(0, 200, (2, 24), generator=g, device=DEV, dtype=torch.int32)
    wides = [torch.zeros_like(wide) for _ in range(2)]

    def step(p, out, wout):
        p.gpu.fork(src)
        p.gpu.step(k, v, pos, q, q.view(2, 1, -1), pos, q, out, 180, 0.99, 0.5)
        p.gpu.attend(wide, wout, wpos)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # (once eagerly, on both)
        step(a, outs[0], wides[0])
    torch.cuda.current_stream().wait_stream(side)
    step(e, outs[1], wides[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, outs[0], wides[0])
    for i in range(4):
        k.normal_(generator=g), q.normal_(generator=g), pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        step(e, outs[1], wides[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(wides[0], wides[1]), i
        for name in ("table", "refs", "len", "pos", "Kidx", "M", "b"):
            assert torch.equal(getattr(a.st, name), getattr(e.st, name)), (i, name)
    assert im.im_query_status(a.h) == 0


def test_calls_give_the_same_bits_each_time_on_any_stream():
    p = Pair(batch=2, heads=(4, 2), capacity=900, max_queries=64)
    p.append(880)
    p.memory()
    q = p.bf(2, 64, 4, 128).cuda()
    qp = torch.randint(0, 880, (2, 64), dtype=torch.int32, device=DEV)
    side, want = torch.cuda.Stream(), {}
    for i in range(3):
        with torch.cuda.stream(side if i == 1 else torch.cuda.current_stream()):
            side.wait_stream(torch.cuda.default_stream())
            for n_q in (1, 3, 64):
                out = torch.zeros((2, n_q, 4, 128), dtype=torch.bfloat16, device=DEV)
                im.im_attn_packed_with_readout(p.h, p.p, p.st, q[:, :n_q].contiguous(), out, qp[:, :n_q].contiguous())
                torch.cuda.synchronize()
                assert torch.equal(out, want.setdefault(n_q, out))


@pytest.mark.parametrize("spread", [2.0 ** 10, 2.0 ** 26, 2.0 ** 60])
@pytest.mark.parametrize("n_q", [1, 20, 40])
def test_values_of_very_different_size(n_q, spread):
    """Queries that see the small values alone get them as exactly as if there were no others."""
    p = Pair(batch=1, heads=(4, 2), capacity=300)
    v = p.bf(1, 2, 280, 128)
    small = torch.arange(280) < 140
    v[:, :, small] = (v[:, :, small].float() / spread).bfloat16()
    v[:, :, 30, 32:64] *= 2.0 ** -40           # smaller still, in one block
    p.append(280, v=v)
    p.attend(n_q, q_pos=np.full((1, n_q), 139))
    p.attend(n_q, q_pos=np.full((1, n_q), 279))
    p.attend(n_q, q_pos=np.linspace(0, 279, n_q).astype(int)[None])
    p.memory()
    p.attend(n_q, q_pos=np.linspace(100, 279, n_q).astype(int)[None])
