"""The operators on a cache whose keys and values are held in 4 bits, in pages: appending, reading back, attention with the
memory readout, compaction after an eviction, and forking sequences.

A case is a plain dict.  Fields:
  op       "append"   `n_new` tokens per sequence enter the cache
           "unpack"   the listed entries are read back as bf16 rows (what im_memory_update takes)
           "attend"   `n_q` queries per sequence attend over the cache and read the memory
           "compact"  the second half of the sequences become forks of the first, and are cut back to `keep` entries
           "fork"     of three neighbouring sequences one stays, one becomes a copy of it, one is emptied
  batch, n_q_heads, n_kv_heads   the layer's shape (head_dim 128, n_q_heads / 4 indexer heads)
  cached   entries per (sequence, KV head) before the call, besides the queries' own tokens
  ragged   the units hold between half of `cached` and all of it
  forked   (append) the second half of the sequences become forks of the first in the same pass, so that the last page,
           which both would write, is copied
  n_listed (unpack) listed entries per unit

A page is 64 slots of one (sequence, KV head) unit.  A row of 128 values is 128 codes of 4 bits (sign, and 0, 0.5, 1, 1.5, 2, 3, 4,
6) and a power of two per 32 of them, the smallest with which none is above 6.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
D, SLOTS, PAGE = 128, 64, 8704
EPS = 1e-6
DEFAULTS = dict(op="attend", batch=1, n_q_heads=32, n_kv_heads=8, cached=256, n_new=0, n_q=0, keep=0, n_listed=0, ragged=False,
                forked=False)
MOST_ENTRIES = 1 << 20          # batch x KV heads x cached of the largest listed cache
MOST_LOGITS = 4096 * 8192 * 32  # batch x query heads x queries x entries of the largest listed attention


def _case(name=None, **kw):
    c = dict(DEFAULTS, **kw)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a decode token of a small batch enters the cache: what a single small call costs
        _case("append-1-b4-2048", op="append", batch=4, cached=2048, n_new=1, ragged=True),
        # a chunk of a long prompt enters the running cache
        _case("append-4096-b1-4096", op="append", cached=4096, n_new=4096),
        # a prompt's evicted entries on their way to the latent memory, at the 16K-context shape
        _case("unpack-14336-b4-16384", op="unpack", batch=4, cached=16384, n_listed=14336),
        # the same for short prompts of odd length, 7 query heads per KV head
        _case("unpack-1167-b2-1500", op="unpack", batch=2, n_q_heads=28, n_kv_heads=4, cached=1500, n_listed=1167),
        # one decode token of one sequence over a small budget
        _case("attend-1-b1-257", cached=256, n_q=1),
        # a decode token of many sequences, ragged, 7 query heads per KV head
        _case("attend-1-b16-2048-g7", batch=16, n_q_heads=28, n_kv_heads=4, cached=2048, n_q=1, ragged=True),
        # a decode token over an uncompressed long context
        _case("attend-1-b1-131072", cached=131071, n_q=1),
        # a chunk of a long prompt attends to the retained entries and to itself
        _case("attend-4096-b1-8192", cached=4096, n_q=4096),
        # decoding candidates of the same prompt: each forks, and one entry leaves
        _case("compact-1-b4-2048", op="compact", batch=4, cached=2049, keep=2048),
        # an eviction event of the chunked prompt in forked sequences
        _case("compact-4096-b2-8192", op="compact", batch=2, cached=8192, keep=4096),
        # a small batch between two requests
        _case("fork-b3-512", op="fork", batch=3, cached=512),
        # many sequences of a large budget
        _case("fork-b15-8192", op="fork", batch=15, n_q_heads=28, n_kv_heads=4, cached=8192),
    ]


HEADS = [(32, 8), (28, 4), (24, 8), (40, 8), (16, 4), (64, 8), (8, 8), (6, 2)]


def _log(rng, lo, hi):
    """A whole number, uniform in its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "append", "unpack", "attend", "attend", "attend", "compact", "fork"])
    hq, hk = rng.choice(HEADS)
    c = _case(op=op, n_q_heads=hq, n_kv_heads=hk, ragged=rng.random() < 0.5)
    if op == "append":
        c["batch"] = _log(rng, 1, 16)
        c["forked"] = c["batch"] % 2 == 0 and rng.random() < 0.5
        most = min(8192, MOST_ENTRIES // (8 * c["batch"] * hk))
        c["cached"], c["n_new"] = _log(rng, 1, most), rng.choice([1, 1, rng.randint(2, 40), _log(rng, 1, most)])
    elif op == "unpack":
        c["batch"] = _log(rng, 1, 8)
        c["cached"] = _log(rng, 64, min(16384, MOST_ENTRIES // (2 * c["batch"] * hk)))
        c["n_listed"] = rng.choice([1, rng.randint(1, max(1, c["cached"] // 2)), max(1, c["cached"] // 2)])
    elif op == "attend":
        c["n_q"] = rng.choice([1, 1, rng.randint(2, 16), _log(rng, 17, 4096)])
        c["batch"] = _log(rng, 1, 16 if c["n_q"] < 64 else 4)
        c["n_q"] = min(c["n_q"], math.isqrt(MOST_LOGITS // (c["batch"] * hq)) - 1)
        most = min(131071, MOST_ENTRIES // (c["batch"] * hk), MOST_LOGITS // (c["batch"] * hq * c["n_q"]) - c["n_q"])
        c["cached"] = _log(rng, 1, most)
    elif op == "compact":
        c["batch"] = rng.choice([2, 2, 4, 8])
        c["cached"] = _log(rng, 16, min(8192, MOST_ENTRIES // (8 * c["batch"] * hk)))
        c["ragged"] = False
        c["keep"] = rng.choice([c["cached"] - 1, rng.randint(1, c["cached"]), max(1, c["cached"] // 8)])
    else:
        c["batch"] = _log(rng, 2, 24)
        c["cached"] = _log(rng, 1, min(8192, MOST_ENTRIES // (2 * c["batch"] * hk)))
    return c


# ---- the page format, by elementary operations ----------------------------------------------------------------
def _row_map():
    """[64][136]: where the bytes of a slot's row lie in its page: K's 64, V's 64, K's 4 scales, V's 4."""
    r = torch.arange(SLOTS, device=DEV).view(-1, 1)
    j, blk = torch.arange(64, device=DEV).view(1, -1), torch.arange(4, device=DEV).view(1, -1)
    tile, four, i = r // 16, r % 16 // 4, r % 4
    return torch.cat([r * 64 + j, 4096 + tile * 1024 + (four * 16 + j // 4) * 16 + i * 4 + j % 4, 8192 + r * 4 + blk,
                      8448 + tile * 64 + four * 16 + blk * 4 + i], 1)


def _pack(x):
    """float rows [..., 128] -> (bytes [..., 64], scale bytes [..., 4])."""
    x = x.float().unflatten(-1, (4, 32))
    a = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a)                                          # a = m 2^e, 0.5 <= m < 1: above 0.75 it is over 6 * 2^(e - 3)
    k = torch.where(a > 0, e - 3 + (m > 0.75).int(), torch.full_like(e, -126)).clamp(min=-126)
    y = torch.ldexp(x.abs(), -k)
    code = ((y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int() + (y > 2.5).int() + (y >= 3.5).int()
            + (y > 5).int() + 8 * (x < 0).int()).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (k.squeeze(-1) + 127).to(torch.uint8)


def _unpack(code, scale):
    """The values of _pack's bytes, float32."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=code.device)
    c = torch.stack([code & 15, code >> 4], -1).flatten(-2).long()
    v = table[c & 7] * (1 - 2 * (c >> 3)).float()
    return torch.ldexp(v.unflatten(-1, (4, 32)), (scale.int() - 127).unsqueeze(-1)).flatten(-2)


def _rows_at(s, unit, slot):
    """Addresses [..., 136] in the pool of the bytes of (unit, slot)."""
    page = s["table"].view(-1, s["table"].shape[-1])[unit, slot // SLOTS].long()
    return page.unsqueeze(-1) * PAGE + _row_map()[slot % SLOTS]


def _store(s, unit, slot, K, V):
    (kc, ks), (vc, vs) = _pack(K), _pack(V)
    s["pages"].view(-1)[_rows_at(s, unit, slot)] = torch.cat([kc, vc, ks, vs], -1)


def _load(s, unit, slot):
    by = s["pages"].view(-1)[_rows_at(s, unit, slot)]
    return _unpack(by[..., :64], by[..., 128:132]), _unpack(by[..., 64:128], by[..., 132:])


def _take_pages(s, need):
    """Pages for the entries of need [units, T], the lowest free ids in order."""
    free = (s["refs"] == 0).nonzero().view(-1)
    table = s["table"].view(need.shape)
    ids = free[:int(need.sum())].int()
    table[need] = ids
    s["refs"][ids.long()] = 1


# ---- inputs ------------------------------------------------------------------------------------------------
def _sizes(c):
    units = c["batch"] * c["n_kv_heads"]
    C = c["cached"] + c["n_new"] + c["n_q"]
    return units, C, (C + SLOTS - 1) // SLOTS


def prepare(case, seed):
    c = case
    B, H, Hk, cached = c["batch"], c["n_q_heads"], c["n_kv_heads"], c["cached"]
    units, C, T = _sizes(c)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = {"case": c, "C": C}
    held = torch.full((units,), cached, device=DEV, dtype=torch.int32)
    if c["ragged"]:
        held = torch.randint(cached // 2, cached + 1, (units,), generator=g, device=DEV, dtype=torch.int32)
    length = held + c["n_q"]
    # an eviction leaves entries in no order of position; the queries' own tokens come last
    order = torch.rand((units, cached), generator=g, device=DEV).argsort(-1).int()
    s["pos"] = torch.randint(0, 1 << 30, (B, Hk, C), generator=g, device=DEV, dtype=torch.int32)   # (behind the entries: anything)
    pos = s["pos"].view(units, C)
    slots = torch.arange(C, device=DEV)
    if cached:
        pos[:, :cached] = torch.where(slots[:cached] < held.view(-1, 1), order, pos[:, :cached])
    if c["n_q"]:
        mine = (held.view(-1, 1) + torch.arange(c["n_q"], device=DEV)).long()
        pos.scatter_(1, mine, (cached + torch.arange(c["n_q"], device=DEV, dtype=torch.int32)).expand(units, -1))
    s["len"] = length.view(B, Hk).contiguous()
    s["n_projected"] = s["len"].clone()
    s["Kidx"] = rand(B, Hk, C, 64).to(torch.bfloat16)
    s["M"], s["b"] = rand(B, Hk, 128, D) * 0.3, rand(B, Hk, 128).abs() + 0.5
    # pages in no order, between free ones
    has = torch.arange(T, device=DEV) * SLOTS < length.view(-1, 1)
    n_used = int(has.sum())
    n_pages = units * (T + 2 * ((c["n_new"] + SLOTS - 1) // SLOTS) + 3 + (T if c["op"] == "compact" else 0))
    where = torch.rand(n_pages, generator=g, device=DEV).argsort()[:n_used].int()
    s["table"] = torch.full((units, T), -1, device=DEV, dtype=torch.int32)
    s["table"][has] = where
    s["table"] = s["table"].view(B, Hk, T)
    s["refs"] = torch.zeros(n_pages, device=DEV, dtype=torch.int32)
    s["refs"][where.long()] = 1
    s["pages"] = torch.randint(0, 256, (n_pages, PAGE), generator=g, device=DEV, dtype=torch.uint8)
    unit, slot = (slots < length.view(-1, 1)).nonzero(as_tuple=True)
    _store(s, unit, slot, rand(len(unit), D).to(torch.bfloat16), rand(len(unit), D).to(torch.bfloat16))
    w = {"Uq": rand(H // 4 * 64 if H >= 4 else 64, H * D), "G": rand(max(1, H // 4), H * D), "Uk": rand(64, D), "Wtheta": rand(128, D), "wg": rand(D)}
    w = {k: (v * 0.02 if k in ("Uq", "G") else v * 0.1).to(torch.bfloat16) for k, v in w.items()}
    w["norm_k_w"] = (1 + 0.1 * rand(64)).to(torch.bfloat16)
    s["w"], s["cg"] = w, 0.25
    if c["op"] == "append":
        s["k_new"], s["v_new"] = rand(B, Hk, c["n_new"], D).to(torch.bfloat16), rand(B, Hk, c["n_new"], D).to(torch.bfloat16)
        s["pos_new"] = (cached + torch.arange(c["n_new"], device=DEV, dtype=torch.int32)).repeat(B, 1).contiguous()
        s["len_before"] = s["len"].clone()
    if c["op"] in ("append", "compact"):
        b = torch.arange(B, device=DEV, dtype=torch.int32)
        s["src_of"] = torch.where(b < B // 2, b, b - B // 2) if c["forked"] or c["op"] == "compact" else b
    if c["op"] == "append":
        begin = s["len"][s["src_of"].long()].unsqueeze(-1)
        s["idx"] = (begin + torch.arange(C, device=DEV, dtype=torch.int32)).clamp(max=C - 1).contiguous()
        s["n_idx"] = torch.full((B, Hk), c["n_new"], device=DEV, dtype=torch.int32)
    if c["op"] == "fork":
        b = torch.arange(B, device=DEV, dtype=torch.int32)
        s["src_of"] = torch.where(b % 3 == 0, b, torch.where(b % 3 == 1, b - 1, torch.full_like(b, -1)))
    if c["op"] == "unpack":
        # which entries leave: the lowest of random scores, their slots ascending
        score = torch.rand((units, C), generator=g, device=DEV).masked_fill(slots >= length.view(-1, 1), 2.0)
        s["idx"] = torch.zeros((units, C), device=DEV, dtype=torch.int32)
        s["idx"][:, :c["n_listed"]] = score.argsort(-1)[:, :c["n_listed"]].sort(-1).values.int()
        s["idx"] = s["idx"].view(B, Hk, C)
        s["n_idx"] = torch.full((B, Hk), c["n_listed"], device=DEV, dtype=torch.int32)
    if c["op"] == "compact":
        n_out = cached - c["keep"]
        score = torch.rand((units, C), generator=g, device=DEV).argsort(-1)
        keep, out = score[:, n_out:].sort(-1).values.int(), score[:, :n_out].sort(-1).values.int()
        forked = (torch.arange(units, device=DEV) >= units // 2)
        s["keep_idx"] = torch.arange(C, device=DEV, dtype=torch.int32).repeat(units, 1)
        s["keep_idx"][forked, :c["keep"]] = keep[forked]
        s["evict_idx"] = torch.zeros((units, C), device=DEV, dtype=torch.int32)
        s["evict_idx"][forked, :n_out] = out[forked]
        s["n_keep"] = torch.where(forked, c["keep"], cached).int().view(B, Hk)
        s["n_evict"] = torch.where(forked, n_out, 0).int().view(B, Hk)
        s["keep_idx"], s["evict_idx"] = s["keep_idx"].view(B, Hk, C), s["evict_idx"].view(B, Hk, C)
        s["idx"] = torch.arange(C, device=DEV, dtype=torch.int32).repeat(B, Hk, 1).contiguous()
        s["n_idx"] = torch.where(forked, c["keep"], 0).int().view(B, Hk)
    if c["op"] in ("append", "unpack", "compact"):
        s["K"], s["V"] = (torch.zeros((B, Hk, C, D), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    if c["op"] == "attend":
        s["q"] = rand(B, c["n_q"], H, D).to(torch.bfloat16)
        s["q_pos"] = None if c["n_q"] == 1 else (cached + torch.arange(c["n_q"], device=DEV, dtype=torch.int32)).repeat(B, 1).contiguous()
        s["out"] = torch.empty((B, c["n_q"], H, D), device=DEV, dtype=torch.bfloat16)
    if own:
        _hand_over(s)
    return s


def _hand_over(s):
    """The handle, weights and state objects that a user of the library keeps."""
    import paper_2605_25475_amd as im
    c, w = s["case"], s["w"]
    cfg = im.Config(batch=c["batch"], n_q_heads=c["n_q_heads"], n_kv_heads=c["n_kv_heads"], capacity=s["C"],
                    n_idx_heads=max(1, c["n_q_heads"] // 4), n_sink=0, max_queries=max(1, c["n_q"]))
    s["h"] = im.Handle(cfg, DEV)
    s["p"] = im.Params(w["Uq"], w["G"], w["Uk"], w["Wtheta"], w["wg"], s["cg"], None, w["norm_k_w"])
    s["st"] = im.PackedState(cfg, s["refs"].numel(), DEV)
    for name in ("Kidx", "pos", "len", "n_projected", "M", "b", "pages", "refs", "table"):
        mine = getattr(s["st"], name)
        mine.copy_(s[name])
        s[name] = mine


# ---- one pass ------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if op == "append":
        return _append(state)
    if op == "unpack":
        return _read_back(state)
    if op == "attend":
        return _attend(state)
    if op == "compact":
        return _compact(state)
    return _fork(state)


def _state_of(s, *names):
    return {name: s[name] for name in names}


def _append(s):
    # a program that drops rejected draft tokens sets the lengths back itself; so every pass appends at the same place
    s["len"].copy_(s["len_before"])
    s["n_projected"].copy_(s["len_before"])
    if s["case"]["forked"]:
        _fork(s)
    if own:
        import paper_2605_25475_amd as im
        im.im_append_packed(s["h"], s["p"], s["st"], s["k_new"], s["v_new"], s["pos_new"])
    else:
        n_new, table = s["case"]["n_new"], s["table"]
        units, C, T = _sizes(s["case"])
        n, t = s["len"].view(-1, 1), torch.arange(T, device=DEV)
        here = (t >= n // SLOTS) & (t <= (n + n_new - 1) // SLOTS)
        old = table.view(units, T).clone()
        shared = (old >= 0) & (s["refs"][old.clamp(min=0).long()] > 1)
        need = here & ((old < 0) | shared)
        copy = here & shared & (t == n // SLOTS)
        # the entries of a shared page that is written
        slot = torch.arange(C, device=DEV)
        unit_c, slot_c = ((slot < n) & copy.repeat_interleave(SLOTS, 1)[:, :C]).nonzero(as_tuple=True)
        rows = s["pages"].view(-1)[_rows_at(s, unit_c, slot_c)]
        _take_pages(s, need)
        s["refs"].index_add_(0, old[here & shared].long(), torch.full_like(old[here & shared], -1))
        s["pages"].view(-1)[_rows_at(s, unit_c, slot_c)] = rows
        at = (n + torch.arange(n_new, device=DEV)).long()
        unit = torch.arange(units, device=DEV).view(-1, 1).expand_as(at)
        k = s["k_new"].view(units, n_new, D)
        _store(s, unit, at, k, s["v_new"].view(units, n_new, D))
        u = k.float() @ s["w"]["Uk"].float().t()
        key = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS) * s["w"]["norm_k_w"].float()
        s["Kidx"].view(units, C, 64)[unit, at] = key.to(torch.bfloat16)
        s["pos"].view(units, C)[unit, at] = s["pos_new"].repeat_interleave(s["case"]["n_kv_heads"], 0)
        s["len"] += n_new
        s["n_projected"].copy_(s["len"])
    return {**_read_back(s), **_state_of(s, "Kidx", "pos", "len", "n_projected", "table", "refs")}


def _read_back(s):
    if own:
        import paper_2605_25475_amd as im
        im.im_unpack_kv(s["h"], s["st"], s["K"], s["V"], s["idx"], s["n_idx"])
    else:
        units, C, _ = _sizes(s["case"])
        unit, i = (torch.arange(C, device=DEV) < s["n_idx"].view(-1, 1)).nonzero(as_tuple=True)
        slot = s["idx"].view(units, C)[unit, i].long()
        k, v = _load(s, unit, slot)
        s["K"].view(units, C, D)[unit, slot] = k.to(torch.bfloat16)
        s["V"].view(units, C, D)[unit, slot] = v.to(torch.bfloat16)
    return _state_of(s, "K", "V")


def _attend(s):
    if own:
        import paper_2605_25475_amd as im
        im.im_attn_packed_with_readout(s["h"], s["p"], s["st"], s["q"], s["out"], s["q_pos"])
        return {"out": s["out"]}
    c, w = s["case"], {k: v.float() for k, v in s["w"].items()}
    B, H, Hk, n_q = c["batch"], c["n_q_heads"], c["n_kv_heads"], c["n_q"]
    units, C, T = _sizes(c)
    slot = torch.arange(C, device=DEV)
    live = slot < s["len"].view(units, 1)
    at = torch.where(live, slot, 0)                                 # (slot 0 always has an entry)
    k, v = _load(s, torch.arange(units, device=DEV).view(-1, 1), at)
    v = v * live.unsqueeze(-1)
    q = s["q"].float().view(B, n_q, Hk, H // Hk, D).transpose(1, 2).reshape(units, n_q * (H // Hk), D)
    seen = live.unsqueeze(1)
    if s["q_pos"] is not None:
        q_pos = s["q_pos"].repeat_interleave(Hk, 0).repeat_interleave(H // Hk, 1).unsqueeze(-1)
        seen = seen & (s["pos"].view(units, 1, C) <= q_pos)
    l = torch.matmul(q * D ** -0.5, k.transpose(1, 2).contiguous()).masked_fill_(~seen, -math.inf)
    l = l.sub_(l.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = l.sum(-1, keepdim=True)
    o = torch.matmul(l, v) / torch.where(total > 0, total, 1.0)
    phi = q @ w["Wtheta"].t()
    den = (phi.square() * s["b"].view(units, 1, 128)).sum(-1, keepdim=True) + EPS
    gate = torch.sigmoid((q * w["wg"]).sum(-1, keepdim=True) + s["cg"])
    o = o + gate * (torch.matmul(phi, s["M"].view(units, 128, D)) / den)
    s["out"].copy_(o.view(B, Hk, n_q, H // Hk, D).transpose(1, 2).reshape(B, n_q, H, D))
    return {"out": s["out"]}


def _compact(s):
    _fork(s)
    if own:
        import paper_2605_25475_amd as im
        im.im_compact_packed(s["h"], s["st"], s["keep_idx"], s["n_keep"], s["evict_idx"], s["n_evict"])
    else:
        units, C, T = _sizes(s["case"])
        n_keep, n_evict = s["n_keep"].view(units, 1), s["n_evict"].view(units, 1)
        i = torch.arange(C, device=DEV)
        keep, evict = s["keep_idx"].view(units, C), s["evict_idx"].view(units, C)
        stay = ((keep < n_keep) & (i < n_keep)).sum(-1, keepdim=True)          # kept entries that need not move
        unit, j = (i < n_keep - stay).nonzero(as_tuple=True)
        src, dst = keep[unit, j + stay[unit, 0]].long(), evict[unit, j].long()
        rows = s["pages"].view(-1)[_rows_at(s, unit, src)]
        key, pos = s["Kidx"].view(units, C, 64)[unit, src], s["pos"].view(units, C)[unit, src]
        # a shared page that entries move into is copied, without them
        old = s["table"].view(units, T).clone()
        shared = (old >= 0) & (s["refs"][old.clamp(min=0).long()] > 1)
        filled = torch.zeros((units, T * SLOTS), dtype=torch.bool, device=DEV)
        filled[unit, dst] = True
        copy = shared & filled.view(units, T, SLOTS).any(-1)
        held = copy.repeat_interleave(SLOTS, 1)[:, :C] & (i < n_keep) & ~filled[:, :C]
        unit_c, slot_c = held.nonzero(as_tuple=True)
        same = s["pages"].view(-1)[_rows_at(s, unit_c, slot_c)]
        _take_pages(s, copy)
        s["pages"].view(-1)[_rows_at(s, unit_c, slot_c)] = same
        s["pages"].view(-1)[_rows_at(s, unit, dst)] = rows
        s["Kidx"].view(units, C, 64)[unit, dst], s["pos"].view(units, C)[unit, dst] = key, pos
        # what lies behind the kept entries is given up
        gone = (torch.arange(T, device=DEV) * SLOTS >= n_keep) & (old >= 0)
        s["refs"].index_add_(0, old[copy | gone].long(), torch.full_like(old[copy | gone], -1))
        s["table"].view(units, T)[gone] = -1
        s["len"].copy_(s["n_keep"])
        s["n_projected"].copy_(s["n_keep"])
    return {**_read_back(s), **_state_of(s, "Kidx", "pos", "len", "n_projected", "table", "refs")}


def _fork(s):
    if own:
        import paper_2605_25475_amd as im
        im.im_fork_packed(s["h"], s["st"], s["src_of"])
    else:
        B, Hk = s["case"]["batch"], s["case"]["n_kv_heads"]
        C, of = s["C"], s["src_of"].long()
        mine = torch.arange(B, device=DEV)
        copied, emptied = (of >= 0) & (of != mine), of < 0
        changed, src = copied | emptied, of[copied]
        given = s["table"][changed].flatten()
        given = given[given >= 0].long()
        s["refs"].index_add_(0, given, torch.full_like(given, -1, dtype=torch.int32))
        taken = s["table"][src].flatten()
        taken = taken[taken >= 0].long()
        s["refs"].index_add_(0, taken, torch.full_like(taken, 1, dtype=torch.int32))
        s["table"][copied] = s["table"][src]
        live = torch.arange(C, device=DEV) < s["len"][src].unsqueeze(-1)
        s["Kidx"][copied] = torch.where(live.unsqueeze(-1), s["Kidx"][src], s["Kidx"][copied])
        s["pos"][copied] = torch.where(live, s["pos"][src], s["pos"][copied])
        s["table"][emptied] = -1
        for name in ("len", "n_projected", "M", "b"):
            s[name][copied] = s[name][src]
            s[name][emptied] = 0
    return _state_of(s, "table", "refs", "len", "n_projected", "pos", "Kidx", "M", "b")


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    c = case
    units, C, T = _sizes(c)
    held = c["cached"] * (0.75 if c["ragged"] else 1.0)
    row, wide, dense = 136, 512, 132                     # a packed row, a bf16 row, its indexer key and position
    memory = 4 * (128 * D + 128)
    if c["op"] == "append":
        n = units * c["n_new"]
        fork = units / 2 * (2 * (held * dense + memory) + 8 * T) if c["forked"] else 0
        return {"bytes": n * (wide + row + dense) + n * (row + 4 + wide) + fork, "flops": 2 * n * 64 * D}
    if c["op"] == "unpack":
        n = units * c["n_listed"]
        return {"bytes": n * (4 + row + wide), "flops": n * 256}
    if c["op"] == "attend":
        # every query sees all cached entries, and its own tokens up to itself
        pairs = c["n_q"] * held + c["n_q"] * (c["n_q"] + 1) / 2
        rows = c["batch"] * c["n_q_heads"] * c["n_q"]
        return {"bytes": units * ((held + c["n_q"]) * (row + (4 if c["n_q"] > 1 else 0)) + memory) + 4 * rows * D,
                "flops": 4 * D * c["batch"] * c["n_q_heads"] * pairs + 4 * rows * 128 * D}
    if c["op"] == "compact":
        n_out = c["cached"] - c["keep"]
        moved = n_out * c["keep"] / c["cached"]
        one = 2 * (c["cached"] * dense + memory) + 8 * T + moved * 2 * (row + dense) + 4 * c["cached"] + c["keep"] * (4 + row + wide)
        return {"bytes": units / 2 * one, "flops": units / 2 * c["keep"] * 256}
    copied = (c["batch"] + 1) // 3 * c["n_kv_heads"]
    emptied = c["batch"] // 3 * c["n_kv_heads"]
    return {"bytes": copied * (2 * (held * dense + memory) + 8 * T) + emptied * (memory + 4 * T) + 4 * c["batch"], "flops": copied}


# ---- the same from the definition, in 64 bits --------------------------------------------------------------------
def _exact_values(pages):
    """Values [n_pages, 64, 128] of K and V."""
    n = pages.shape[0]
    kc = pages[:, :4096].reshape(n, 64, 64)
    vc = pages[:, 4096:8192].reshape(n, 4, 4, 16, 4, 4).permute(0, 1, 2, 4, 3, 5).reshape(n, 64, 64)
    ks = pages[:, 8192:8448].reshape(n, 64, 4)
    vs = pages[:, 8448:].reshape(n, 4, 4, 4, 4).permute(0, 1, 2, 4, 3).reshape(n, 64, 4)

    def value(code, scale):
        x = torch.stack([code % 16, code // 16], -1).reshape(n, 64, 128).double()
        sign, x = torch.where(x >= 8, -1.0, 1.0).double(), x % 8
        e, m = x // 2, x % 2
        mag = torch.where(e > 0, (1 + m / 2) * 2.0 ** (e - 1), m / 2)
        return sign * mag * (2.0 ** (scale.double() - 127)).repeat_interleave(32, -1)

    return value(kc, ks), value(vc, vs)


def _exact_round(x):
    """Rows [..., 128] as the cache holds them: the nearest of the fifteen values, by distance."""
    x = x.double().reshape(*x.shape[:-1], 4, 32)
    a = x.abs().amax(-1, keepdim=True)
    unit = 2.0 ** torch.ceil(torch.log2(a / 6)).clamp(min=-126)
    y = (x / unit).abs()
    level = torch.tensor([0, 1, 2, 4, 0.5, 1.5, 3, 6], device=x.device, dtype=torch.float64)[[0, 4, 1, 5, 2, 6, 3, 7]]
    middle = (level[1:] + level[:-1]) / 2
    code = torch.bucketize(y, middle)                    # a value in the middle goes to the even code
    tie = (code < 7) & (y == middle[code.clamp(max=6)]) & (code % 2 == 1)
    return (torch.sign(x) * level[code + tie.long()] * unit).reshape(*x.shape[:-2], 128)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    B, H, Hk = c["batch"], c["n_q_heads"], c["n_kv_heads"]
    C, T = s["C"], s["table"].shape[-1]
    if c["op"] == "append":
        out = {"K": s["K"].double(), "V": s["V"].double(), "Kidx": s["Kidx"].double()}
        k, v = _exact_round(s["k_new"]), _exact_round(s["v_new"])
        y = s["k_new"].double() @ s["w"]["Uk"].double().t()
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * s["w"]["norm_k_w"].double()
        for b, f in enumerate(s["src_of"].tolist()):
            for h in range(Hk):
                n = int(s["len_before"][f, h])
                out["Kidx"][b, h, :n] = s["Kidx"][f, h, :n].double()
                for name, new in (("K", k), ("V", v), ("Kidx", y)):
                    out[name][b, h, n:n + c["n_new"]] = new[b, h]
        return out
    if c["op"] == "fork":
        out = {n: s[n].double() for n in ("Kidx", "M", "b")}
        for b, f in enumerate(s["src_of"].tolist()):
            if f < 0:
                out["M"][b], out["b"][b] = 0, 0
            elif f != b:
                out["M"][b], out["b"][b] = s["M"][f].double(), s["b"][f].double()
                for h in range(Hk):
                    n = int(s["len"][f, h])
                    out["Kidx"][b, h, :n] = s["Kidx"][f, h, :n].double()
        return out
    if c["op"] == "attend":
        out = torch.zeros((B, c["n_q"], H, D), dtype=torch.float64, device=DEV)
        w = {k: v.double() for k, v in s["w"].items()}
        for b in range(B):
            for h in range(Hk):
                n = int(s["len"][b, h])
                used = s["table"][b, h, :(n + SLOTS - 1) // SLOTS].long()
                k, v = (x.reshape(-1, D)[:n] for x in _exact_values(s["pages"][used]))
                ok = torch.ones((c["n_q"], n), dtype=torch.bool, device=DEV)
                if s["q_pos"] is not None:
                    ok = s["pos"][b, h, :n].unsqueeze(0) <= s["q_pos"][b].unsqueeze(1)
                for j in range(h * (H // Hk), (h + 1) * (H // Hk)):
                    q = s["q"][b, :, j].double()
                    p = torch.softmax((q @ k.t() / math.sqrt(D)).masked_fill(~ok, -math.inf), -1)
                    phi = q @ w["Wtheta"].t()
                    m = phi @ s["M"][b, h].double() / ((phi * phi) @ s["b"][b, h].double() + EPS).unsqueeze(-1)
                    out[b, :, j] = torch.where(ok.any(-1, keepdim=True), p @ v, 0.0) + torch.sigmoid(q @ w["wg"] + s["cg"]).unsqueeze(-1) * m
        return {"out": out}
    # unpack, compact: the rows themselves
    out = {"K": s["K"].double(), "V": s["V"].double()}
    if c["op"] == "compact":
        out["Kidx"] = s["Kidx"].double()
    for b in range(B):
        for h in range(Hk):
            f = int(s["src_of"][b]) if c["op"] == "compact" else b
            used = s["table"][f, h].clamp(min=0).long()
            k, v = (x.reshape(-1, D)[:C] for x in _exact_values(s["pages"][used]))
            if c["op"] == "unpack":
                at = s["idx"][b, h, :c["n_listed"]].long()
                out["K"][b, h, at], out["V"][b, h, at] = k[at], v[at]
            elif f != b:
                n = c["keep"]
                kept, left = s["keep_idx"][b, h, :n].long(), s["evict_idx"][b, h, :c["cached"] - n].long()
                inside = int((kept < n).sum())
                src = torch.arange(n, device=DEV)
                src[left[:n - inside]] = kept[inside:]   # the holes take the entries from behind, in order
                out["K"][b, h, :n], out["V"][b, h, :n] = k[src], v[src]
                out["Kidx"][b, h] = s["Kidx"][f, h].double()
                out["Kidx"][b, h, :n] = s["Kidx"][f, h, src].double()
    return out

