"""Host-side checks of the calls on the 4-bit cache (no GPU): refusals before anything is enqueued, and the model of its rounding."""
import ctypes as C

import numpy as np
import pytest

import paper_2605_25475_amd as im
from packed_model import LEVELS, quantise
from paper_2605_25475_amd import binding as B

X = 1 << 21   # a non-null stand-in address; every call below must fail before using it
E = im.IM_ERR_INVALID_ARG


def _handle(**kw):
    d = dict(batch=2, n_q_heads=32, n_kv_heads=8, capacity=512, n_idx_heads=8, max_queries=16)
    d.update(kw)
    lib, c, h = im.load_library(), im.Config(**d).c_struct(), C.c_void_p()
    assert lib.im_create(C.byref(c), 1 << 20, lib.im_workspace_bytes(C.byref(c)), C.byref(h)) == im.IM_OK
    return lib, h


ST = B.ImState(None, None, X, X, X, X, X, X)
PR = B.ImParams(X, X, X, None, None, X, X, 0.0)
PK = B.ImPacked(X, X, X, 16)


def _calls(st=ST, pr=PR, pk=PK, **bad):
    """name -> arguments behind the handle, with one of them replaced."""
    st, pr, pk = C.byref(st), C.byref(pr), C.byref(pk)
    v = dict(k=X, v=X, pos=X, n_new=1, idx=X, n_idx=X, K=X, V=X, q=X, q_pos=X, n_q=1, out=X, keep=X, n_keep=X, evict=X, n_evict=X, src_of=X)
    v.update(bad)
    return {
        "im_append_packed": (pr, st, pk, v["k"], v["v"], v["pos"], v["n_new"], None),
        "im_unpack_kv": (st, pk, v["idx"], v["n_idx"], v["K"], v["V"], None),
        "im_attn_packed_with_readout": (pr, st, pk, v["q"], v["q_pos"], v["n_q"], v["out"], None, None),
        "im_compact_packed": (st, pk, v["keep"], v["n_keep"], v["evict"], v["n_evict"], None),
        "im_fork_packed": (st, pk, v["src_of"], None),
    }


@pytest.mark.parametrize("name", list(_calls()))
def test_states_pools_and_handles_are_checked(name):
    lib, h = _handle()
    f = getattr(lib, name)
    assert f(None, *_calls()[name]) == E
    for i in range(2, 8):
        parts = [None, None] + [X] * 6
        parts[i] = None
        assert f(h, *_calls(st=B.ImState(*parts))[name]) == E
    for pk in (B.ImPacked(None, X, X, 16), B.ImPacked(X, None, X, 16), B.ImPacked(X, X, None, 16), B.ImPacked(X, X, X, 0),
               B.ImPacked(X, X, X, -1), B.ImPacked(X + 8, X, X, 16)):
        assert f(h, *_calls(pk=pk)[name]) == E
        assert b"pages" in lib.im_last_error(h)
    lib2, shared = _handle(head_shared=1, idx_dim=16)
    assert f(shared, *_calls()[name]) == im.IM_ERR_UNSUPPORTED
    assert name.encode() in lib.im_last_error(shared)


@pytest.mark.parametrize("name,bad", [
    ("im_append_packed", dict(k=None)), ("im_append_packed", dict(v=None)), ("im_append_packed", dict(pos=None)),
    ("im_append_packed", dict(n_new=0)), ("im_append_packed", dict(n_new=513)), ("im_append_packed", dict(pr=B.ImParams(X, X, None, None, None, X, X, 0.0))),
    ("im_unpack_kv", dict(K=None)), ("im_unpack_kv", dict(V=None)), ("im_unpack_kv", dict(idx=None)), ("im_unpack_kv", dict(n_idx=None)),
    ("im_attn_packed_with_readout", dict(q=None)), ("im_attn_packed_with_readout", dict(out=None)),
    ("im_attn_packed_with_readout", dict(n_q=0)), ("im_attn_packed_with_readout", dict(n_q=(1 << 31) // 64)),
    ("im_attn_packed_with_readout", dict(pr=B.ImParams(X, X, X, None, None, None, X, 0.0))),
    ("im_compact_packed", dict(keep=None)), ("im_compact_packed", dict(n_keep=None)), ("im_compact_packed", dict(evict=None)),
    ("im_compact_packed", dict(n_evict=None)), ("im_fork_packed", dict(src_of=None))])
def test_arguments_are_checked(name, bad):
    lib, h = _handle()
    assert getattr(lib, name)(h, *_calls(**bad)[name]) == E


@pytest.mark.parametrize("name,arg", [("im_append_packed", "k"), ("im_append_packed", "v"), ("im_unpack_kv", "K"), ("im_unpack_kv", "V"),
                                      ("im_attn_packed_with_readout", "q"), ("im_attn_packed_with_readout", "out")])
@pytest.mark.parametrize("off", [2, 8])
def test_rows_that_begin_off_a_16_byte_boundary_are_refused(name, arg, off):
    lib, h = _handle()
    assert getattr(lib, name)(h, *_calls(**{arg: X + off})[name]) == E
    assert b"boundary" in lib.im_last_error(h)


def test_a_readout_off_a_16_byte_boundary_is_refused():
    lib, h = _handle()
    assert lib.im_attn_packed_with_readout(h, C.byref(PR), C.byref(ST), C.byref(PK), X, X, 1, X, X + 4, None) == E


def test_scoring_and_selection_take_a_state_without_rows_and_the_others_do_not():
    lib, h = _handle()
    st, pr = C.byref(ST), C.byref(PR)
    # (refused for other reasons: the state itself passes)
    assert lib.im_index_score(h, pr, st, X, X, X, 0, X, None) == E and b"n_q" in lib.im_last_error(h)
    assert lib.im_topb_select(h, X, st, 513, X, X, X, X, None) == E and b"budget" in lib.im_last_error(h)
    for rc in (lib.im_memory_update(h, pr, st, X, X, 0.9, 0.5, None), lib.im_compact_kv(h, st, X, X, X, X, None),
               lib.im_append_kv(h, st, X, X, X, 1, None), lib.im_decode_attn_with_readout(h, pr, st, X, X, None, None)):
        assert rc == E and b"state" in lib.im_last_error(h)


def test_the_models_rounding():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 128)) * 10.0 ** rng.integers(-20, 20, (50, 1))
    got = quantise(x)
    for row in range(50):
        for c in range(4):
            part, q = x[row, 32 * c:32 * c + 32], got[row, 32 * c:32 * c + 32]
            big = np.abs(part).max()
            u = 2.0 ** np.ceil(np.log2(big / 6))
            assert 3 * u < big <= 6 * u
            assert set(np.abs(q / u)) <= set(LEVELS)
            assert (np.abs(q - part) <= np.abs(part[:, None] - np.concatenate([LEVELS, -LEVELS]) * u).min(1) * (1 + 1e-9)).all()
    ties = np.zeros(128)
    ties[:8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5]
    assert list(quantise(ties)[:8]) == [6, 0, 1, 1, 2, 2, 4, -4]
    assert np.isnan(quantise(np.full(128, np.inf))).all() and (quantise(np.zeros(128)) == 0).all()


def test_scoring_and_selection_refuse_a_state_with_half_of_its_rows_and_shared_heads_without_any():
    lib, h = _handle()
    _, shared = _handle(head_shared=1, idx_dim=16)
    pr = C.byref(PR)
    for handle, st in ((h, B.ImState(None, X, *[X] * 6)), (h, B.ImState(X, None, *[X] * 6)), (shared, ST),
                       (shared, B.ImState(None, X, *[X] * 6)), (shared, B.ImState(X, None, *[X] * 6))):
        # (n_q and the budget are wrong as well, so that nothing is enqueued whatever is looked at)
        assert lib.im_index_score(handle, pr, C.byref(st), X, X, X, 0, X, None) == E
        assert b"state" in lib.im_last_error(handle)
        assert lib.im_topb_select(handle, X, C.byref(st), 513, X, X, X, X, None) == E
        assert b"state" in lib.im_last_error(handle)
