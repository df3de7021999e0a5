"""Host-side checks of the serving step's entry points: what they refuse before anything is launched, their workspaces, and the rotary frequencies."""
import ctypes as C
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def b():
    import paper_2408_00741_amd.binding as binding
    return binding


HERE = 4096 * 16          # an address that is never read: every call below is refused before a launch


def _step(b, ws=HERE, nbytes=1 << 20, **kw):
    d = dict(n_req=4, n_token=8, page_tokens=16, n_page=32, max_pages=4, ctx_len=HERE, new_len=HERE, block_table=HERE, free_pages=HERE, free_state=HERE)
    o = dict(cu_new=HERE * 2, kv_len=HERE * 3, next_len=HERE * 4, pos=HERE * 5, slot=HERE * 6, free_state=HERE * 7)
    for k, v in kw.items():
        (o if k.startswith("o_") else d)[k[2:] if k.startswith("o_") else k] = v
    return b._lib.dyn_kv_step(C.byref(b._KvRequests(**d)), C.byref(b._KvPlan(**o)), ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(ctx_len=None), -1), (dict(o_cu_new=None), -1), (dict(o_slot=None), -1), (dict(ws=None), -1), (dict(n_req=0), -2), (dict(n_token=-1), -2),
    (dict(page_tokens=0), -2), (dict(page_tokens=24), -2), (dict(page_tokens=8192), -2), (dict(n_page=0), -2), (dict(n_page=1 << 27), -2),
    (dict(max_pages=1 << 30), -2), (dict(max_pages=0), -2), (dict(o_free_state=HERE), -3), (dict(o_next_len=HERE), -3), (dict(ws=HERE + 8), -6), (dict(nbytes=256), -6)])
def test_step_refuses(b, kw, status):
    assert _step(b, **kw) == status
    assert b.dyn_last_error()


def _heads(**kw):
    d = dict(n_token=3, n_q_head=8, n_kv_head=2, head_dim=64, type=2, cache_type=2, page_tokens=16, n_page=32)
    d.update(kw)
    return d


BAD_HEADS = [(dict(n_kv_head=3), -2), (dict(n_kv_head=0), -2), (dict(n_q_head=0), -2), (dict(head_dim=72), -2), (dict(head_dim=144), -2), (dict(head_dim=0), -2),
             (dict(type=3), -3), (dict(type=0), -3), (dict(cache_type=1), -3), (dict(page_tokens=48), -2), (dict(n_page=0), -2), (dict(n_page=1 << 28), -2), (dict(n_token=-1), -2)]


def _append(b, **kw):
    rows = b._Rows(HERE, 512, 64)
    w = np.ones(64)
    d = _heads(q=rows, k=rows, v=rows, q_out=rows, pos=HERE, slot=HERE, k_cache=HERE, v_cache=HERE, k_scale=None, v_scale=None, rotary_dim=64, interleaved=0,
               inv_freq=w.ctypes.data, amplitude=1.0)
    d.update(kw)
    return b._lib.dyn_rope_append(C.byref(b._Append(**d)), None)


@pytest.mark.parametrize("kw,status", BAD_HEADS + [
    (dict(rotary_dim=66), -2), (dict(rotary_dim=63), -2), (dict(rotary_dim=-2), -2), (dict(inv_freq=None), -1), (dict(amplitude=math.nan), -4),
    (dict(k_scale=HERE), -3), (dict(pos=None), -1), (dict(k_cache=None), -1), (dict(v_cache=HERE + 8), -2)])
def test_append_refuses(b, kw, status):
    assert _append(b, **kw) == status


def test_append_refuses_frequencies_that_are_not_finite(b):
    w = np.ones(64)
    w[31] = math.inf
    assert _append(b, inv_freq=w.ctypes.data) == -4
    assert _append(b, n_token=0, pos=None, slot=None) == 0            # nothing to do


def _attend(b, ws=HERE, nbytes=1 << 40, **kw):
    rows = b._Rows(HERE, 512, 64)
    d = _heads(n_req=2, max_pages=8, max_new=2, max_kv=100, window=0, n_sink=0, scale=0.1, q=rows, out=rows, k_cache=HERE, v_cache=HERE, k_scale=None,
               v_scale=None, block_table=HERE, cu_new=HERE, kv_len=HERE)
    d.update(kw)
    return b._lib.dyn_paged_attention(C.byref(b._Attention(**d)), ws, nbytes, None)


@pytest.mark.parametrize("kw,status", BAD_HEADS + [
    (dict(n_req=0), -2), (dict(max_pages=0), -2), (dict(max_new=-1), -2), (dict(max_kv=-1), -2), (dict(max_pages=1 << 28), -2), (dict(window=-1), -3), (dict(n_sink=-1), -3),
    (dict(scale=math.inf), -4), (dict(v_scale=HERE), -3), (dict(kv_len=None), -1), (dict(q=None), -1), (dict(k_cache=HERE + 2), -2), (dict(ws=None), -1),
    (dict(ws=HERE + 16), -6), (dict(nbytes=300), -6), (dict(n_token=2 ** 31 - 1, n_q_head=64), -2)])
def test_attention_refuses(b, kw, status):
    if "q" in kw:
        kw = dict(q=b._Rows(None, 512, 64))
    assert _attend(b, **kw) == status
    assert _attend(b, n_token=0, q=b._Rows(None, 0, 0)) == 0


def test_workspaces(b):
    assert b.dyn_kv_step_workspace(0) == 0 and b.dyn_kv_step_workspace(5000) >= 256 + 2 * 5001 * 4
    assert b.dyn_paged_attention_workspace(0, 1, 8, 8, 64, 1, 1) == 0 and b.dyn_paged_attention_workspace(1, 1, 8, 3, 64, 1, 1) == 0
    # never less for more keys, and bounded
    for B, T, H, G, D, n in ((1, 1, 64, 8, 128, 1), (64, 64, 64, 8, 128, 1), (3, 700, 32, 8, 128, 300), (1, 8192, 32, 8, 128, 8192), (2, 40, 8, 1, 64, 30)):
        sizes = [b.dyn_paged_attention_workspace(B, T, H, G, D, n, kv) for kv in (1, 40, 100, 777, 1000, 5000, 5001, 40000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[-1] < 160 << 20 and all(s % 256 == 0 for s in sizes)


def test_rope_frequencies(b):
    w, a = b.dyn_rope_frequencies(64, 10000.0)
    want = [10000.0 ** (-2.0 * i / 64) for i in range(32)]
    assert np.allclose(w, want, rtol=1e-15, atol=0) and a == 1.0
    w2, _ = b.dyn_rope_frequencies(64, 10000.0, b.DYN_ROPE_LINEAR, 4.0)
    assert np.allclose(w2, w / 4, rtol=1e-15, atol=0)
    w3, a = b.dyn_rope_frequencies(64, 10000.0, b.DYN_ROPE_PARTS, 4.0, 8192.0, 1.0, 32.0)
    turns = 8192 * w / (2 * math.pi)
    assert np.allclose(w3[turns >= 32], w[turns >= 32], rtol=1e-15) and np.allclose(w3[turns <= 1], w[turns <= 1] / 4, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and np.all((w3[mid] < w[mid]) & (w3[mid] > w[mid] / 4)) and abs(a - (0.1 * math.log(4.0) + 1)) < 1e-15
    for kw in (dict(rotary_dim=63), dict(rotary_dim=130), dict(rotary_dim=0), dict(base=0.0), dict(base=math.inf), dict(scaling=3), dict(scaling=1, factor=0.5), dict(scaling=2, factor=2.0),
               dict(scaling=2, factor=2.0, original_tokens=10.0, slow_turns=4.0, fast_turns=4.0)):
        with pytest.raises(b.DynError):
            b.dyn_rope_frequencies(**{"rotary_dim": 64, **kw})


def test_the_plain_step_on_a_worked_example():
    from tests import serve_plain as plain
    # pages of 4: request 0 holds 6 tokens (pages 5, 2) and adds 3 (one new page); 1 is through (page 0); 2 starts with 5 tokens (two pages), one free page is left: refused
    table = np.array([[5, 2, -1], [0, -1, -1], [-1, -1, -1]], np.int32)
    ring = np.array([3, 1, 9, 9, 9, 9, 4, 7], np.int32)[:8]
    cu, kv, nxt, pos, slot, t, r, st, refused = plain.step(np.array([6, 2, 0]), np.array([3, -1, 5]), table, ring, np.array([0, 2]), 4, 8)
    assert cu.tolist() == [0, 3, 3, 8] and kv.tolist() == [9, 0, 0] and nxt.tolist() == [9, 0, 0] and refused == [False, False, True]
    assert pos.tolist() == [6, 7, 8, -1, -1, -1, -1, -1] and slot.tolist() == [2 * 4 + 2, 2 * 4 + 3, 3 * 4, -1, -1, -1, -1, -1]
    assert t[0].tolist() == [5, 2, 3] and r[:3].tolist() == [3, 1, 0] and st.tolist() == [1, 2]
