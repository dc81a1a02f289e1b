"""Long-cache calls without a GPU: what they refuse, the size of the 4-bit pool, and the float64 definitions of the tests
against hand-worked values."""
import ctypes as C

import numpy as np
import pytest

from paper_2601_07568_amd import binding as B
from paper_2601_07568_amd import synth
from tests import long_cache as R

BF = synth.ModelShape(2, 64, 6, 3, 64, 64, 64, 63)
P = 0x4000                                                                  # stands for device memory; the host never reads it


def make(ms=BF, **kw):
    d = dict(page_tokens=32, max_pages_per_seq=8, n_pages=8, max_batch=2, max_q=32, max_tokens=0)
    d.update(kw)
    L, cfg = B.lib(), B.make_config(ms, **d)
    lw = (B.LayerW * max(1, cfg.n_layers))()
    for l in range(cfg.n_layers):
        for name, _ in B.LayerW._fields_:
            setattr(lw[l], name, 0x1000)
    w, ctx = B.Weights(0x1000, 0x1000, 0x1000, lw), C.c_void_p()
    assert L.dllm_create(C.byref(ctx), C.byref(cfg), C.byref(w), 0x10000, L.dllm_kv_pool_bytes(C.byref(cfg)), 0x20000 * 256,
                         L.dllm_workspace_bytes(C.byref(cfg))) == B.DLLM_OK
    return L, cfg, ctx


def test_kv4_pool_bytes_and_attach():
    L, cfg, ctx = make(page_tokens=64)
    assert L.dllm_kv4_pool_bytes(C.byref(cfg), 5) == 2 * 5 * 3 * 2 * 34 * 64
    assert L.dllm_kv4_pool_bytes(C.byref(cfg), 0) == 0
    assert L.dllm_kv4_pool_bytes(C.byref(cfg), (1 << 25)) == 0              # 2^31 slots
    n = L.dllm_kv4_pool_bytes(C.byref(cfg), 5)
    assert L.dllm_kv4_attach(None, 0x10000, n, 5) == B.DLLM_EINVAL
    assert L.dllm_kv4_attach(ctx, 0x10000, n, 0) == B.DLLM_EINVAL
    assert L.dllm_kv4_attach(ctx, 0x10010, n, 5) == B.DLLM_EINVAL           # not 256-byte aligned
    assert L.dllm_kv4_attach(ctx, 0x10000, n - 1, 5) == B.DLLM_ENOSPACE
    assert L.dllm_kv4_attach(ctx, 0x10000, n, 5) == B.DLLM_OK
    assert L.dllm_kv4_attach(ctx, None, 0, 0) == B.DLLM_OK
    assert L.dllm_kv4_store(ctx, None, 32, P, P) == B.DLLM_EINVAL           # detached again
    L.dllm_destroy(ctx)


@pytest.mark.parametrize("ms,page", [(synth.TINY, 32), (BF, 16), (BF, 40)])
def test_kv4_needs_bf16_and_whole_groups(ms, page):
    L, cfg, ctx = make(ms, page_tokens=page)
    assert L.dllm_kv4_pool_bytes(C.byref(cfg), 4) == 0
    assert L.dllm_kv4_attach(ctx, 0x10000, 1 << 30, 4) == B.DLLM_ESHAPE
    L.dllm_destroy(ctx)


def test_plan_and_slots_refuse():
    L, cfg, ctx = make()
    ok = (P, P, P, P, P, P)
    for i in (0, 2, 3, 4):                                                   # `first` and `granted` may be NULL
        args = list(ok)
        args[i] = None
        assert L.dllm_plan_pages(ctx, None, B.POOL_KV, 1, 0, *args) == B.DLLM_EINVAL
    assert L.dllm_plan_pages(None, None, B.POOL_KV, 1, 0, *ok) == B.DLLM_EINVAL
    assert L.dllm_plan_pages(ctx, None, B.POOL_KV, 0, 0, *ok) == B.DLLM_EINVAL
    assert L.dllm_plan_pages(ctx, None, B.POOL_KV, 1, -1, *ok) == B.DLLM_EINVAL
    assert L.dllm_plan_pages(ctx, None, B.POOL_KV, 3, 0, *ok) == B.DLLM_ESHAPE
    assert L.dllm_plan_pages(ctx, None, B.POOL_KV4, 1, 0, *ok) == B.DLLM_EINVAL     # no such pool
    assert L.dllm_plan_pages(ctx, None, 2, 1, 0, *ok) == B.DLLM_EINVAL
    for i in range(5):
        args = [P] * 5
        args[i] = None
        assert L.dllm_slot_map(ctx, None, B.POOL_KV, 1, 4, *args) == B.DLLM_EINVAL
    assert L.dllm_slot_map(ctx, None, B.POOL_KV, 0, 4, P, P, P, P, P) == B.DLLM_EINVAL
    assert L.dllm_slot_map(ctx, None, B.POOL_KV, 1, 0, P, P, P, P, P) == B.DLLM_EINVAL
    assert L.dllm_slot_map(ctx, None, B.POOL_KV, 3, 4, P, P, P, P, P) == B.DLLM_ESHAPE
    assert L.dllm_slot_map(ctx, None, B.POOL_KV4, 1, 4, P, P, P, P, P) == B.DLLM_EINVAL
    L.dllm_destroy(ctx)
    L, cfg, ctx = make(page_tokens=1 << 20, max_pages_per_seq=1 << 11, n_pages=1)   # 2^31 positions
    assert L.dllm_slot_map(ctx, None, B.POOL_KV, 1, 4, P, P, P, P, P) == B.DLLM_ESHAPE
    L.dllm_destroy(ctx)


def test_moves_refuse():
    L, cfg, ctx = make()
    assert L.dllm_kv4_load(ctx, None, 32, P, P) == B.DLLM_EINVAL            # no pool
    n = L.dllm_kv4_pool_bytes(C.byref(cfg), 4)
    assert L.dllm_kv4_attach(ctx, 0x10000, n, 4) == B.DLLM_OK
    for f in (L.dllm_kv4_store, L.dllm_kv4_load):
        assert f(None, None, 32, P, P) == B.DLLM_EINVAL
        assert f(ctx, None, 0, P, P) == B.DLLM_EINVAL
        assert f(ctx, None, 32, None, P) == B.DLLM_EINVAL
        assert f(ctx, None, 32, P, None) == B.DLLM_EINVAL
    assert L.dllm_kv4_store(ctx, None, 33, P, P) == B.DLLM_EINVAL           # not whole groups
    L.dllm_destroy(ctx)


def test_attend_and_step_view_refuse():
    L, cfg, ctx = make()

    def view(window=0, n_sink=0, len4=None, table4=None):
        return C.byref(B.CacheView(window, n_sink, len4, table4))
    A, S = L.dllm_attend, L.dllm_denoise_step_view
    assert A(ctx, None, 2, 1, 32, 64, P, P, None, P, None, P + 16) == B.DLLM_EINVAL       # layer
    assert A(ctx, None, -1, 1, 32, 64, P, P, None, P, None, P + 16) == B.DLLM_EINVAL
    assert A(ctx, None, 0, 1, 32, 64, P, P, None, P, None, P) == B.DLLM_EINVAL            # in place
    assert A(ctx, None, 0, 1, 32, 64, P + 8, P, None, P, None, P + 16) == B.DLLM_EINVAL   # alignment
    assert A(ctx, None, 0, 1, 32, 64, P, P, None, P, None, P + 20) == B.DLLM_EINVAL
    assert A(ctx, None, 0, 1, 32, 64, P, P, None, P, None, None) == B.DLLM_EINVAL
    assert A(ctx, None, 0, 1, 32, 64, None, P, None, P, None, P) == B.DLLM_EINVAL
    assert A(ctx, None, 0, 1, 32, -1, P, P, None, P, None, P + 16) == B.DLLM_EINVAL
    assert A(ctx, None, 0, 3, 32, 64, P, P, None, P, None, P + 16) == B.DLLM_ESHAPE
    assert A(ctx, None, 0, 1, 33, 64, P, P, None, P, None, P + 16) == B.DLLM_ESHAPE
    assert A(ctx, None, 0, 1, 32, 225, P, P, None, P, None, P + 16) == B.DLLM_ESHAPE      # 257 keys in 8 pages of 32
    assert S(ctx, None, 1, 32, 225, P, P, None, P, None, P, P, None) == B.DLLM_ESHAPE
    assert S(ctx, None, 1, 32, 64, P, P, None, P, None, None, P, None) == B.DLLM_EINVAL
    assert S(ctx, None, 1, 32, 64, P, P, None, P, None, P, None, None) == B.DLLM_EINVAL
    for bad in (view(-1), view(4, -1), view(len4=P), view(table4=P), view(len4=P, table4=P)):   # (the last: no 4-bit pool)
        assert A(ctx, None, 0, 1, 32, 64, P, P, None, P, bad, P + 16) == B.DLLM_EINVAL
        assert S(ctx, None, 1, 32, 64, P, P, None, P, bad, P, P, None) == B.DLLM_EINVAL
    L.dllm_destroy(ctx)


# ------------------------------------------------------------------------------------------------ the definitions

def test_encode_by_hand():
    x = np.zeros(32)
    x[:8] = [7.0, 6.5, -5.0, 2.5, 0.25, 0.75, -0.2, 3.5]                    # amax 7: s = 1
    code, byte = R.encode(x)
    assert byte == 127 and code[:8].tolist() == [7, 7, 8 + 6, 4, 0, 2, 0, 6]
    x[0] = 7.25                                                             # s = 2
    code, byte = R.encode(x)
    assert byte == 128 and R.decode(code, byte)[:4].tolist() == [8.0, 6.0, -4.0, 2.0]
    assert R.encode(np.zeros(32))[1] == 7
    x = np.full(32, 1.0)
    x[:3] = [np.inf, -np.inf, np.nan]
    code, byte = R.encode(x)
    assert byte == 125 and R.decode(code, byte)[:4].tolist() == [1.5, -1.5, 0.0, 1.0]
    assert R.encode(np.full(32, 3e38))[1] == 252


def test_plan_by_hand():
    # pages of 4; sequence 0 grows from 1 to 3 pages, 1 ends, 2 asks for more than is left, 3 needs nothing
    t, s, n, g, bl, bp = R.plan_pages(4, 6, 0, [9, 0, 20, 4], None, [[5, -1, -1, -1, -1], [2, 3, -1, -1, -1], [-1] * 5, [1] + [-1] * 4],
                                      [0, 4, 9, 9, 9, 9], 2)
    assert t == [[5, 3, 2, -1, -1], [-1] * 5, [-1] * 5, [1] + [-1] * 4] and g == [1, 1, 0, 1] and n == 2 and s[:4] == [0, 4, 2, 3] and not bl and not bp
    # a head and a tail: positions 0 .. 1 and 9 .. 11 of pages of 4
    t, s, n, *_ = R.plan_pages(4, 6, 2, [12], [9], [[0, 1, 2]], [3, 4, 5, 9, 9, 9], 3)
    assert t == [[0, -1, 2]] and n == 4 and s[3] == 1
    assert R.slot_map(4, 6, [1, 0], [6, 2], [[5, 3], [-1, 0]], 9) == ([0, 5, 7], [21, 22, 23, 12, 13, -1, -1, -1, -1], False)
