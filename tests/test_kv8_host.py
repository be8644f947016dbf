"""The 8-bit pool and the page calls without a GPU: the oracle against torch's conversions and a worked page, and what the
calls refuse before anything would be enqueued."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2410_01228_amd import binding as cs


def test_oracle_codes_are_e4m3():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.isnan(codes), np.isnan(kv8.VALUES))
    assert np.array_equal(codes[~np.isnan(codes)], kv8.VALUES[~np.isnan(codes)].astype(np.float32))
    # every halfway point between neighbours, and either side of it
    pos = kv8.VALUES[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, mid * (1 - 2.0 ** -20), mid * (1 + 2.0 ** -20)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv8.encode(x), want)
    assert kv8.encode(np.nan) & 127 == 127 and kv8.encode(1e9) == 126 and kv8.encode(-np.inf) == 254


@pytest.mark.parametrize("D", [64, 128])
def test_oracle_places_fill_a_block_once(D):
    t, d = np.arange(16)[:, None], np.arange(D)
    for index in (kv8.k_index, kv8.v_index):
        assert sorted(index(t, d).ravel()) == list(range(16 * D))
    # a unit of K is 16 features of a token, a unit of V 4 tokens of a feature in 4 feature tiles
    assert list(kv8.k_index(3, np.arange(16, 32))) == [(16 + 3) * 16 + i for i in range(16)]
    assert list(kv8.v_index(np.arange(4, 8), 2)) == [(16 + 2) * 16 + i for i in range(4)]
    assert kv8.v_index(4, 18) == (16 + 2) * 16 + 4


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.01, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -100), (1e-35, -100)])
def test_oracle_exponent(top, e):
    assert kv8.exponent_for(top) == e


def test_page_bytes():
    assert cs.cs_kv8_page_bytes(8, 128) == 2 * 8 * 16 * 128 + 64 == kv8.page_bytes(8, 128)
    assert cs.cs_kv8_page_bytes(1, 64) == 2 * 16 * 64 + 16 == kv8.page_bytes(1, 64)       # 8 bytes of scales, 8 of padding
    assert cs.cs_kv8_page_bytes(3, 128) % 16 == 0
    for bad in ((0, 128), (-1, 64), (8, 96), (8, 0), (70000, 128)):
        assert cs.cs_kv8_page_bytes(*bad) == 0


def _pool8(base=0x1000, L=2, P=8, Hkv=2, D=64, ps=None, ls=None):
    ps = 2 * Hkv * (16 * D + 4) if ps is None else ps
    return cs.cs_kv8_pool(base, L, P, Hkv, D, P * ps if ls is None else ls, ps)


def _batch(ctx, ql, blocks=64, dev=0x2000):
    h = torch.tensor(ctx, dtype=torch.int32)
    cu = torch.zeros(len(ql) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(ql, dtype=torch.int32), 0)
    return cs.cs_batch(len(ctx), int(cu[-1]), dev, blocks, dev, dev, h.data_ptr(), cu.data_ptr()), (h, cu)


BAD_POOLS = [
    (dict(base=0), cs.CS_ERR_INVALID_ARG), (dict(base=0x1008), cs.CS_ERR_INVALID_ARG), (dict(L=0), cs.CS_ERR_INVALID_ARG),
    (dict(P=0), cs.CS_ERR_INVALID_ARG), (dict(Hkv=0, ps=64), cs.CS_ERR_INVALID_ARG), (dict(D=96), cs.CS_ERR_UNSUPPORTED), (dict(D=256), cs.CS_ERR_UNSUPPORTED),
    (dict(ps=2 * 2 * 16 * 64), cs.CS_ERR_INVALID_ARG), (dict(ps=4120), cs.CS_ERR_INVALID_ARG), (dict(ls=7 * 4128), cs.CS_ERR_INVALID_ARG),
    (dict(ls=8 * 4128 + 8), cs.CS_ERR_INVALID_ARG), (dict(ps=1 << 62, ls=0), cs.CS_ERR_INVALID_ARG),
]


@pytest.mark.parametrize("change,status", BAD_POOLS)
def test_pools_that_are_refused(change, status):
    pool, (b, _keep) = _pool8(**change), _batch([3], [1])
    L, P, B = cs.lib(), ctypes.byref, ctypes.byref
    for f16 in ("", "_f16"):
        assert getattr(L, "cs_kv8_append" + f16)(P(pool), 0, B(b), 0x3000, 0x4000, None) == status
        assert getattr(L, "cs_paged_attention_mixed_kv8" + f16)(P(pool), 0, B(b), 0x3000, 0x4000, 4, 1.0, None, 0, None) == status
    assert L.cs_kv8_page_space(P(pool), ctypes.byref(cs.cs_page_space())) == status


def test_append_and_attention_refusals():
    L, r = cs.lib(), ctypes.byref
    pool, (b, _keep) = _pool8(), _batch([3, 0], [1, 20])
    inv = cs.CS_ERR_INVALID_ARG
    for fn in (L.cs_kv8_append, L.cs_kv8_append_f16):
        assert fn(None, 0, r(b), 0x3000, 0x4000, None) == inv
        assert fn(r(pool), -1, r(b), 0x3000, 0x4000, None) == inv and fn(r(pool), 2, r(b), 0x3000, 0x4000, None) == inv
        assert fn(r(pool), 0, None, 0x3000, 0x4000, None) == inv
        assert fn(r(pool), 0, r(b), None, 0x4000, None) == inv and fn(r(pool), 0, r(b), 0x3000, None, None) == inv
        assert fn(r(pool), 0, r(b), 0x3008, 0x4000, None) == inv and fn(r(pool), 0, r(b), 0x3000, 0x4004, None) == inv
        empty, (_k, _c) = _batch([], [])
        assert fn(r(pool), 0, r(empty), None, None, None) == cs.CS_OK
        short, _k2 = _batch([60], [10], blocks=4)
        assert fn(r(pool), 0, r(short), 0x3000, 0x4000, None) == inv                       # the table is too narrow
    for fn in (L.cs_paged_attention_mixed_kv8, L.cs_paged_attention_mixed_kv8_f16):
        def call(p=pool, layer=0, batch=b, q=0x3000, out=0x4000, hq=4, scale=1.0, ws=None, n=0, fn=fn):
            return fn(r(p), layer, r(batch), q, out, hq, scale, ws, n, None)
        assert call(layer=2) == inv and call(hq=0) == inv and call(hq=3) == inv and call(hq=34) == cs.CS_ERR_UNSUPPORTED
        assert call(q=None) == inv and call(out=0) == inv and call(q=0x3004) == inv and call(out=0x4008) == inv
        for s in (0.0, -1.0, float("inf"), float("nan")):
            assert call(scale=s) == inv
        # a batch whose tiles or sequences are cut needs its workspace
        cut, _k3 = _batch([100000], [1], blocks=8192)
        need = L.cs_paged_attention_kv8_workspace_bytes(r(cut), 4, 2, 64)
        assert need > 0
        assert call(batch=cut) == inv and call(batch=cut, ws=0x5000, n=need - 1) == cs.CS_ERR_WORKSPACE_TOO_SMALL and call(batch=cut, ws=0x5008, n=need) == inv
    assert L.cs_paged_attention_kv8_workspace_bytes(r(b), 4, 3, 64) == 0 and L.cs_paged_attention_kv8_workspace_bytes(None, 4, 2, 64) == 0


def _space(base=0x1000, L=3, P=8, pb=4128, ls=None, ps=None):
    ps = pb if ps is None else ps
    return cs.cs_page_space(base, L, P, pb, P * ps if ls is None else ls, ps)


def _tables(bt=0x2000, lens=0x3000, counts=0x4000, rows=4, blocks=8, pages=8, size=16):
    return cs.cs_page_tables(bt, lens, counts, rows, blocks, pages, size)


BAD_SPACES = [dict(base=0), dict(base=0x1004), dict(L=0), dict(P=0), dict(pb=0), dict(pb=4120), dict(ps=4112), dict(ps=4136), dict(ls=8 * 4128 - 16),
              dict(ls=8 * 4128 + 4), dict(ps=(1 << 62) - 16)]
BAD_TABLES = [dict(bt=0), dict(lens=0), dict(counts=0), dict(rows=0), dict(blocks=0), dict(pages=0), dict(size=0), dict(pages=9)]


@pytest.mark.parametrize("change", BAD_SPACES)
def test_page_spaces_that_are_refused(change):
    L, r, inv = cs.lib(), ctypes.byref, cs.CS_ERR_INVALID_ARG
    bad, good, t = _space(**change), _space(), _tables()
    assert L.cs_kv_pages_copy(r(bad), 0, 0x5000, r(good), 0, 0x6000, 1, 2, None) == inv
    assert L.cs_kv_pages_copy(r(good), 0, 0x5000, r(bad), 0, 0x6000, 1, 2, None) == inv
    assert L.cs_kv_pages_fork(r(bad), 0, 1, r(t), 0x5000, 0x6000, 0x7000, 1, None) == inv
    assert L.cs_kv_pages_compact(r(bad), 0, 1, r(t), r(t), 0x5000, 0x6000, 0x7000, 1 << 20, None) == inv


@pytest.mark.parametrize("change", BAD_TABLES)
def test_page_tables_that_are_refused(change):
    L, r, inv = cs.lib(), ctypes.byref, cs.CS_ERR_INVALID_ARG
    bad, s, t = _tables(**change), _space(), _tables()
    assert L.cs_kv_pages_fork(r(s), 0, 1, r(bad), 0x5000, 0x6000, 0x7000, 1, None) == inv
    assert L.cs_kv_pages_compact(r(s), 0, 1, r(bad), r(t), 0x5000, 0x6000, 0x7000, 1 << 20, None) == inv
    assert L.cs_kv_pages_compact(r(s), 0, 1, r(t), r(bad), 0x5000, 0x6000, 0x7000, 1 << 20, None) == inv
    if "pages" not in change or change["pages"] == 0:
        assert L.cs_kv_pages_free(r(bad), 0x5000, 1, 0x6000, 0x7000, None) == inv


def test_page_call_refusals():
    L, r, inv = cs.lib(), ctypes.byref, cs.CS_ERR_INVALID_ARG
    s, t = _space(), _tables()

    def copy(src=s, sl=0, si=0x5000, dst=s, dl=0, di=0x6000, layers=1, n=2):
        return L.cs_kv_pages_copy(r(src), sl, si, r(dst), dl, di, layers, n, None)
    assert copy(n=0) == cs.CS_OK and copy(layers=0) == cs.CS_OK and copy(sl=3, layers=0) == cs.CS_OK
    assert copy(n=-1) == inv and copy(layers=-1) == inv and copy(sl=-1) == inv and copy(dl=4, layers=0) == inv and copy(sl=2, layers=2) == inv
    assert copy(dl=1, layers=3) == inv and copy(si=None, n=9) == inv and copy(di=None, n=9) == inv
    assert copy(dst=_space(pb=4144)) == inv
    fork = L.cs_kv_pages_fork
    assert fork(r(s), 0, 1, r(t), None, None, None, 0, None) == cs.CS_OK
    assert fork(r(s), 0, 1, r(t), 0x5000, 0x6000, 0x7000, -1, None) == inv
    assert fork(r(s), 2, 1, r(t), 0x5000, 0x6000, 0x7000, 1, None) == inv and fork(r(s), 0, 4, r(t), 0x5000, 0x6000, 0x7000, 1, None) == inv
    for k in range(3):
        lists = [0x5000, 0x6000, 0x7000]
        lists[k] = None
        assert fork(r(s), 0, 1, r(t), *lists, 1, None) == inv
    assert L.cs_kv_pages_free(r(t), None, 1, 0x6000, 0x7000, None) == inv and L.cs_kv_pages_free(r(t), 0x5000, -1, 0x6000, 0x7000, None) == inv
    assert L.cs_kv_pages_free(r(t), 0x5000, 1, None, 0x7000, None) == inv and L.cs_kv_pages_free(r(t), 0x5000, 1, 0x6000, None, None) == inv
    need = L.cs_kv_pages_compact_workspace_bytes(8)
    assert need > 0 and L.cs_kv_pages_compact_workspace_bytes(0) == 0 == L.cs_kv_pages_compact_workspace_bytes(-5)

    def compact(new=t, ids=0x5000, used=0x6000, ws=0x7000, n=need, l0=0, l1=3):
        return L.cs_kv_pages_compact(r(s), l0, l1, r(t), r(new), ids, used, ws, n, None)
    assert compact(ids=None) == inv and compact(used=None) == inv and compact(ws=None) == inv and compact(ws=0x7004) == inv
    assert compact(n=need - 1) == cs.CS_ERR_WORKSPACE_TOO_SMALL and compact(l1=4) == inv and compact(l0=2, l1=1) == inv
    assert compact(new=_tables(rows=5)) == inv and compact(new=_tables(blocks=7)) == inv and compact(new=_tables(size=8)) == inv


def test_spaces_of_pools():
    s = cs.cs_page_space()
    p16 = cs.cs_kv_pool(0x1000, 2, 8, 16, 2, 64, 8 * 5000, 5000)
    assert cs.lib().cs_kv_page_space(ctypes.byref(p16), ctypes.byref(s)) == cs.CS_OK
    assert (s.base, s.num_layers, s.num_pages, s.page_bytes, s.layer_stride, s.page_stride) == (0x1000, 2, 8, 8192, 80000, 10000)
    p8 = _pool8(ps=4224)
    assert cs.lib().cs_kv8_page_space(ctypes.byref(p8), ctypes.byref(s)) == cs.CS_OK
    assert (s.page_bytes, s.layer_stride, s.page_stride) == (4112, 8 * 4224, 4224)
    assert cs.lib().cs_kv8_page_space(ctypes.byref(p8), None) == cs.CS_ERR_INVALID_ARG
    assert cs.lib().cs_kv_page_space(ctypes.byref(p16), None) == cs.CS_ERR_INVALID_ARG


def host_batch(ctx, new):
    blocks = max(-(-(c + n) // 16) for c, n in zip(ctx, new))
    return cs.Batch(torch.zeros((len(ctx), max(blocks, 1)), dtype=torch.int32), torch.tensor(ctx, dtype=torch.int32),
                    torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), device="cpu")


def test_attention_plans_of_drawn_batches():
    """The plan, and with it the workspace, is a function of the batch: the same when other batches were planned between."""
    r = np.random.default_rng(4)
    drawn = []
    for _ in range(60):
        hq, hkv, d = [(32, 8, 128), (28, 4, 128), (64, 8, 128), (40, 8, 128), (4, 2, 64), (6, 6, 64)][r.integers(6)]
        n = int(r.integers(1, 40))
        ctx = (10 ** r.uniform(0, 4.3, n)).astype(int).tolist()
        new = np.where(r.random(n) < 0.8, 1, r.integers(0, 900, n)).tolist()
        drawn.append((ctx, new, hq, hkv, d))
    first = [cs.cs_paged_attention_kv8_workspace_bytes(host_batch(c, n), hq, hkv, d) for c, n, hq, hkv, d in drawn]
    for (c, n, hq, hkv, d), x in reversed(list(zip(drawn, first))):
        b = host_batch(c, n)
        assert cs.cs_paged_attention_kv8_workspace_bytes(b, hq, hkv, d) == x < 1 << 31
        cs.cs_paged_attention_workspace_bytes(b, hq, hkv, d)                        # (the 16-bit plan of the same lengths is another)
        assert cs.cs_paged_attention_kv8_workspace_bytes(b, hq, hkv, d) == x


def test_the_binding_refuses_lists_that_are_too_short_or_of_another_type():
    staging = cs.PageSpace.staging(torch.zeros((2, 4, 64), dtype=torch.uint8))
    ids = torch.zeros(3, dtype=torch.int32)
    for src, dst, n in ((ids, ids[:2], None), (ids[:1], None, 2), (ids.long(), ids, None), (None, ids.long(), None)):
        with pytest.raises(AssertionError):
            cs.cs_kv_pages_copy(staging, 0, src, staging, 0, dst, 2, n, stream=0)
    tables = cs.PageTables(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(AssertionError):
        cs.cs_kv_pages_fork(staging, 0, 2, tables, ids, ids, ids[:2], stream=0)
    with pytest.raises(AssertionError):
        cs.cs_kv_pages_fork(staging, 0, 2, tables, ids, ids.long(), ids, stream=0)
    with pytest.raises(AssertionError):
        cs.cs_kv_pages_free(tables, ids, ids, ids, stream=0)
    with pytest.raises(AssertionError):
        cs.cs_kv_pages_free(tables, ids, torch.zeros(4, dtype=torch.int32), ids[:0], stream=0)
    with pytest.raises(AssertionError):
        cs.cs_kv_pages_compact(staging, 0, 2, tables, tables, ids, ids, torch.zeros(256, dtype=torch.uint8), stream=0)
    with pytest.raises(AssertionError):
        cs.Pool8(torch.zeros(cs.cs_kv8_page_bytes(2, 64) * 3 - 1, dtype=torch.uint8), 1, 3, 2, 64)


def test_the_binding_refuses_views_that_the_kernels_would_read_past():
    """Every second entry of a list, heads out of wider rows, too few rows: the calls take bare addresses, and would read the neighbours."""
    staging, ids = cs.PageSpace.staging(torch.zeros((2, 4, 64), dtype=torch.uint8)), torch.zeros(4, dtype=torch.int32)
    bad = torch.zeros(8, dtype=torch.int32)[::2]
    tables = cs.PageTables(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    scratch = torch.zeros(256, dtype=torch.uint8)
    for call in (lambda: cs.cs_kv_pages_copy(staging, 0, bad, staging, 0, ids, 2, stream=0),
                 lambda: cs.cs_kv_pages_copy(staging, 0, None, staging, 0, bad, 2, stream=0),
                 lambda: cs.cs_kv_pages_fork(staging, 0, 2, tables, bad, ids, ids, stream=0),
                 lambda: cs.cs_kv_pages_fork(staging, 0, 2, tables, ids, bad, ids, stream=0),
                 lambda: cs.cs_kv_pages_fork(staging, 0, 2, tables, ids, ids, bad, stream=0),
                 lambda: cs.cs_kv_pages_free(tables, bad, ids, ids, stream=0),
                 lambda: cs.cs_kv_pages_free(tables, ids, bad, ids, stream=0),
                 lambda: cs.cs_kv_pages_free(tables, ids, ids, bad, stream=0),
                 lambda: cs.cs_kv_pages_compact(staging, 0, 2, tables, tables, bad, ids, scratch, stream=0),
                 lambda: cs.cs_kv_pages_compact(staging, 0, 2, tables, tables, ids, bad, scratch, stream=0)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(AssertionError):
        cs.PageTables(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32, device="meta"))
    pool = cs.Pool8(torch.zeros(cs.cs_kv8_page_bytes(2, 64) * 3, dtype=torch.uint8), 1, 3, 2, 64)
    b = host_batch([0], [5])
    good = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    wider = torch.zeros((5, 6, 64), dtype=torch.bfloat16)
    for rows in (wider[:, :2], good[:4]):
        for f16 in ("", "_f16"):
            append, attend = getattr(cs, "cs_kv8_append" + f16), getattr(cs, "cs_paged_attention_mixed_kv8" + f16)
            for k, v in ((rows, good), (good, rows)):
                with pytest.raises(AssertionError):
                    append(pool, 0, b, k, v, stream=0)
                with pytest.raises(AssertionError):
                    attend(pool, 0, b, k, v, 2, 0.125, None, stream=0)
    with pytest.raises(AssertionError):
        cs.Pool8(torch.zeros((3, 2 * cs.cs_kv8_page_bytes(2, 64)), dtype=torch.uint8)[:, ::2], 1, 3, 2, 64)


#: Query heads, kv heads, (decodes, their shortest and longest context), chunks as (context, tokens), and what a chip of 256 CUs does
#: with them: the arrangement (0 two kernels, 1 decode behind the tiles, 2 beside) and the ranges of the longest cut tile.
ARRANGED = [
    (28, 4, (64, 1024, 8192), [(3276, 512), (9712, 512), (10901, 512), (6220, 512)], (1, 1)),     # whole, though a grid of their own would cut them
    (40, 8, (10, 239, 956), [(6461, 576), (768, 861), (232, 761), (3545, 984)], (0, 1)),
    (64, 8, (60, 500, 2000), [(3000, 300)], (1, 4)),
    (64, 8, (128, 2048, 32768), [(30720, 1024)], (2, 3)),
    (32, 8, (200, 1000, 6000), [(4000, 200)], (1, 1)),
]


def arranged_batch(decodes, chunks):
    r = np.random.default_rng(40)
    n, lo, hi = decodes
    return [int(x) for x in r.integers(lo, hi, n)] + [c for c, _ in chunks], [1] * n + [q for _, q in chunks]


@pytest.mark.parametrize("Hq,Hkv,decodes,chunks,want", ARRANGED)
def test_arrangements_of_8_bit_mixes(Hq, Hkv, decodes, chunks, want):
    b = host_batch(*arranged_batch(decodes, chunks))
    try:
        cs.cs_debug_set_cu_count(256)
        assert cs.cs_debug_mixed_kv8(b, Hq, Hkv, 128) == want
        for mode, forced in ((0, 0), (2, 1), (3, 2)):
            cs.cs_set_mixed_fusion(mode)
            assert cs.cs_debug_mixed_kv8(b, Hq, Hkv, 128)[0] == forced
    finally:
        cs.cs_set_mixed_fusion(1)
        cs.cs_debug_set_cu_count(0)
    with pytest.raises(cs.CsError):
        cs.cs_debug_mixed_kv8(b, Hq, 3, 128)
    assert cs.lib().cs_debug_mixed_kv8(ctypes.byref(b.c), Hq, Hkv, 128, None) in (0, 1, 2)
