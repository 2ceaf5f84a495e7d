"""Host-only checks of the page calls: refusals before any launch, legal no-ops, workspace sizes."""
import ctypes

import pytest
import torch

from paper_2608_14498_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14498_b200 import build

    build.build()
    return B.load_library()


def pool(table=0x1000, stride=8, cols=8, rows=4, lens=0x1000, refs=0x1000, nb=64):
    return B.PagePool(table, stride, cols, rows, lens, refs, nb)


def ref(p):
    return ctypes.byref(p) if p is not None else None


BAD_POOLS = [(None, -1), (pool(table=None), -1), (pool(refs=None), -1), (pool(stride=7), -2), (pool(rows=-1), -2),
             (pool(cols=-1), -2), (pool(nb=-1), -2)]


def test_free(lib):
    for p, code in BAD_POOLS + [(pool(lens=None), -1)]:
        assert lib.rpx_pages_free(ref(p), 0x1000, 1, None, None) == code
    assert lib.rpx_pages_free(ref(pool()), None, 1, None, None) == -1
    assert lib.rpx_pages_free(ref(pool()), 0x1000, -1, None, None) == -2
    assert lib.rpx_pages_free(ref(pool()), None, 0, None, None) == 0


def test_fork(lib):
    def call(p=None, src=0x1000, dst=0x1000, n=1, extra=0, cs=0x1000, cd=0x1000, ws=0x1000, ws_bytes=1 << 20, none=False):
        return lib.rpx_pages_fork(None if none else ref(p if p is not None else pool()), src, dst, n, extra, cs, cd, ws, ws_bytes,
                                  None, None)

    assert call(none=True) == -1
    for p, code in BAD_POOLS[1:] + [(pool(lens=None), -1)]:
        assert call(p) == code
    for bad in (dict(src=None), dict(dst=None), dict(cs=None), dict(cd=None)):
        assert call(**bad) == -1
    assert call(n=-1) == -2 and call(extra=-1) == -2
    assert call(ws=None) == -5 and call(ws_bytes=16) == -5 and call(ws=0x1010) == -4
    assert call(n=0, src=None, ws=None) == 0
    p = pool()
    assert lib.rpx_pages_fork_workspace_bytes(ref(p), 10) == 512  # (2 * 10 + 4 + 64 + 1) words, rounded up to 256 bytes
    assert lib.rpx_pages_fork_workspace_bytes(None, 10) == 0


def test_compact(lib):
    def call(p=None, out=0x1000, stride=8, refs=0x1000, cs=0x1000, cd=0x1000, live=0x1000, ws=0x1000, ws_bytes=1 << 20):
        return lib.rpx_pages_compact(ref(p if p is not None else pool()), out, stride, refs, cs, cd, live, ws, ws_bytes, None, None)

    for p, code in BAD_POOLS[1:]:
        assert call(p) == code
    for bad in (dict(out=None), dict(refs=None), dict(cs=None), dict(cd=None), dict(live=None)):
        assert call(**bad) == -1
    assert call(stride=7) == -2 and call(pool(nb=0)) == -2
    assert call(out=pool().block_table, stride=9) == -2  # in place with another stride
    assert call(ws=None) == -5 and call(ws_bytes=16) == -5 and call(ws=0x1040) == -4
    assert lib.rpx_pages_compact_workspace_bytes(ref(pool())) == 512  # 64 places, 1 chunk, 1 count of moves


def test_copy_pages(lib):
    def call(k=0x1000, v=0x1000, layers=1, stride=0, nb=8, hkv=2, d=128, src=0x1000, dst=0x1000, n=1):
        return lib.rpx_cache_copy_pages(k, v, layers, stride, nb, hkv, d, src, dst, n, None, None)

    for bad in (dict(k=None), dict(v=None), dict(src=None), dict(dst=None)):
        assert call(**bad) == -1
    for bad in (dict(layers=-1), dict(nb=-1), dict(n=-1), dict(hkv=0), dict(d=96), dict(layers=2, stride=8 * 2 * 16 * 128 - 8)):
        assert call(**bad) == -2
    for bad in (dict(k=0x1008), dict(layers=2, stride=8 * 2 * 16 * 128 + 4)):
        assert call(**bad) == -4
    assert call(n=0, k=None, src=None) == 0 and call(layers=0, k=None) == 0


def test_append(lib):
    cache = B.KvCache(0x1000, 0x1000, 8, 16, 0x1000, 4)

    def call(k=0x1000, v=0x1000, ks=256, vs=256, total=9, hkv=2, d=128, dtype=0, ids=None, n_ids=0, cu=0x1000, lens=0x1000,
             batch=1, most=4, c=cache):
        return lib.rpx_cache_append(k, v, ks, vs, total, hkv, d, dtype, ids, n_ids, cu, lens, batch, most, ref(c), None, None)

    for bad in (dict(k=None), dict(v=None), dict(cu=None), dict(lens=None), dict(c=None),
                dict(c=B.KvCache(0x1000, 0x1000, 8, 16, None, 4))):
        assert call(**bad) == -1
    for bad in (dict(ks=248), dict(vs=128), dict(total=-1), dict(hkv=0), dict(d=32), dict(batch=-1), dict(most=-1),
                dict(n_ids=-1), dict(c=B.KvCache(0x1000, 0x1000, 8, 8, 0x1000, 4))):
        assert call(**bad) == -2
    assert call(dtype=4) == -3
    for bad in (dict(k=0x1004), dict(ks=260)):
        assert call(**bad) == -4
    assert call(batch=0, k=None) == 0 and call(most=0, cu=None) == 0


def test_status_string():
    assert B.status_string(-10) == "the page pool has too few free pages"


def test_wrapper_checks():
    table, lens, refs = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    p = B._page_pool(table[:, :3], lens, refs)
    assert (p.rows, p.table_cols, p.block_table_stride, p.num_blocks) == (3, 3, 4, 9)
    with pytest.raises(TypeError):
        B._page_pool(table.long(), lens, refs)
    for bad in ((table.t(), lens, refs), (table, lens[:2], refs), (table, lens, refs[::2])):
        with pytest.raises(ValueError):
            B._page_pool(*bad)
    with pytest.raises(TypeError):
        B._row_list(lens.long())
