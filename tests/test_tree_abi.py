"""Host-only checks of the tree attention entry point: refusals before any launch, legal no-ops, workspace sizes."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2608_14498_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14498_b200 import build

    build.build()
    return B.load_library()


GOOD = B.AttnDesc(4, 2, 128, 0.0, B.RPX_BF16)
CACHE = B.KvCache(0x1000, 0x1000, 8, 16, 0x1000, 4)


def call(lib, desc=GOOD, q=0x1000, k=0x1000, v=0x1000, strides=(512, 256, 256), cu=0x1000, parents=0x1000, lens=0x1000,
         batch=1, total=16, max_tree=16, max_cached=64, cache=CACHE, out=0x1000, ws=0x1000, ws_bytes=1 << 30):
    return lib.rpx_tree_attn(ctypes.byref(desc) if desc is not None else None, q, k, v, *strides, cu, parents, lens, batch,
                             total, max_tree, max_cached, ctypes.byref(cache) if cache is not None else None, out, None, ws,
                             ws_bytes, None, None)


def test_refusals(lib):
    assert call(lib, desc=None) == -1
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(parents=None), dict(lens=None), dict(out=None),
                dict(cache=None), dict(cache=B.KvCache(None, 0x1000, 8, 16, 0x1000, 4))):
        assert call(lib, **bad) == -1, bad
    for bad in (dict(desc=B.AttnDesc(4, 3, 128, 0.0, 0)), dict(desc=B.AttnDesc(4, 2, 80, 0.0, 0)), dict(total=-1),
                dict(batch=-1), dict(max_tree=-1), dict(max_tree=B.TREE_MAX_NODES + 1), dict(strides=(256, 256, 256)),
                dict(cache=B.KvCache(0x1000, 0x1000, 8, 32, 0x1000, 4))):
        assert call(lib, **bad) == -2, bad
    # more than 128 query heads per KV head: only small trees
    assert call(lib, desc=B.AttnDesc(160, 1, 64, 0.0, 0), strides=(160 * 64, 64, 64), max_tree=129) == -2
    assert call(lib, desc=B.AttnDesc(4, 2, 128, 0.0, 9)) == -3
    for bad in (dict(q=0x1008), dict(out=0x1004), dict(strides=(516, 256, 256)), dict(ws=0x1010)):
        assert call(lib, **bad) == -4, bad
    assert call(lib, ws=None) == -5
    assert call(lib, ws_bytes=64) == -5
    # nothing to do
    assert call(lib, batch=0, q=None, lens=None, ws=None) == 0
    assert call(lib, total=0, q=None, ws=None) == 0
    assert call(lib, max_tree=0, q=None, ws=None) == 0


def test_workspace_sizes(lib):
    small = B.tree_attn_workspace_bytes(28, 4, 128, B.RPX_BF16, 64, 8, 8)
    assert 0 < small < 32 << 20 and small % 256 == 0
    # 8 x 200 nodes in two-tile blocks: 9 first units, 148 pieces of 2 x 256 rows with (maximum, sum) and 128 floats each, then
    # ancestor sets of 8 words and a copy of the values (8 rows more a sequence)
    wide = B.tree_attn_workspace_bytes(28, 4, 128, B.RPX_BF16, 8 * 200, 8, 200)
    assert wide == 256 + 148 * 512 * 8 + 148 * 512 * 128 * 4 + 1600 * 8 * 4 + (1600 + 64) * 4 * 128 * 2
    # 16 nodes of 5 heads fit one 128-row tile
    one = B.tree_attn_workspace_bytes(40, 8, 128, B.RPX_BF16, 16, 1, 16)
    assert one == 256 + 148 * 256 * 8 + 148 * 256 * 128 * 4 + 16 * 4 * 4 + (16 + 8) * 8 * 128 * 2
    f32 = B.tree_attn_workspace_bytes(4, 2, 64, B.RPX_F32, 10, 2, 5)
    assert f32 == 256 + 256  # the attention call's piece, and 10 sets of 4 words
    assert B.tree_attn_workspace_bytes(28, 4, 128, B.RPX_BF16, 0, 8, 8) == 0


def test_a_size_query_ends_no_process(lib):
    """Fewer query heads than KV heads and a tree for the tensor-core form: a division by zero once, so in a child."""
    code = "import sys; from paper_2608_14498_b200 import binding as B; " \
           "sys.exit(B.tree_attn_workspace_bytes(4, 8, 128, 0, 200, 1, 200) != 0)"
    assert subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(B.__file__)), timeout=120).returncode == 0


@pytest.mark.parametrize("heads", [(4, 8), (4, 3), (0, 1), (1, 0), (-4, 2), (4, -2), (0, 0)])
@pytest.mark.parametrize("max_tree", [1, 8, 129, 200, 1024])
def test_sizes_for_heads_that_are_refused(lib, heads, max_tree):
    """The size query answers 0 where the call refuses, for whoever asks for the size first."""
    assert B.tree_attn_workspace_bytes(*heads, 128, B.RPX_BF16, 200, 1, max_tree) == 0
    assert B.tree_attn_workspace_bytes(*heads, 128, B.RPX_F32, 200, 1, max_tree) == 0
    assert call(lib, desc=B.AttnDesc(*heads, 128, 0.0, B.RPX_BF16), max_tree=max_tree, strides=(1024, 1024, 1024)) == -2


def test_sizes_of_other_refusals(lib):
    assert B.tree_attn_workspace_bytes(4, 2, 80, B.RPX_BF16, 200, 1, 200) == 0
    assert B.tree_attn_workspace_bytes(4, 2, 128, 7, 200, 1, 200) == 0
    assert B.tree_attn_workspace_bytes(4, 2, 128, B.RPX_BF16, 2000, 1, B.TREE_MAX_NODES + 1) == 0
    assert lib.rpx_tree_attn_workspace_bytes(None, 200, 1, 200) == 0


def test_sizes_that_no_launch_holds(lib):
    """Refused on the host, before the launches in front of the one that could not hold them."""
    f32, big = B.AttnDesc(4, 2, 128, 0.0, B.RPX_F32), 1 << 40
    assert call(lib, desc=f32, batch=65536, total=65536, max_tree=1, ws_bytes=big) == -2
    assert call(lib, max_tree=64, cache=B.KvCache(0x1000, 0x1000, 1 << 29, 16, 0x1000, 4)) == -2  # 2^31 groups of eight keys
    assert call(lib, desc=B.AttnDesc(128, 1, 64, 0.0, 0), strides=(128 * 64, 64, 64), batch=1 << 18, total=1 << 20, max_tree=1024,
                ws_bytes=big) == -2
