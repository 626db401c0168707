"""The head store refuses caches of keys and values that share a place, and no
others, without a GPU: pairs that are apart are told by another refusal."""
import ctypes
import itertools

import numpy as np
import pytest

from paper_2606_29982_amd import caee

FAKE = 1 << 40           # aligned, never dereferenced
BASE = dict(T=4, heads=2, kv_heads=2, dim=64, rope=0, adjacent=0, x_dtype=caee.CAEE_BF16, block_size=3, n_blocks=3, eps=1e-6,
            q_stride=128, k_stride=128, v_stride=128, q_out_stride=128)


def _refusal(strides, apart, **kw):
    """What a call says of caches that are `apart` elements from each other; its q_out reaches into its keys, so that it
    is refused in any case."""
    d = caee.HeadStoreDesc(**dict(BASE, **dict(zip(("page_stride", "row_stride", "head_stride"), strides)), **kw))
    q, k, v = FAKE, FAKE + (1 << 20), FAKE + (2 << 20)
    at = FAKE + (1 << 30)
    assert caee.lib.caee_head_store(ctypes.byref(d), q, k, v, None, None, None, None, FAKE, k + 16, at, at + 2 * apart,
                                    None) == caee.CAEE_ERR_INVALID_ARG
    return caee.lib.caee_last_error().decode()


def _places(strides, n_blocks, block, heads, dim):
    p, r, h = (np.arange(n) * s for n, s in zip((n_blocks, block, heads), strides))
    return set((p[:, None, None, None] + r[:, None, None] + h[:, None] + np.arange(dim)).ravel().tolist())


@pytest.mark.parametrize("n_blocks,block,heads", [(3, 3, 2), (1, 3, 2), (3, 1, 2), (3, 3, 1), (1, 1, 1)])
@pytest.mark.parametrize("strides", [
    (384, 128, 64),          # by token, dense
    (384, 64, 192),          # by head, dense
    (768, 128, 64),          # halves of one array: 384 apart
    (1024, 200, 96),         # gaps everywhere
    (1600, 96, 512),
    (1152, 384, 192),        # a row holds the keys' heads, the values' and something else
])
def test_caches_that_share_a_place(strides, n_blocks, block, heads):
    size = dict(n_blocks=n_blocks, block_size=block, kv_heads=heads, k_stride=64 * heads, v_stride=64 * heads)
    own = _places(strides, n_blocks, block, heads, 64)
    aparts = sorted(set(itertools.chain(range(-400, 401, 8), range(-2 * strides[0], 2 * strides[0] + 1, 64),
                                        (k * s + e for s in strides for k in range(-3, 4) for e in (-64, -56, 0, 56, 64)))))
    for apart in aparts:
        meet = any(x + apart in own for x in own)
        said = _refusal(strides, apart, **size)
        assert ("k_cache and v_cache overlap" in said) == meet, (apart, said)
        assert meet or "q_out overlaps k" in said
