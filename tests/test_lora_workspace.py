"""How much scratch the adapters' calls ask for: nothing for fragments that no kernel of the call reads."""
import os

import pytest

from paper_2508_19373_amd import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B._LIB_PATH):
        import __graft_entry__ as g
        g.build()


def _padded(n):
    return (n + 255) // 256 * 256


def _slices(T, K):
    """Parts of the first product's sum over K."""
    return min(-(-512 // -(-T // 64)), -(-K // 512), 8)


@pytest.mark.parametrize("T,K,N,r,L", [(65, 64, 64, 8, 1), (4096, 4096, 4096, 32, 8), (4_400_001, 8, 8, 8, 3), (300, 520, 264, 64, 9)])
def test_a_forward_that_adds_up_v_itself(T, K, N, r, L):
    """Its products read v's parts, the rows in order and the tiles; no packed fragments of 12 KB for every 64 rows."""
    tiles = T // 64 + min(L + 1, T)
    need = sum(_padded(n) for n in (_slices(T, K) * T * r * 4, (L + 2) * 4, T * 4, tiles * 16))
    assert B.moe_lora_workspace_bytes(T, K, N, r, L) == need


def test_a_forward_of_wide_ranks_packs_them():
    assert B.moe_lora_workspace_bytes(4096, 512, 512, 128, 3) >= 4096 // 64 * 4 * 4 * 3 * 1024
