"""Sizes at the ends of what salr_linear_cross_entropy takes: a launch holds fewer than 2^32 threads, and what would need more is refused on the
host with SHAPE, before anything is written.  No GPU needed: where a size is taken, the call stops at its workspace, which is too small."""
import pytest

FAKE = 0x10000   # never dereferenced


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    salr.lib()
    return salr


def _call(salr, T, K, V, dh, dw):
    return salr.lib().salr_linear_cross_entropy(FAKE, T, K, FAKE, V, FAKE, FAKE, FAKE, FAKE, FAKE if dh else None, FAKE if dw else None, FAKE, 0, None)


# tiles of 256 x 256 (128 where that is the tile): 2^23 of them less those that make the grid a multiple of 8 are the most
MOST_TILES = (1 << 23) - 8


@pytest.mark.parametrize("T,K,V,dh,dw,taken", [
    (1 << 20, 8, 256 * 2047, False, False, True),         # 4096 x 2047 tiles
    (1 << 20, 8, 256 * 2048, False, False, False),
    (1, 8, 256 * MOST_TILES, False, False, True),         # one row of tiles
    (1, 8, 256 * MOST_TILES + 1, False, False, False),
    (1, 8, (1 << 31) - 1, False, False, False),
    (1, 8, (1 << 31) - 1, True, False, True),             # pieces of the vocabulary: a launch each
    (1 << 20, 8, 256 * 2048, True, False, True),
    (1 << 20, 8, 256 * 2048, True, True, False),          # (the statistics are one launch)
    (((1 << 22) - 1) * 64, 8, 8, False, False, True),     # rows: 64 a workgroup of 1024 threads
    (((1 << 22) - 1) * 64 + 1, 8, 8, False, False, False),
    (1 << 20, (1 << 15) - 8, 300, True, False, True),     # T K / 8
    (1 << 20, 1 << 15, 300, True, False, False),
    (1 << 20, 1 << 15, 300, False, False, True),
    ((1 << 24) - 1, 8, 256, False, True, True),           # one workgroup a token where the exponentials are held
    (1 << 24, 8, 256, False, True, False),
    (1 << 24, 8, 257, False, True, True),
    (1 << 24, 8, 256, True, False, True),
])
def test_launches_fit(salr, T, K, V, dh, dw, taken):
    assert _call(salr, T, K, V, dh, dw) == (salr.SALR_ERR_CAPACITY if taken else salr.SALR_ERR_SHAPE)
    assert (salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, dh, dw) > 0) == taken


@pytest.mark.parametrize("dh,dw", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("T,K,V", [(1, 4096, 131072), (48, 512, 4099), (64, 8192, 131072), (1111, 2720, 50003), (2000, 2048, 65536), (4096, 4096, 131072),
                                   (16384, 8192, 131072), (524288, 64, 300), (600000, 64, 256), (600000, 64, 5000), (1, 8, 1 << 30)])
def test_workspace_is_what_its_terms_add_up_to(salr, T, K, V, dh, dw):
    """The terms that the header names, each at its most: nothing grows with T * V but the statistics, 8 bytes per token and tile of words."""
    words = (V + 255) // 256 * 256
    cap = max(1, (256 << 20) // (512 * T)) * 256      # words of the largest piece
    one_piece = words <= cap
    need = 32 * T + 8 * T * (min(words, cap) if dh and not dw else words) // (64 if T <= 64 or words <= 96 * 256 else 256)
    if dh or dw:
        need += 2 * T * min(words, cap)
    assert not (dh or dw) or 2 * T * min(words, cap) <= max(256 << 20, 512 * T)
    if dw:
        need += (4 * T * words if one_piece else 0) + 2 * T * K
    if dh:
        need += 4 * T * K * (64 if T <= 64 else 16)
    got = salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, dh, dw)
    assert 0 < got <= need + 9 * 256
    if dw and one_piece:
        assert got >= 6 * T * V
