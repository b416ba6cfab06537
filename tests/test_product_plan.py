"""How the products of the residual-block operators are cut up (lipz_test_product_plan; host only)."""
import random

import pytest

import paper_1811_12843_amd as L

KIND = {"f32": L.LIPZ_F32, "bf16": L.LIPZ_BF16, "f16": L.LIPZ_F16, "fp8": L.LIPZ_FP8}


def covered(n, tile):
    return -(-n // tile) * tile


@pytest.mark.parametrize("kind", sorted(KIND))
def test_tiles_are_not_mostly_padding(kind):
    """A larger tile may cover more than 64 x 64 ones do by what it saves on the same outputs (16 x 2.75 / 24 with 16 bits,
    4 x 7.85 / 33.3 in fp32, 4 x 4.05 / 14.7 with e4m3), a tenth, and an eighth for the rounding to whole waves of 256 tiles
    where there are more than eight."""
    most = 1.1 * 1.125 * {"f32": 4 * 7.85 / 33.3, "fp8": 4 * 4.05 / 14.7}.get(kind, 16 * 2.75 / 24)
    rng = random.Random(5)
    sizes = [(10, 2048, 512, 32), (8, 65536, 2048, 1), (8, 512, 512, 64), (300, 260, 1032, 48), (64, 4096, 1024, 16)]
    while len(sizes) < 3000:
        m, n, k = (int(2 ** rng.uniform(0, 13.5)) for _ in range(3))
        cells = int(2 ** rng.uniform(0, 7))
        if m * n * cells < 1 << 28:
            sizes.append((m, n, k, cells))
    for m, n, k, cells in sizes:
        tile, splits = L.lipz_test_product_plan(KIND[kind], m, n, k, cells)
        assert tile in (64, 128, 256) and splits >= 1 and (tile == 64 or splits == 1)
        if covered(m, 64) * covered(n, 64) * cells > 8 * 256 * 4096:
            assert covered(m, tile) * covered(n, tile) <= most * covered(m, 64) * covered(n, 64), (m, n, k, cells)
    for m, n, k, cells in sizes[:5]:  # few rows, or a little over a tile
        assert L.lipz_test_product_plan(KIND[kind], m, n, k, cells)[0] == 64, (m, n, k, cells)


def test_large_products_take_large_tiles():
    for kind in ("bf16", "f16"):
        assert L.lipz_test_product_plan(KIND[kind], 8192, 8192, 4096)[0] == 256
        assert L.lipz_test_product_plan(KIND[kind], 1000, 4096, 4096)[0] == 128
    assert L.lipz_test_product_plan(KIND["f32"], 1000, 4096, 4096)[0] == 128
    assert L.lipz_test_product_plan(KIND["fp8"], 8192, 4096, 8192)[0] == 128


def test_few_outputs_split_long_sums():
    for kind in KIND.values():
        tile, splits = L.lipz_test_product_plan(kind, 1, 4096, 4096)
        assert tile == 64 and splits > 1
        assert L.lipz_test_product_plan(kind, 1, 64, 1)[1] == 1


def test_refused_sizes():
    for bad in ((4, 1, 1, 1, 1), (0, 0, 1, 1, 1), (0, 1, 0, 1, 1), (0, 1, 1, 0, 1), (0, 1, 1, 1, 0), (0, 1 << 21, 1 << 20, 1, 1)):
        with pytest.raises(L.LipzError):
            L.lipz_test_product_plan(*bad)


def test_grids_stay_below_2_to_the_32_threads():
    """The most outputs that the calls take: 2^24 blocks of 64 x 64, a workgroup of 256 threads each."""
    for kind in sorted(KIND):
        for m, n, cells in ((1 << 21, 512, 64), (64, 1 << 20, 1024), (1, 64, 65535), (1 << 20, 64, 1024)):
            for k in (1, 4096):
                tile, splits = L.lipz_test_product_plan(KIND[kind], m, n, k, cells)
                assert (covered(m, tile) // tile) * (covered(n, tile) // tile) * cells * splits * (512 if tile == 256 else 256) < 1 << 32
