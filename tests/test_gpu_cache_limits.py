"""The cache operators at the borders of their forms: page updates on both sides of the one-launch
placement's limits."""
import numpy as np
import pytest

from _gpu import log
from oracle import cache as C
from test_gpu_pages import same, state, update

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


# (rows, table width, pages of the pool): 60 KB of places and starts, 256 workgroups of 1024 entries,
# 1024 rows
BORDERS = [(32, 40, 15328), (32, 40, 15329), (1024, 16, 14336), (1024, 16, 14337), (1024, 256, 9000), (1024, 257, 9000),
           (1025, 16, 9000)]


@pytest.mark.parametrize("rows,m,pages", BORDERS)
def test_update_at_the_borders_of_the_one_launch_placement(lib, rows, m, pages):
    rng = np.random.default_rng(rows + pages)
    table, lens, count = state(rng, 20, 16, m, 240, 0)
    count = np.concatenate([count, np.zeros(pages - len(count), np.int32)])
    parents = rng.integers(-1, 20, rows).astype(np.int32)
    new = (np.where(parents >= 0, lens[np.maximum(parents, 0)], 0) + rng.integers(0, 18, rows)).astype(np.int32)
    log(f"update rows={rows} width={m} pages={pages}")
    same(update(lib, table, lens, parents, new, count, 16), C.pages_update(table, lens, parents, new, count, 16))


def test_update_of_nothing(lib):
    none = np.zeros(0, np.int32)
    got = update(lib, np.zeros((0, 4), np.int32), none, None, none, np.array([0, 2, 0, 1], np.int32), 16)
    assert got[1].tolist() == [0, 2, 0, 1] and got[4].tolist() == [0, 0]
