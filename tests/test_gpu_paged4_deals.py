"""Paged attention where its tiles of 128 rows are cut in each of the ways that there are (paged_deals.py), against the definition in 64 bits."""
import math

import pytest

import paged_deals as deals
from test_gpu_paged import Setup
from test_gpu_paged4 import Setup4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("i", range(len(deals.DEALS)), ids=lambda i: f"{i}_{deals.DEALS[i][5]}")
def test_every_way_to_cut(i, causal):
    d, h_kv, g, lens, news, _ = deals.DEALS[i]
    Setup4(lens, news, h_kv=h_kv, g=g, d=d, page=[16, 64, 256][i % 3], behind=math.nan, spare=i % 2, seed=50 + i).check(causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,news", [([1200], [1200]), ([700, 1100, 20], [700, 650, 2])])
def test_resident_tiles_over_pages_of_bf16(d, causal, lens, news):
    """None is cut; more than one a CU, the later ones taken from the other end."""
    Setup(lens, news, h_kv=32, g=1, d=d, page=64, behind=math.nan, seed=70).check_attend(causal)
