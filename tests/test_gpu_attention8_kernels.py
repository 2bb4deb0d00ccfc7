"""Every kernel of the attention on every kind of call, whatever the rule would choose."""
import pytest
import torch

import layer_ref as r
import test_gpu_attention8 as t
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1], ids=["few", "many"])
def kernel(request):
    layer._load().ccq_attention_force(request.param)
    yield
    layer._load().ccq_attention_force(-1)


@pytest.mark.parametrize("pairs,P,D,Hkv,Hq,window,causal", [
    ([(1, 1)], 16, 64, 1, 1, 0, True), ([(1, 200), (1, 3), (1, 0), (1, 130)], 32, 128, 2, 14, 0, True), ([(1, 3000)], 64, 128, 1, 8, 0, True),
    ([(3, 70), (5, 5), (1, 40), (0, 9)], 16, 128, 2, 6, 0, True), ([(33, 33), (17, 100)], 32, 64, 2, 2, 20, True), ([(70, 70)], 64, 128, 1, 7, 0, True),
    ([(130, 400), (9, 900)], 64, 128, 1, 4, 100, True), ([(200, 333)], 128, 64, 2, 4, 0, False), ([(270, 300)], 16, 128, 1, 1, 0, True), ([(60, 700)], 256, 64, 1, 5, 64, True),
])
def test_call(kernel, pairs, P, D, Hkv, Hq, window, causal):
    t._run(pairs, P, D, Hkv, Hq, window, causal, seed=P + Hq)


@pytest.mark.parametrize("pairs", [[(1, 600)], [(40, 300)]])
def test_scales_far_apart_and_peaks(kernel, pairs):
    t.test_scales_far_apart(pairs, 3)
    t.test_peaked_rows(pairs, 2)


def test_pages_that_are_not_there(kernel):
    t.test_pages_that_are_not_there([(20, 200), (8, 90)])


def test_nan(kernel):
    t.test_nan_in_queries_and_keys_reach_the_rows_that_see_them()


def test_bounds(kernel):
    t.test_lengths_past_the_bounds_and_the_table()


def test_more_rows_than_a_tile_in_splits(kernel):
    """Few sequences and long: the cached tokens are cut, rows of several tiles."""
    t._run([(45, 5000)], 64, 128, 1, 2, seed=3)
