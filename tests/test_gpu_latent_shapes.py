"""Attention over latent rows with four row groups a workgroup, which large caches take and small ones do not: the tests of the other
shape once more, with room for half a million rows a sequence, and calls on both sides of the rule that chooses."""
import functools

import pytest

import test_gpu_latent_attn as narrow

pytestmark = pytest.mark.gpu


@pytest.fixture
def wide(monkeypatch):
    monkeypatch.setattr(narrow, "Case", functools.partial(narrow.Case, max_pages=16384))


@pytest.mark.parametrize("D", [576, 288])
@pytest.mark.parametrize("Hq", [17, 20, 32, 33, 40, 64, 65, 127, 128])
def test_heads(wide, D, Hq):
    narrow.test_heads(D, Hq)


@pytest.mark.parametrize("D", [576, 288])
@pytest.mark.parametrize("n", [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 4097, 20011])
def test_lengths(wide, D, n):
    narrow.test_lengths(D, n)


@pytest.mark.parametrize("B,Hq,D,page,lens,W,n_new", [
    (4, 16, 576, 32, [40, 5, 64, 700], 4, [1, 4, 0, 3]),
    (3, 5, 288, 64, [33, 3, 1], 7, [7, 3, 1]),
    (2, 128, 576, 128, [300, 129], 2, [2, 1]),
    (3, 20, 576, 32, [10, 0, 1000], 16, [16, 4, 9]),
    (1, 1, 288, 32, [90], 70, None),
    (2, 40, 288, 256, [2000, 513], 5, [5, 2]),
    (1, 8, 576, 32, [1200], 1024, None),
])
def test_several_new_tokens(wide, B, Hq, D, page, lens, W, n_new):
    narrow.test_several_new_tokens(B, Hq, D, page, lens, W, n_new)


@pytest.mark.parametrize("Hq,D", [(32, 576), (128, 576), (40, 288)])
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_reach_who_sees_them(wide, Hq, D, odd):
    narrow.test_values_that_are_not_finite_reach_who_sees_them(Hq, D, odd)


@pytest.mark.parametrize("Hq,D", [(128, 576), (32, 288)])
def test_large_and_rising_scores(wide, Hq, D):
    narrow.test_large_and_rising_scores(Hq, D)


def test_another_stream_and_a_graph_that_is_replayed(wide):
    narrow.test_another_stream_and_a_graph_that_is_replayed()


def test_the_same_bits_again(wide):
    narrow.test_the_same_bits_again()


@pytest.mark.parametrize("D,B,Hq,n,hint", [(576, 10, 64, 4096, 4096), (576, 10, 64, 4097, 4097), (288, 64, 40, 900, 800), (288, 64, 40, 900, 1000),
                                           (576, 128, 17, 640, 640), (576, 128, 17, 641, 641)])
def test_both_sides_of_the_rule(D, B, Hq, n, hint):
    lens = [n - 7 * (i % 11) for i in range(B)]
    c = narrow.Case(n, B, Hq, D, 32, lens)
    c.check(*c.run(hint=hint))
