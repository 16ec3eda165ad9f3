"""Attention over planes that do not fit a block's shared memory, or are too many for it (tensor cores, the FP32 kernel), and over batches of
small planes, whose blocks take several turns of queries.  Formula and tolerances are those of test_gpu_attention."""
import numpy as np
import pytest

import attention_ref as R
import test_gpu_attention as A
from gpu_util import B

pytestmark = pytest.mark.gpu

LONG = [  # N, heads, kv heads, D, query plane, key plane
    (1, 1, 1, 5, (11, 12), (24, 25)), (1, 2, 2, 33, (13, 13), (20, 19)), (2, 4, 2, 40, (19, 19), (19, 19)), (46, 1, 1, 64, (17, 1), (1, 385)),
    (7, 1, 1, 64, (1, 128), (1, 512)), (40, 1, 1, 64, (3, 7), (2, 192)), (3, 2, 1, 128, (12, 11), (13, 16)), (2, 3, 1, 96, (9, 16), (1, 257)),
    (7, 1, 1, 32, (127, 1), (640, 1)), (6, 1, 1, 32, (129, 1), (641, 1)), (1, 1, 1, 1, (5, 5), (1, 700)), (25, 8, 4, 48, (10, 10), (10, 10)),
    (16, 16, 16, 64, (11, 12), (8, 16)), (3, 1, 1, 7, (33, 3), (33, 17)), (40, 4, 2, 128, (9, 9), (9, 9)), (30, 8, 8, 32, (9, 8), (9, 8))]
MANY = [(64, 8, 8, 64, (7, 7), (7, 7)), (200, 2, 2, 16, (8, 8), (8, 8)), (100, 6, 2, 20, (5, 5), (6, 6)), (90, 4, 2, 33, (8, 8), (3, 5)), (2, 1, 1, 128, (40, 40), (9, 7)),
        (1, 1, 1, 32, (17, 1), (1, 500)), (1, 1, 1, 64, (1, 21), (1, 300)), (1, 2, 1, 128, (1, 33), (4, 42)), (70, 3, 3, 3, (2, 9), (1, 2)), (160, 1, 1, 128, (1, 12), (1, 129))]

SPREAD = [  # rows of all heads few, keys many: their blocks share out the keys in every mode
    (1, 1, 1, 32, (5, 10), (60, 61)), (1, 4, 2, 64, (7, 7), (33, 31)), (2, 3, 1, 20, (1, 100), (27, 28)), (1, 1, 1, 128, (1, 700), (1, 190)), (3, 2, 2, 48, (8, 16), (2, 260))]


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("shape", SPREAD)
def test_few_rows_over_many_keys(shape, mode):
    assert B.small_attention_workspace_bytes(*shape, B.MATH[mode]) == 0
    A.test_matches_the_formula(shape, mode)
    A.test_bias_cap_and_padded_images(shape, 3.0, mode)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("shape", LONG + MANY)
def test_matches_the_formula(shape, mode):
    takes = B.small_attention_workspace_bytes(*shape, B.MATH[mode])
    assert (takes > 0) == (shape in LONG and mode != "fp32")    # the tensor cores lay keys and values out once
    A.test_matches_the_formula(shape, mode)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("shape", LONG + MANY)
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_bias_cap_and_padded_images(shape, cap, mode):
    A.test_bias_cap_and_padded_images(shape, cap, mode)


@pytest.mark.parametrize("mode", A.MODES)
def test_infinite_and_lowest_values_in_the_table(mode):
    A.test_infinite_and_lowest_values_in_the_table((24, 25), mode)


@pytest.mark.parametrize("mode", A.MODES)
def test_what_lies_outside_the_extents_has_no_part(mode):
    rng = np.random.default_rng(31)
    plane, ke = (23, 19), np.array([[23, 19], [5, 19], [22, 3], [0, 19], [1, 1]], np.int32)
    q, k, v = A.make(rng, 5, 2, 1, 64, plane, plane)
    ref = R.attention(q, k, v, 2, 1, 0.125, k_extents=ke, q_extents=ke)
    for fill in (np.nan, np.inf, -np.inf, 3e38):
        parts = [t.copy() for t in (q, k, v)]
        for n in range(5):
            for t in parts:
                t[n, :, ke[n, 0]:], t[n, :, :, ke[n, 1]:] = fill, fill
        got = A.run(*parts, 2, 1, mode, ke=ke, qe=ke)
        A.close(got, ref, mode)
        assert (got[3] == 0).all()


@pytest.mark.parametrize("mode", A.MODES)
def test_values_that_are_not_finite_are_not_hidden(mode):
    rng = np.random.default_rng(32)
    q, k, v = A.make(rng, 3, 1, 1, 32, (19, 19), (25, 25))
    ref = R.attention(q, k, v, 1, 1, 32 ** -0.5)
    v[1, 4, 3, 3] = np.nan
    k[2, 0, 24, 24] = np.nan
    got = A.run(q, k, v, 1, 1, mode)
    assert np.isnan(got[1, 4]).all() and np.isnan(got[2]).all()
    got[1, 4], got[2] = ref[1, 4], ref[2]
    A.close(got, ref, mode)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("qs,ks,vs", [(1e4, 1e-4, 1.0), (1e-15, 1e15, 1e20), (1.0, 1.0, 1e-20), (1e-20, 1e19, 1e-30)])
def test_scales_of_the_operands(qs, ks, vs, mode):
    rng = np.random.default_rng(33)
    q, k, v = A.make(rng, 2, 2, 2, 32, (25, 24), (25, 24))
    v[:, :, ::2] *= 1e-3
    q, k, v = (q * qs).astype(np.float32), (k * ks).astype(np.float32), (v * vs).astype(np.float32)
    scale = 1.0 / (32 ** 0.5 * qs * ks)
    A.close(A.run(q, k, v, 2, 2, mode, scale=scale) / vs, R.attention(q, k, v, 2, 2, scale) / vs, mode)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("scale", [0.0, -0.15])
def test_scales_that_are_not_positive(scale, mode):
    rng = np.random.default_rng(34)
    q, k, v = A.make(rng, 2, 2, 1, 40, (19, 19), (19, 19))
    for args in (dict(), dict(bias=A.table(rng, 2, (19, 19), (19, 19))), dict(cap=2.0)):
        A.close(A.run(q, k, v, 2, 1, mode, scale=scale, **args), R.attention(q, k, v, 2, 1, scale, **args), mode)


@pytest.mark.parametrize("mode", A.MODES)
@pytest.mark.parametrize("shape", [(2, 4, 2, 64, (19, 18), (19, 18)), (16, 4, 4, 32, (7, 7), (7, 7))])
def test_repeatable_on_streams_and_in_a_graph(shape, mode):
    A.test_repeatable_on_streams_and_in_a_graph(shape, mode)


@pytest.mark.parametrize("mode", ["3xtf32", "tf32"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_a_cap_without_a_table_over_many_tiles_of_keys(D, mode):
    """The tensor cores' general form without a table: more tiles of 128 keys than places of them are held (8), block after block on each SM."""
    shape = (2, 4, 2, D, (40, 33), (39, 34))
    assert B.small_attention_workspace_bytes(*shape, B.MATH[mode]) > 0
    rng = np.random.default_rng(35)
    q, k, v = A.make(rng, *shape)
    ke = np.array([[39, 34], [30, 33]], np.int32)
    ref = R.attention(q, k, v, 4, 2, D ** -0.5, cap=3.0, k_extents=ke)
    for _ in range(3):
        A.close(A.run(q, k, v, 4, 2, mode, cap=3.0, ke=ke), ref, mode)
