"""The gated experts' and the head's tests with a comparison that no NaN passes: a result or a bound that is no number fails it."""
import numpy as np
import pytest

import test_gpu_gated_ffn as gated
import test_gpu_head_logprobs as head

pytestmark = pytest.mark.gpu


def near(got, want, what):
    g = gated.f64(got)
    assert g.shape == want.value.shape, what
    assert not np.isnan(want.off).any() and not np.isnan(want.value).any(), (what, "a bound that is no number")
    ok = np.abs(g - want.value) <= want.off + 1e-37
    assert ok.all(), (what, int((~ok).sum()), int(np.isnan(g).sum()), float(np.abs(g - want.value).max()), float(want.off.max()))


@pytest.fixture(autouse=True)
def _strict(monkeypatch):
    monkeypatch.setattr(gated, "near", near)
    monkeypatch.setattr(head, "near", near)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,behind,d,F", gated.CASES)
def test_gated(counts, behind, d, F, dtype, act):
    gated.test_layer_and_gradient(counts, behind, d, F, dtype, act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d,F", [(1, 768, 2048), (33, 200, 104), (600, 136, 72)])
def test_gated_one_block(R, d, F, dtype):
    gated.test_one_block(R, d, F, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d,F", [([1, 2, 0, 1, 3], 200, 3176), ([1, 0, 1], 4104, 136)])
def test_gated_long_sums(counts, d, F, dtype):
    gated.test_few_tiles_of_a_long_sum(counts, d, F, dtype, "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_large_values(dtype):
    gated.test_large_and_special_values(dtype)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V,padded", head.CASES)
def test_head(N, d, V, padded, dtype, bias):
    head.test_scores_and_gradient(N, d, V, padded, dtype, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(5, 400), (90, 400), (300, 400), (12, 9000), (90, 4000), (300, 1500)])
def test_head_masked(N, V, dtype):
    head.test_masked_ids_and_padded_rows(N, V, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(3, 77), (100, 77), (200, 77), (3, 9000), (100, 2000), (200, 1000)])
def test_head_everything_masked(N, V, dtype):
    head.test_everything_masked(N, V, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_equal_weights(dtype):
    head.test_equal_weights_and_no_gradient(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 511, 513])
def test_head_few_rows_of_many_ids(N, dtype):
    head.test_few_rows_of_many_ids(N, dtype)
