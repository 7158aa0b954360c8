"""Stages that keep their saved aggregations in 8 bits where the aggregation's own rows are borrowed from the weight gradients' rows: no gradient of the
input, or layers whose other gradient rows are narrower."""
from __future__ import annotations

import pytest

from synth.configs import Workload
from test_gpu_save8_train import save8, test_nothing_but_weight_gradients_changes as nothing_but_weight_gradients_changes  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("need_input_grad", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("variant,dims,K", [("gcn", [128, 128], 4), ("gcn", [64, 256], 1), ("gcn", [100, 256, 46], 4), ("sage", [64, 100, 100], 3), ("gcn", [32, 64, 128, 128], 4)])
def test_rows_borrowed_from_the_weight_gradients(variant, dims, K, dtype, need_input_grad, save8):  # noqa: F811
    w = Workload(f"s8_room_{variant}_{len(dims)}_{dims[0]}", "er", 700, 31, dims, K, dtype=dtype, variant=variant, avg_degree=8.0)
    nothing_but_weight_gradients_changes(w, need_input_grad, save8)
