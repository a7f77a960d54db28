"""The many-row form with a window and sinks where items are few and short, or about half as many as workgroups: shared or one to a
workgroup, each is held to binary64."""
import pytest
import torch

from test_gpu_kv_sinks import sinks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [1, 64, 200, 390])
@pytest.mark.parametrize("D,H", [(64, 1), (128, 3)])
def test_few_items(window, D, H):
    sinks([900, 500], [96, 70], 64, 4 * H, H, D, window, 4)


@pytest.mark.parametrize("window", [64, 200, 390])
def test_about_half_as_many_items_as_workgroups(window):
    half = torch.cuda.get_device_properties(0).multi_processor_count // 2
    for heads in (half - 1, half, half + 1):
        sinks([700], [65], 32, heads, heads, 64, window, 4)
