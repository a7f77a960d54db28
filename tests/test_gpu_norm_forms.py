"""The three forms of residual + norm + quantizer at the sizes that choose them, bit for bit (the plain evaluation is
that of test_gpu_add_norm)."""
import pytest

from test_gpu_add_norm import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,bias", [("rms", False), ("rms", True), ("layer", False), ("layer", True)])
@pytest.mark.parametrize("res_type", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("K", [8320, 9216])
def test_many_long_tokens(K, res_type, kind, bias):
    """32 elements per thread: more than eight tokens per SM and more than 8192 features."""
    run(1300, K, kind, bias, "bf16" if res_type == "f32" else "f16", res_type, K)


@pytest.mark.parametrize("M,K", [(4001, 1152), (2500, 5120), (1200, 8192), (6007, 640), (1500, 4224)])
@pytest.mark.parametrize("kind,bias,res_type", [("rms", False, "f16"), ("layer", True, "f32"), ("rms", True, "f32"), ("layer", False, "bf16")])
@pytest.mark.parametrize("in_place", [False, True])
def test_several_tokens_per_cta(M, K, kind, bias, res_type, in_place):
    """The pipelined form with several warps and, with up to eight CTAs per SM, three tokens and more per CTA, the last round uneven."""
    run(M, K, kind, bias, "bf16", res_type, M + K, in_place)


@pytest.mark.parametrize("M", [296, 297, 600, 1184, 1185])
def test_at_the_limits_of_the_forms(M):
    run(M, 8320, "layer", True, "bf16", "f32", M)
    run(M, 2048, "rms", False, "f16", "f16", M)
