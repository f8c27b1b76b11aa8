"""Scalars that fp32 does not hold are refused on the host, before anything is launched (no GPU needed; the pointers are never
dereferenced): the kernels work with them in fp32, where they would be 0 or an infinity and make every value NaN."""
import pytest

from test_training_step_abi import adamw, back, norm, refused


@pytest.mark.parametrize("kw,word", [
    (dict(eps=1e-46), "eps"), (dict(eps=1e-39), "eps"), (dict(eps=1e39), "eps"),
    (dict(lr=1e39), "lr"), (dict(lr=1e38, beta1=0.999), "lr"),                        # lr / (1 - beta1) = 1e41
    (dict(lr=1e20, decay=1e20), "decay"), (dict(decay=1e300), "decay")])
def test_adamw_scalars_beyond_fp32(kw, word):
    refused(adamw(**kw), word)


@pytest.mark.parametrize("call", [norm, back])
@pytest.mark.parametrize("eps", [float("inf"), 1e39])
def test_layer_norm_eps_beyond_fp32(call, eps):
    refused(call(eps=eps), "eps")
