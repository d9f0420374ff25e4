"""Exact attention of float queries and keys far from 1 whose products are ordinary, against the definition in 64 bits."""
import pytest
import torch

from tests.gpu_harness import DEV
from tests.test_gpu_exact_attention import Problem, dev_ints
from tests.test_gpu_kv_cache import Serving

pytestmark = pytest.mark.gpu


def counted(x):
    """What a tensor of values below 2^-109 counts as: multiples of 2^-133."""
    return (torch.round(x.double() * 2.0 ** 133) * 2.0 ** -133).float()


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("power", [40, 80, 100, 112, 116, 120])
@pytest.mark.parametrize("tiny", ["Q", "K"])
def test_products_of_tiny_and_huge_operands(tiny, power, d):
    """Scores as ever from queries and keys that are 2^power apart from them."""
    p = Problem([60, 9], [60, 300], 4, 2, d, "f32", True)
    down, up = (p.Q, p.K) if tiny == "Q" else (p.K, p.Q)
    down *= 2.0 ** -power
    up *= 2.0 ** power
    p.call()
    if d <= 128 and power > 109:
        setattr(p, tiny, counted(down))
    p.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [80, 100, 112, 116, 120])
@pytest.mark.parametrize("tiny", ["Q", "K"])
def test_some_features_apart(tiny, power, d):
    """One feature tiny in the one and huge in the other, the others 0 in the huge one's rows or ordinary."""
    for zeros in (False, True):
        p = Problem([60, 9], [60, 300], 4, 2, d, "f32", True)
        down, up = (p.Q, p.K) if tiny == "Q" else (p.K, p.Q)
        if zeros:
            up[:, :, :5], up[:, :, 6:] = 0.0, 0.0
        down[:, :, 5] *= 2.0 ** -power
        up[:, :, 5] *= 2.0 ** power
        p.call()
        if power > 109:
            down[:, :, 5] = counted(down[:, :, 5])
        p.check()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("power", [40, 100, 116, 120])
def test_tiny_queries_of_huge_cached_keys(power, d):
    s = Serving(2, 4, 2, d, 64, 6, "f32")
    K, V = s.rows(303, 2), s.rows(303, 2)
    s.store([300, 0], K * 2.0 ** power, V)
    s.lengths[0] += dev_ints([0, 40])
    Q, O, lse, off = s.attend([3, 0], Q=s.rows(6, 4, 2.0) * 2.0 ** -power)
    s.check_attention(s.reference(), counted(Q) if power > 109 else Q, O, lse, off)


@pytest.mark.parametrize("scale", [2.0 ** -90, 2.0 ** 70])
def test_scales_far_from_1(scale):
    """Ordinary scores by a scale far from 1, of keys down to 2^-40 of the largest."""
    p = Problem([60, 9], [60, 300], 4, 2, 64, "f32", True)
    p.Q *= 0.125 / scale
    p.K *= torch.exp2(torch.randint(-40, 1, p.K.shape, device=DEV).float())
    p.scale = scale
    p.call().check()
