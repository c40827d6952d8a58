"""The 4-bit cache at the lower end of bf16: subnormal numbers and the smallest normal ones, where the scale can go no lower."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64, say
from synth_inputs import bf16_bits_to_f64
from test_gpu_kv4 import rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


@pytest.mark.parametrize("largest", [0x0001, 0x003f, 0x007f, 0x0080, 0x00ff, 0x0100, 0x0180, 0x01df, 0x01e0, 0x025f, 0x0260, 0x02ff, 0x0360])
def test_smallest_numbers(sp, largest):
    """Every bf16 number up to `largest`, of either sign, in groups with `largest`."""
    say("kv4 small values up to %#x" % largest)
    bits = np.arange(largest + 1, dtype=np.uint16)
    bits = np.concatenate([bits, bits | 0x8000])
    bits = np.concatenate([bits, np.zeros(-len(bits) % 31, np.uint16)]).reshape(-1, 31)
    bits = np.concatenate([bits, np.full((len(bits), 1), largest, np.uint16)], 1)
    bits = np.concatenate([bits, np.zeros((-len(bits) % 4, 32), np.uint16)]).reshape(1, -1, 1, 128)
    n = bits.shape[1]
    cache = sp.KvCache4.empty(1, n, 1, 128)
    sp.slimpipe_attn_kv4_store(dev_bf16(bits), dev_bf16(bits ^ 0x8000), cache, 0)
    want, scales = rounded(bf16_bits_to_f64(bits))
    assert np.array_equal(cache.k_scales.cpu().numpy(), scales)
    k, v = sp.slimpipe_attn_kv4_load(cache, 0, n)
    assert np.array_equal(host_f64(k), want) and np.array_equal(host_f64(v), -want)
