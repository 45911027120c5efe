"""The 4-bit decode over batches of 129 to 256 (sequence, kv head) pairs, on the GPU:
attention within the bound that q4_ref.attend derives."""
import numpy as np
import pytest

from tests.test_gpu_cache4 import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hkv,G,Dh,k,W", [
    (17, 8, 4, 128, 200, 700), (43, 3, 1, 64, 64, 400), (19, 8, 8, 128, 40, 410), (20, 7, 2, 64, 0, 1000), (130, 1, 4, 256, 300, 1900),
    (17, 8, 8, 256, 90, 1500), (33, 4, 1, 256, 100, 290), (27, 8, 2, 128, 33, 1200), (28, 8, 2, 128, 33, 1300),
])
def test_attend_batches_too_large_to_split(B, Hkv, G, Dh, k, W):
    rng = np.random.default_rng(B * Hkv + Dh)
    counts = [int(x) for x in rng.integers(0, 2 * W, B)]
    attend(rng, B, Hkv * G, Hkv, Dh, k, W, counts, [int(x) for x in rng.integers(0, k + 1, B)])
