"""The library's two 4-bit quantizers on the same rows: how far each is from the values, and from the other."""
import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _handles, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_both_keep_values_within_half_a_step(dp):  # noqa: F811
    rng = np.random.default_rng(5)
    T, H, D = 700, 2, 128
    x = (rng.standard_normal((T, H, D)) * 2.0 ** rng.uniform(-8, 8, (T, H, 1))).astype(np.float16)
    cu, lens, table, blocks = ref.random_batch(rng, [T], [T], 16)
    c, b = _handles(dp, ref.random_cache(rng, blocks, H, 16, D), cu, lens, table)
    rows, back = torch.from_numpy(x).cuda(), [torch.empty((T, H, D), dtype=torch.float16, device="cuda") for _ in range(2)]
    dp.dptq_kv4_append(c, b, rows, rows)
    dp.dptq_kv4_read(c, b, *back)
    codes, scales = torch.empty((T, H * D // 2), dtype=torch.uint8, device="cuda"), torch.empty((T, H), device="cuda")
    dp.dptq_kv4_quantize(rows.flatten(1), 128, codes, scales)
    one = ref.unpack(codes.cpu().numpy()).reshape(T, H, D) * scales.cpu().numpy().astype(np.float64)[..., None]
    step = np.abs(x.astype(np.float64)).max(axis=2, keepdims=True) / 7
    # half a step, and a unit in the last place of the fp32 scale; half a step of a scale that is up to 2^-8 larger
    assert (np.abs(one - x) <= step / 2 * (1 + 2.0 ** -20)).all()
    for k in back:
        two = k.cpu().numpy().astype(np.float64)
        assert (np.abs(two - x) <= step / 2 * (1 + 2.0 ** -8) * (1 + 2.0 ** -20)).all()
        # of the same rows: errors alike in the mean square, within what scales 2^-8 apart change
        e1, e2 = (np.sqrt(np.mean(((v - x) / step) ** 2)) for v in (one, two))
        assert abs(e2 / e1 - 1) < 2.0 ** -6
    dp.dptq_last_device_error()
