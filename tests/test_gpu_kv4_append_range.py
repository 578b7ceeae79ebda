"""Appending values near the end of FP16: what is held follows from the smallest value and a fifteenth of the range alone.  Formula: test_gpu_kv4, exact in FP32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_gpu_kv4 import HALF, U, Held, appended, ints


@pytest.mark.parametrize("name,dtype", [("f32", torch.float32), ("bf16", torch.bfloat16)])
def test_values_beyond_fp16(name, dtype):
    rng = np.random.default_rng(3)
    # (smallest, largest, whether what is held is finite: 65520 and more is rounded to an infinity; 65280 is a bf16 value)
    ranges = [(0.0, 70000.0, True), (-60000.0, 900000.0, True), (-65000.0, 917000.0, True), (-70000.0, 0.0, False), (66000.0, 66000.0, False), (0.0, 1e6, False),
              (-65280.0, 65280.0, True), (1e5, 2e5, False), (-1e30, 1e30, False), (-3e38, 3e38, False)]
    held = Held(rng, [16], 1, 64, 16)
    x = torch.from_numpy(np.stack([np.concatenate(([a, b], rng.uniform(a, b, 62))) if b < 1e30 else np.linspace(a / 2, b / 2, 64) * 2 for a, b, _ in ranges])[:, None]).to(dtype)
    out = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    oz.kv4_append(held.cache, x.cuda(), x.cuda(), ints([0, len(ranges)]), held.gpu_table, held.gpu_lengths, held=out)
    c, s, o = appended(x)
    fine = np.isfinite(s) & np.isfinite(o)
    assert fine[:, 0].tolist() == [f for _, _, f in ranges]
    page = held.table[0, 0]
    got = held.cache.k_scales.cpu().numpy()[page, 0, 16 - len(ranges) :]
    assert np.array_equal(got[:, 0][fine[:, 0]], s[fine]) and np.array_equal(got[:, 1][fine[:, 0]], o[fine])
    assert np.array_equal(np.isfinite(got).all(1), fine[:, 0])
    codes = held.cache.k_codes.cpu().numpy()[page, 0, 16 - len(ranges) :]
    assert np.array_equal(codes[fine[:, 0]], (c[:, 0, 0::2] | c[:, 0, 1::2] << 4)[fine[:, 0]])
    value = c * s.astype(np.float64)[..., None] + o.astype(np.float64)[..., None]
    for t in out:
        t = t.double().cpu().numpy()
        assert np.array_equal(np.isfinite(t).all(2)[:, 0], fine[:, 0])
        assert (np.abs(t - value) <= (HALF[name] + 2 * U) * np.abs(value))[fine].all()
