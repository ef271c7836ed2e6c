"""Clipping where the factor leaves fp32's numbers, against the oracle in 64
bits (u = 2^-24).  An entry is rounded with the factor (u), in the product (u),
to its type, and by half its type's smallest number below its normal ones (a
factor that is itself below them has lost at most 2^-150 of entries up to 2^128,
less than that)."""
import numpy as np
import pytest

import oracle.ends_oracle as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"fp32": (torch.float32, 0.0, 2.0 ** -149), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133), "fp16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_norm", [1e-29, 1e-31, 1e-38, 1e-45, 1e-60, 1e-75, 1e-80, 1e-84, 1e-90, 1e-92, 1e-100, 1e-200, 1e-300, 5e-324])
@pytest.mark.parametrize("largest", [1.0, 3e38])
def test_norms_far_below(dtype, max_norm, largest):
    from paper_2607_13511_amd import binding
    t, e, tiny = TYPES[dtype]
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.uniform(0.25, 1.0, 3001) * min(largest, float(torch.finfo(t).max))).to(t).cuda()
    norm, (want,) = ref.clip([x.double().cpu().numpy()], max_norm)
    apart = torch.full_like(x, 3.0)
    got = binding.clip_gradients([x], max_norm, out=[apart])
    assert abs(got.item() - norm) <= 2 * U * norm or norm > 3.4e38
    binding.clip_gradients([x], max_norm)
    for clipped in (x, apart):
        assert (np.abs(clipped.double().cpu().numpy() - want) <= (2 * U + e) * np.abs(want) * (1 + 4 * U) + tiny).all()
