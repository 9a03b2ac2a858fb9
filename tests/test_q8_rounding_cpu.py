"""The judge of key rounding without a GPU: it takes the formula's numbers and plain fp32's, and none
with a little noise."""
import numpy as np
import pytest
import torch

import q8ref as R
import q8rounding as Q


def _inputs(n, d, normed, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((n, d), generator=g) * 2).to(torch.bfloat16)
    w = 1 + 0.3 * torch.randn(d, generator=g) if normed else None
    a = torch.arange(n, dtype=torch.float64)[:, None] * torch.from_numpy(R.theta(d, 1e4))
    return x, w, a.cos(), a.sin()


def test_forms_agree_with_the_other_plain_ones():
    x, w, cos, sin = _inputs(300, 64, True, 1)
    want, _ = Q.turned64(x, w, 1e-6, cos, sin)
    other, _ = R.norm_rotate(R.f64(x)[:, None], R.f64(w), 1e-6, np.arange(300), R.theta(64, 1e4))
    assert np.allclose(want.numpy(), other[:, 0], rtol=1e-12, atol=1e-12)
    num, e = R.quantise(want.numpy())
    p = Q.power(want.abs().amax(-1))
    assert np.array_equal(p.numpy(), 2.0 ** e.astype(np.float64))
    assert np.array_equal(Q.rounded((want / p[:, None]).clamp(-448, 448)).numpy(), num)


@pytest.mark.parametrize("normed", [False, True], ids=["plain", "normed"])
def test_judge(normed):
    bound = Q.NORMED if normed else Q.PLAIN
    x, w, cos, sin = _inputs(16384, 64, normed, 2)
    want, size = Q.turned64(x, w, 1e-6, cos, sin)
    p = Q.power(want.abs().amax(-1))
    assert Q.judged(Q.rounded((want / p[:, None]).clamp(-448, 448)), p, want, size, bound) == (0, 0)
    Q.judged(*Q.quantised32(Q.turned32(x, w, 1e-6, cos, sin)), want, size, bound)
    for noise in (2.0 ** -16, 2.0 ** -13):
        y = want * (1 + noise * torch.randn(want.shape, generator=torch.Generator().manual_seed(3)).double())
        with pytest.raises(AssertionError):
            Q.judged(*Q.quantised32(y.float()), want, size, bound)
