"""GPU: routing by scores where 32 bits end: NaN and infinities in rows whose weights are renormalised, logits and biases
far apart, biases whose sums cancel or overflow; against the plain 64-bit forms.  Tolerances are test_gpu_scored's."""
import numpy as np
import pytest

import scoredref
from test_gpu_scored import DEV, _bias, _check, _f64, _logits, _run

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("T", [40, 6400])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_nan_stays_in_renormalised_softmax_weights(T, bad):
    """A softmax over a NaN or plus infinity is NaN throughout, also where that expert is not selected, may not be, or is
    in another group; the rows beside it are as they were."""
    import torch
    z = _logits(T, 32, 60, "float32")
    rows = [1, 2, 3, T - 1]
    for i, t in enumerate(rows):
        z[t, 5 * i + 2] = float(bad)
    clean = [t for t in range(T) if t not in rows]
    b = _bias(32, 60)
    out = b.clone()
    out[[2, 7, 12, 17]] = -INF
    for bias in (None, b, out):
        for groups, top in ((1, 1), (4, 2)):
            idx, w, _ = _run(z, 4, score="softmax", bias=bias, n_groups=groups, top_groups=top, renorm=True)
            assert torch.isnan(w[rows]).all() and (idx[rows] >= 0).all()
            ri, rw, _ = scoredref.route(_f64(z[clean]), 4, "softmax", None if bias is None else _f64(bias), groups, top, 2, True)
            assert np.array_equal(idx.cpu().numpy()[clean], ri)
            np.testing.assert_allclose(_f64(w)[clean], rw, rtol=2.5e-6, atol=1e-30)
