import numpy as np
import torch

import norm_reference
from oracle import mx


def test_the_reference_of_large_norms_is_the_oracle():
    g = np.random.Generator(np.random.PCG64(4))
    h, gy, w = g.standard_normal((7, 45)), g.standard_normal((7, 45)), g.standard_normal(45)
    t = [torch.from_numpy(a) for a in (h, gy, w)]
    y, rstd = norm_reference.norm(t[0], t[2], 1e-3, 0.5)
    oy, orstd = mx.rms_norm(h, w, 1e-3, 0.5)
    gh, near, far, gw, size = norm_reference.gradients(t[1], t[0], rstd, t[2], 0.5)
    ogh, ogw = mx.rms_norm_grad(gy, h, orstd, w, 0.5)
    for a, b in ((y, oy), (rstd, orstd), (gh, ogh), (gw, ogw)):
        assert np.allclose(a.numpy(), b, rtol=1e-13, atol=1e-13)
    assert bool((near + far >= gh.abs() * (1 - 1e-12)).all()) and bool((size >= gw.abs() * (1 - 1e-12)).all())
