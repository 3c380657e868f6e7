"""The sine and cosine of a rotation, read off vectors (1, 0), to fp32's relative precision."""
import math

import numpy as np
import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("reach", [100, 2 ** 20, 2 ** 30])
@pytest.mark.parametrize("inverse", [False, True])
def test_sine_and_cosine(layout, reach, inverse):
    dim, tokens = 128, 700
    freq = fdb.fd_rope_frequencies(dim)[0]
    coords = torch.randint(-reach, reach, (tokens,), generator=torch.Generator().manual_seed(reach), dtype=torch.int32)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if layout == "interleaved" else (slice(0, 64), slice(64, 128))
    x = torch.zeros(tokens, 1, dim)
    x[..., first] = 1.0
    got = fdb.Rope(freq, layout=layout, inverse=inverse)(x.cuda(), coords.cuda())[:, 0].cpu().double().numpy()
    angle = coords.double().numpy()[:, None] * freq
    sign = -1.0 if inverse else 1.0
    for part, want in ((first, np.cos(angle)), (second, sign * np.sin(angle))):
        # one step of the function (2^-23 of its value), half a step each of the angle's correction, whose square is
        # below 2^-45, and of its own rounding; the angle in 64 bits: three roundings here and one in the reference
        tol = np.abs(want) * 4 * 2.0 ** -24 + 2.0 ** -45 + np.abs(angle) * 4 * 2.0 ** -53
        assert (np.abs(got[:, part] - want) <= tol).all()
