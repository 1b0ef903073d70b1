"""Rotation at positions and frequencies up to the largest that it takes, against angles reduced with 60 digits.

The kernel's fraction of a turn is off by at most 2^-26 + 2^-51 |t f / 2 pi| turns: 32 bits of the fraction, and the
roundings of 2 pi, of the quotient and of the product in 64 bits.  Of a turned value, amplitude 1, that is 2 pi times as
much of |a| + |b|, and 2^-21 of it covers all else (see test_gpu_rope)."""
import decimal
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_31093_amd import pisa

PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494")


@pytest.mark.parametrize("turn", ["fwd", "bwd"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(turn, layout):
    pos = [0, 1, -1, 4096, (1 << 20) + 7, 1 << 24, -(1 << 26) + 3, (1 << 30) - 1, (1 << 31) - 1, -(1 << 31)]
    freq = [1.0, 0.1, 1e-4, 1 / 3, math.pi, 1e6, 999999.3, -2.5, 0.0, 1e-9]
    N, d, rot = len(pos), 64, 2 * len(freq)
    r = pisa.make_rope(1, 1, 1, N, d, rot=rot, layout=layout, dtype="f32")
    for i, f in enumerate(freq):
        r.freq[i] = f
    x = torch.randn((1, 1, N, d), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    fn, sign = (pisa.rope_fwd, 1) if turn == "fwd" else (pisa.rope_bwd, -1)
    y, _ = fn(r, x, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    x, y = x[0, 0].double().cpu().numpy(), y[0, 0].double().cpu().numpy()
    assert np.array_equal(x[:, rot:], y[:, rot:])
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        for n, t in enumerate(pos):
            for i, f in enumerate(freq):
                turns = decimal.Decimal(t) * decimal.Decimal(f) / (2 * PI)
                angle = float((turns - turns.to_integral_value()) * 2 * PI)
                ia, ib = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
                a, b, c, s = x[n, ia], x[n, ib], math.cos(angle), sign * math.sin(angle)
                off = 2.0 ** -26 + 2.0 ** -51 * abs(float(turns))
                tol = (2 * math.pi * off + 2.0 ** -21) * (abs(a) + abs(b))
                assert abs(y[n, ia] - (a * c - b * s)) <= tol and abs(y[n, ib] - (b * c + a * s)) <= tol, (t, f)
