"""Cosines and sines at far positions against angles of 60 digits."""
from decimal import Decimal, getcontext

import pytest
import torch

from paper_2502_06888_amd import rope_binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494")


def angles(positions, cfg):
    """Angles in (-pi, pi], exact but for their own rounding to 64 bits."""
    rot, theta, factor = cfg["rot_dim"], Decimal(cfg["theta"]), Decimal(cfg.get("factor", 1.0))
    rows = []
    w = [(theta ** (Decimal(-2 * i) / rot)) / factor / (2 * PI) for i in range(rot // 2)]
    for p in positions:
        turns = [v * p for v in w]
        rows.append([float((t - t.to_integral_value()) * 2 * PI) for t in turns])
    return torch.tensor(rows, dtype=torch.float64)


@pytest.mark.parametrize("cfg", [dict(rot_dim=64, theta=10000.0), dict(rot_dim=128, theta=500000.0, factor=4.0), dict(rot_dim=10, theta=1.0), dict(rot_dim=32, theta=1.5)])
def test_far_positions(cfg):
    g = torch.Generator().manual_seed(1)
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1] + [int(p) for p in torch.randint(2 ** 30, 2 ** 31, (150,), generator=g)]
    pos += [-int(p) for p in torch.randint(2 ** 27, 2 ** 31, (50,), generator=g)] + [int(p) for p in torch.randint(0, 2 ** 20, (50,), generator=g)]
    half = cfg["rot_dim"] // 2
    x = torch.zeros((len(pos), 1, 2 * half), dtype=torch.float32, device=DEV)
    x[..., :half] = 1                                                         # becomes the cosines, then the sines
    P.rotate(P.Rope(**cfg), torch.tensor(pos, dtype=torch.int32, device=DEV), x)
    got, a = x.cpu().double()[:, 0], angles(pos, cfg)
    # The angle: 2^-25 of a quarter turn.  Each function: two steps of 32 bits, those of numbers up to 1; products with 1 and 0 are exact.
    tol = 2.0 ** -25 * float(PI) / 2 + 2 * 2.0 ** -24
    for name, part, f in (("cosine", got[:, :half], torch.cos(a)), ("sine", got[:, half:], torch.sin(a))):
        err = (part - f).abs()
        at = (err == err.max()).nonzero()[0].tolist()
        assert err.max() <= tol, f"{name} off by {err.max():.3e} of {tol:.3e} at position {pos[at[0]]}, pair {at[1]}"
