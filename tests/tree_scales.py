"""Units whose steps are scaled, for the tests of tree attention with keys and values of unusual size."""
import numpy as np
import torch

from verify_units import Units


class ScaledUnits(Units):
    """Units with the steps of both sides multiplied by powers of two (keys and values grow by them)."""

    def __init__(self, rows, capacity, seed, k_scale=1.0, v_scale=1.0, **kw):
        super().__init__(rows, capacity, seed, **kw)
        for side, f in ((0, k_scale), (1, v_scale)):
            S = self.sides[side]
            S.delta_h *= np.float32(f)
            S.delta.copy_(torch.as_tensor(S.delta_h))
            self.delta[side][:] = [np.float32(x) for x in S.delta_h]
