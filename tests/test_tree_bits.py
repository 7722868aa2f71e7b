"""The limits of tree_bits separate a tree attention that keeps the second part of keys and queries from one that loses it,
negates it or meets it with the wrong feature (a model of each on the CPU)."""
import numpy as np
import pytest

pytest.importorskip("torch")

import tree_bits as tb
from verify_units import Units


@pytest.mark.parametrize("base", [500000.0, 0.0])
def test_the_limit_separates(base):
    units, rng = Units(tb.ROWS, tb.TOKENS, 50, device="cpu"), np.random.default_rng(50)
    for u in range(len(tb.ROWS)):
        q = tb.large_queries(units, u, 60, base, rng)
        assert np.isfinite(q).all()
        ref = tb.attended(units, u, tb.logits(units, u, q, base, "exact"))
        err = {f: tb.rms(tb.attended(units, u, tb.logits(units, u, q, base, f)) - ref) for f in ("first", "both", "negated", "shuffled")}
        limit = tb.LIMIT[bool(base)] * err["first"]
        assert err["both"] <= (0.35 if base else 0.02) * err["first"], (u, err)
        assert min(err["negated"], err["shuffled"]) > limit and err["first"] > limit
        assert limit > 2 * tb.other_roundings(units, u, tb.logits(units, u, q, base, "exact")), (u, err)
