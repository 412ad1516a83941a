"""Frequencies of rotary positions for contexts longer than the trained one (binding.rope_frequencies), against the definition in its docstring.  No GPU."""
import math

import numpy as np
import pytest

from paper_2603_09221_amd import binding


@pytest.mark.parametrize("rot", [16, 64, 128])
@pytest.mark.parametrize("trained", [2048, 4096, 32768, 131072, 1 << 20])
@pytest.mark.parametrize("factor", [4.0, 32.0])
def test_bands_of_frequencies(rot, trained, factor):
    """Pair i turns trained * f_i / 2 pi times within the trained length.  Mixed linearly over the index between those whole indices that enclose
    the range from `fast` to `slow` turns; a slow end that lies behind the last pair leaves that one mixed."""
    plain = binding.rope_frequencies(rot)[0].numpy()
    got, scale = binding.rope_frequencies(rot, scaling="bands", factor=factor, trained=trained)
    assert scale == pytest.approx(0.1 * math.log(factor) + 1.0, rel=1e-15)

    def index(turns):   # the real number i at which 10000^(-2i/rot) * trained / 2 pi = turns
        return 0.5 * rot * math.log(trained / (2 * math.pi * turns)) / math.log(10000.0)

    lo, hi = math.floor(index(32.0)), math.ceil(index(1.0))
    assert lo >= 0 and hi <= rot - 1
    mix = np.clip((np.arange(rot // 2) - lo) / (hi - lo), 0.0, 1.0)
    np.testing.assert_allclose(got.numpy(), plain * (1 - mix) + plain / factor * mix, rtol=1e-13)
    turns = trained * plain / (2 * math.pi)
    if turns[-1] > 1.0:     # no pair turns less than `slow` times: none is divided fully
        assert (got.numpy() > plain / factor * (1 + 1e-6)).all()


def test_last_pair_by_hand():
    """trained = 131072, base 10000, rot = 128: from index 45 (32 turns at 45.02) to 70 (one at 69.1); the last pair, 63, turns 2.4 times and is 18/25 of the way."""
    plain = binding.rope_frequencies(128)[0]
    got = binding.rope_frequencies(128, scaling="bands", factor=4.0, trained=131072)[0]
    assert float(got[-1] / plain[-1]) == pytest.approx(7 / 25 + 18 / 25 / 4, rel=1e-12)
    assert float(got[45] / plain[45]) == 1.0 and float(got[46] / plain[46]) < 1.0
