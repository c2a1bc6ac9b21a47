"""Scaled rotary frequencies against constants worked out apart from the code, with 40 decimal digits from the scheme's definition, and the
properties that the schemes are chosen for.  Double precision: relative 1e-12."""
import math

import pytest

from paper_2605_07330_amd import srs


def test_by_index():
    """Base 1e6, 32768 positions, four times slower: pair 23.6 turns 32 times and pair 39.7 once, so 23 and those before it stay and 40 and those behind
    it are slowed down."""
    f, magnitude = srs.rope_frequencies(128, 1e6, "parts by index", 4.0, 32768)
    for i, want in {0: 1.0, 23: 6.978305848598663e-3, 24: 5.375321490790102e-3, 31: 8.029597275452303e-4, 39: 6.490394320837029e-5, 40: 4.445698525097307e-5,
                    63: 3.102344401879299e-7}.items():
        assert f[i].item() == pytest.approx(want, rel=1e-12), i
    assert magnitude == pytest.approx(1.1386294361119891, rel=1e-14)
    f, magnitude = srs.rope_frequencies(64, 1e4, "parts by index", 16.0, 2048)
    for i, want in {0: 1.0, 8: 0.1, 9: 6.958153000055960e-2, 14: 1.008831588387466e-2, 20: 4.256912234842049e-4, 21: 1.482108566038535e-4, 31: 8.334508951020775e-6}.items():
        assert f[i].item() == pytest.approx(want, rel=1e-12), i
    assert magnitude == pytest.approx(1.2772588722239781, rel=1e-14)


def test_by_turns():
    f, magnitude = srs.rope_frequencies(128, 5e5, "turns", 8.0, 8192, fast_turns=4.0, slow_turns=1.0)
    for i, want in {0: 1.0, 20: 1.656044008099445e-2, 28: 3.211445994752591e-3, 29: 2.166570763503359e-3, 31: 8.567514129196321e-4, 33: 3.126937503840651e-4,
                    34: 1.785078127679964e-4, 35: 9.556212353964683e-5, 36: 7.784655273932450e-5, 63: 3.068925988914511e-7}.items():
        assert f[i].item() == pytest.approx(want, rel=1e-12), i
    assert magnitude == 1.0
    same, scaled = srs.rope_frequencies(128, 5e5, "parts", 8.0, 8192, fast_turns=4.0, slow_turns=1.0)
    assert same.tolist() == f.tolist() and scaled == pytest.approx(0.1 * math.log(8.0) + 1)


@pytest.mark.parametrize("scaling", ["turns", "parts", "parts by index"])
@pytest.mark.parametrize("rot,base,context", [(128, 1e6, 32768), (2, 1e4, 4096), (64, 1e4, 40), (64, 1e4, 3), (80, 5e5, 10**7)])
def test_between_unscaled_and_slowed(scaling, rot, base, context):
    """Every pair lies between its own frequency and that over the factor, and never rises again; contexts that no pair, or every pair, turns often in."""
    plain, f = srs.rope_frequencies(rot, base)[0], srs.rope_frequencies(rot, base, scaling, 4.0, context)[0]
    share = plain / f
    assert bool((share >= 1 - 1e-12).all() and (share <= 4 + 1e-12).all()) and bool((share.diff() >= -1e-12).all())
    assert srs.rope_frequencies(rot, base, scaling, 1.0, context)[0].tolist() == pytest.approx(plain.tolist(), rel=1e-15)


def test_refusals():
    for scaling in ("turns", "parts", "parts by index"):
        for kw in ({}, {"original_context": -5}, {"original_context": 4096, "fast_turns": 1.0}):
            with pytest.raises(ValueError):
                srs.rope_frequencies(64, 1e4, scaling, 4.0, **kw)
    for kw in ({"base": 1.0}, {"slow_turns": 0.0}):
        with pytest.raises(ValueError):
            srs.rope_frequencies(64, scaling="parts by index", factor=4.0, original_context=4096, **kw)
