"""How the token-sequence units are compiled (no GPU)."""
from paper_2601_22275_amd import build

FREE = ("-fno-honor-nans", "-fno-honor-infinities", "-ffinite-math-only", "-ffast-math", "-Ofast")


def test_units_that_define_what_nan_and_infinities_do_keep_them():
    """The header says what infinities and NaN do in these calls; a compiler told that there are none may drop the code that keeps to it."""
    units = {src: build.FLAGS + build.EXTRA.get(src, []) + own for src, _, own in build.SOURCES if src.startswith("seq_") or src == "rotary.hip"}
    assert len(units) == 6
    for src, flags in units.items():
        assert not set(flags) & set(FREE), (src, flags)
