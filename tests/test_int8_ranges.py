"""The ranges that launches of the int8 product are cut into (csrc/vnm_i8_rules.h), compiled for the host."""

from tests.test_int8_rules import rule  # noqa: F401  (a fixture)


def test_a_range_fits_a_launch(rule):  # noqa: F811
    y, tiles, rows = rule("kI8GridY", "kI8GridTiles", "kI8GridRows")
    assert y <= 65535 and tiles * 512 < 2 ** 32 and -(-rows // 4) <= 65535
