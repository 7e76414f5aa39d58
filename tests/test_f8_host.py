"""Host programs of the 8-bit float layers: the addresses of products whose rows are cut into launches.  CPU only."""
from paper_2512_18453_amd import build


def test_launches_of_a_product_stay_inside_its_operands():
    assert build.host_program("f8_call_selftest.cpp").endswith("f8_call_selftest: ok")


def test_quotients_are_divisions():
    """Two thirds of a billion quotients; optimised, because the sanitized build of this would take minutes."""
    assert build.host_program("f8_quotient_selftest.cpp", flags=["-O3", "-march=native"]).endswith("f8_quotient_selftest: ok")
