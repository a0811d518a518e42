"""Texts of the device status words, whose bits several calls may have OR-ed in.  No kernel is
launched."""
import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2609_32444_gb300 import binding as b
    from paper_2609_32444_gb300 import build
    build.build()
    b.lib()
    return b


@pytest.mark.parametrize("code", range(4, 32, 4))
def test_every_set_of_bits_has_its_names(binding, code):
    text = binding.status_string(code)
    for bit, name in ((4, "CIS_ERR_DEVICE_TIMEOUT"), (8, "CIS_ERR_BAD_TOKEN_ID"),
                      (16, "CIS_ERR_BAD_INPUT")):
        assert (name in text) == bool(code & bit), text


def test_a_repeated_id_is_named(binding):
    assert "twice" in binding.status_string(binding.CIS_ERR_BAD_TOKEN_ID)


@pytest.mark.parametrize("code", [-1, 5, 6, 32, 36, 64])
def test_other_codes_are_unknown(binding, code):
    assert binding.status_string(code) == "unknown cis status"
