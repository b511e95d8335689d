"""The decoding loop's launches go by the device's number of SMs, which they are given."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2608_06690_gb300" / "csrc"


@pytest.mark.parametrize("name", ["k_cache.cu", "k_attend.cu", "k_sample.cu"])
def test_no_number_of_sms_is_written_out(name):
    code = re.sub(r"//[^\n]*|/\*.*?\*/", "", (CSRC / name).read_text(), flags=re.S)
    assert not re.search(r"\b(148|152|160)\b", code)
    assert re.search(r"\bnum_sms\b", code)
