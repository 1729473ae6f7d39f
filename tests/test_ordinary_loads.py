"""The products begin before the kernel in front of them has ended.  What such a kernel may write (operands, scales, results of quantisers) is
read by ordinary loads; the read-only path, which asks for data that nothing writes while a kernel lives, is left to offsets and parameters."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2209_10778_b200" / "csrc"


@pytest.mark.parametrize("name", ["nfad_product.cuh", "nfad_split.cuh", "nfad_few_rows.cuh", "nfad_scaled.cuh", "nfad_scaled_split.cuh", "nfad_blocks.cuh", "nfad_bytes.cuh"])
def test_read_only_path(name):
    text = (CSRC / name).read_text()
    assert not re.search(r"ld\.global(\.\w+)*\.nc", text)
    for use in re.findall(r"__ldg\(([^;]*);", text):
        assert use.startswith("g.offsets"), use
