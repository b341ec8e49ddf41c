"""Host side of the calls over 8-bit caches and pages: calls whose tensors the library cannot be told of.  No GPU."""
import re
from pathlib import Path

import pytest
import torch

from paper_2605_07243_b200 import binding as sb
from test_quant_cpu import INVALID, append, cache


def test_rows_that_overlap_are_refused():
    """An expanded tensor has a stride of 0 between its rows, which to the library is the ordinary one."""
    one = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    for rows in (one.expand(5, 2, 64), torch.zeros(1024, dtype=torch.bfloat16).as_strided((5, 2, 64), (64, 64, 1)),
                 torch.zeros(4, 1, 2, 64, dtype=torch.bfloat16).expand(4, 3, 2, 64)):
        with pytest.raises(ValueError, match="overlap"):
            sb._rows_of(rows, 2, 64, -1, "rows", rows.dim())
    assert sb._rows_of(one.expand(1, 2, 64), 2, 64, -1, "rows") == (one.data_ptr(), 128)
    fused = torch.zeros(5, 7, 64, dtype=torch.bfloat16)
    assert sb._rows_of(fused[:, 3:5], 2, 64, -1, "rows") == (fused.data_ptr() + 2 * 3 * 64, 7 * 64)
    # layers may repeat: their stride has its own argument
    assert sb._rows_of(fused[None, :, 3:5].expand(4, 5, 2, 64), 2, 64, -1, "rows", 4)[1] == 7 * 64


def test_strided_rows_of_other_dimensions_are_refused():
    """[rows, 1, heads, dim] as a slice: the stride that counts is not the one before the heads."""
    fused = torch.zeros(5, 1, 7, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="dimensions"):
        sb._rows_of(fused[:, :, 3:5], 2, 64, -1, "rows")
    assert sb._rows_of(fused, 7, 64, -1, "rows") == (fused.data_ptr(), 7 * 64)


@pytest.mark.parametrize("page_size", [0, 16])
def test_append_refuses_layers_that_overlap(page_size):
    """8 pages (or 2 sequences) of 16 tokens, 2 heads of 64: a layer has 16384 (4096) codes and 16 (4) scales."""
    codes, scales = (16384, 16) if page_size else (4096, 4)
    for n_layers, code_stride, scale_stride in ((2, codes - 16, scales), (2, codes, scales - 1), (3, 0, scales), (2, codes, 0)):
        kv = cache(n_layers=n_layers, codes_layer_stride=code_stride, scale_layer_stride=scale_stride, page_size=page_size, kv_capacity=16)
        assert append(kv=kv) == INVALID


def test_the_number_of_sms_is_asked_for_in_one_place():
    """The planner of the 8-bit attention, the choice of its merge buffer and the grid of the page copies go by the same device."""
    csrc = Path(sb.__file__).parent / "csrc"
    for name in ("quant_attention.cu", "quant_attention_rows.cu", "quant_attention_tc.cu", "kv_append_quant.cu", "pages.cu"):
        code = re.sub(r"//[^\n]*", "", (csrc / name).read_text())
        assert not re.search(r"\b148\b", code), name
    assert "device_sms()" in (csrc / "pages.cu").read_text() and "device_sms()" in (csrc / "quant_attention.cu").read_text()
