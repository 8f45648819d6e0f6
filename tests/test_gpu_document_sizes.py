"""Attention of packed documents at sizes that choose other paths than short rows do; the cases and tolerances are those of
test_gpu_attention_docs.py."""
import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu


def test_spans_of_more_than_2_to_the_30_documents():
    # almost all of them empty; the sum of two of their indices is beyond an int
    n, rows = (1 << 30) + 1000, 100
    ends = torch.zeros(n, dtype=torch.int32, device="cuda")
    ends[-3:] = torch.tensor([40, 40, 90], dtype=torch.int32, device="cuda")
    spans = torch.full((4 * rows + 1,), -9, dtype=torch.int32, device="cuda")
    B.dapple_doc_spans(ends.data_ptr(), n, rows, spans.data_ptr())
    lo, hi, qlo, qhi = spans[:-1].view(4, rows).cpu().tolist()
    assert int(spans[-1]) == 90
    for i in range(rows):
        begin, end = (0, 40) if i < 40 else (40, 90)
        assert (lo[i], hi[i], qlo[i], qhi[i]) == ((begin, i + 1, i, end) if i < 90 else (90,) * 4), i
