"""The query encoder's host side, without a GPU."""
import pytest
import torch

from paper_2506_00812_amd.query_encoder import QueryEncoder


@pytest.mark.parametrize("absent", [None, [], (), torch.empty(0), torch.empty(0, dtype=torch.int64), [1, 3], torch.tensor([1, 3])])
def test_absent_labels(absent):
    """No absent label at all is an ordinary answer of a table's sizes."""
    enc = QueryEncoder(8, 4, 5, dtype=torch.float32, absent=absent, device="cpu")
    want = [1, 3] if absent is not None and len(absent) else []
    assert torch.nonzero(torch.isneginf(enc.params["bl"]))[:, 0].tolist() == want
