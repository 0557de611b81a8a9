"""janus_batch_plan at the ends of the range of lengths."""
import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu
TOP = 2 ** 63 - 1


@pytest.mark.parametrize("page", [1, 24, 40, 64, 96])
@pytest.mark.parametrize("cached", [TOP, TOP - 1, 2 ** 62, 2 ** 40])
def test_lengths_that_no_table_holds(page, cached):
    """Rows of such a session have their position, 2^63 - 1 at most, and no place; the sessions beside it are served."""
    width, new = 3, [2, 5, 1]
    tables = torch.arange(9, dtype=torch.int32, device="cuda").view(3, width).contiguous()
    lens = torch.tensor([1, cached, 0], device="cuda")
    out = B.batch_plan_buffers(3, 10, 16, want_key_rows=True)
    B.janus_batch_plan(lens, torch.tensor(new, device="cuda"), tables, torch.arange(20, 29, dtype=torch.int32, device="cuda"), page_size=page, n_phys_pages=40, max_rows=10,
                       key_offsets=torch.tensor([0, 1000, 2000], device="cuda"), out=out)
    with pytest.raises(B.JanusError, match="CAPACITY_EXCEEDED"):
        B.check_dev_status()
    assert out["row_offsets"].tolist() == [0, 2, 7, 8] and out["kv_lens"].tolist() == [3, width * page, 1]
    assert out["positions"].tolist() == [1, 2] + [min(cached + i, TOP) for i in range(5)] + [0, -1, -1]
    assert out["slots"].tolist()[2:7] == [-1] * 5 and out["key_rows"].tolist()[2:7] == [-1] * 5
    assert all(s >= 0 for s in out["slots"].tolist()[:2] + out["slots"].tolist()[7:8])
    assert tables[1].tolist() == [3, 4, 5]
