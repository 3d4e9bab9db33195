"""A bounded wait of a paged attention kernel that runs out: the call records BD_ERR_TIMEOUT, waits for what it has in flight and
returns; a row is either right or left unwritten, and the next call is served normally.  The wait is made to run out on the
host's side of the kernel's own protocol (a barrier of the first CTA expects one arrival more than it gets; the copies themselves
are made and arrive); no trap, no endless loop."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from test_paged_accuracy_gpu import WAYS, i32, world
from util import to_device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
def test_rows_are_right_or_unwritten_after_a_wait_that_runs_out(kind, way):
    w, q, t, heads = world(way, kind, seed=70)
    q = to_device(q, kind)
    b = bd.PagedBatch(w.table, w.slots, i32([w.seqs[0].length]), i32([0, t]), t)
    size = bd.paged_attention_workspace_size(w.cache, b, t, heads)
    good_lse = torch.empty(t, heads, device="cuda")
    good = bd.paged_attention(w.cache, b, q, dtype=torch.float32, lse=good_lse)
    bd.poll_status()
    for junk in (0x00, 0x7f):                                       # what the parts' places hold before: zeros, large numbers
        workspace = torch.full((max(size, 256),), junk, dtype=torch.uint8, device="cuda")
        out, lse = torch.full_like(good, -7.0), torch.full_like(good_lse, -7.0)
        try:
            bd.debug_fault(poll_limit=10 * 1024, skip_first_code_stage=True)
            bd.paged_attention(w.cache, b, q, out=out, lse=lse, workspace=workspace)
            with pytest.raises(bd.BdError) as e:
                bd.poll_status()
            assert e.value.status == 7                              # BD_ERR_TIMEOUT
        finally:
            bd.debug_fault(0, False)
        right, unwritten = (out == good).all(-1) & (lse == good_lse), (out == -7).all(-1) & (lse == -7)
        assert (right | unwritten).all() and unwritten.any()
        if WAYS[way][2] > 1:
            assert right.any()                                      # the other KV head's CTA is not concerned
        again = bd.paged_attention(w.cache, b, q, dtype=torch.float32, workspace=workspace)
        bd.poll_status()
        assert torch.equal(again, good)
