"""The runner's call for the bounds of keys, without a GPU."""
import pytest
import torch

from paper_2502_13542_amd import binding as B

from paged_utils import Batch, shape_of


@pytest.mark.parametrize("n_rows", [None, -1])
def test_rows_without_their_number_are_refused(n_rows):
    """Of row_start alone nobody knows how many rows it deals out: without the number (it was 0 then) the bounds were left as they were, in silence."""
    b = Batch(shape_of(4, 2, 64, "fp32"), [(2, 40), (3, 200)], 3)
    r, t = b.runner("cpu"), b.dev("cpu")
    bounds = torch.zeros(b.n_pages, 2, 2, 64)
    with pytest.raises(B.ActQKVError, match="row_start with n_rows"):
        r.key_bounds(t["n_ctx"], t["pages"], t["k_pages"], bounds, row_start=t["row_start"], **({} if n_rows is None else dict(n_rows=n_rows)))
    for kw in ({}, dict(row_start=t["row_start"], n_rows=5)):
        with pytest.raises(B.ActQKVError, match="not on the GPU"):                 # (sizes are right: the next check is the device)
            r.key_bounds(t["n_ctx"], t["pages"], t["k_pages"], bounds, **kw)
    r.key_bounds(t["n_ctx"], t["pages"], t["k_pages"], bounds, row_start=t["row_start"], n_rows=0)      # no rows: nothing to do
