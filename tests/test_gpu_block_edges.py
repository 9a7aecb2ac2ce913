"""Norm, block means, block choice and block-sparse attention where values are
not finite, ties lie close or a call is taken in parts, against the fp64 oracle.

Finite values are held to the bounds of test_gpu_block.py; a value that the
formula makes an infinity or no number has to be that."""
import numpy as np
import pytest

from oracle import block as B
from test_gpu_block import U, check_attend, dev, dt_of, host, huge, not_finite, rs3, run_attend, run_select
from workloads import storage_to_f64, to_storage

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- select --------------------------------------------------------------------
@pytest.mark.parametrize("make", [not_finite, huge])
@pytest.mark.parametrize("n_obj,n_q,n_kv,top_k,first,last,vis", [
    (2, 37, 1500, 4, 2, 2, "ragged"), (2, 37, 1500, 3, 0, 3, "causal"), (3, 300, 5000, 2, 2, 0, "ragged"),
    (2, 1, 1500, 4, 2, 2, "ragged")])
def test_forced_blocks_alone_fill_the_list(make, n_obj, n_q, n_kv, top_k, first, last, vis):
    """No block is chosen, whatever its score: the list is the forced ones and
    its count no more than top_k."""
    run_select(n_obj, n_q, n_kv, 4, 2, 64, 32, top_k, first, last, vis, "bf16", seed=n_q + top_k, make=make)
