"""Checks, from the source of the tiles over windows and 8-bit caches whose parts a pair of blocks joins, that no block waits for another
one while it holds what that one may need (as test_kernel_waits_spans.py for their other waits)."""

import re

from test_kernel_waits_spans import kernel


def test_tensor_memory_is_free_before_a_block_waits_for_its_partner():
    # The allocation waits, without a limit, for columns that another block of the SM holds. Were they held across the pair's barrier, two
    # pairs with blocks on the same two SMs could each hold the columns that the other's partner waits for.
    body = kernel()
    free, meet = body.index("ptx::tmem_dealloc("), body.index("ptx::cluster_sync_all()")
    assert body.count("ptx::tmem_dealloc(") == body.count("ptx::tmem_alloc(") == 1
    assert body.index("ptx::tmem_alloc(") < body.rindex("__syncthreads()") < free < meet
    assert not re.search(r"tmem_|mma_|cluster_arrive|cluster_wait", body[free + len("ptx::tmem_dealloc("):])
    assert "cluster" not in body[body.index("ptx::tmem_alloc("):free]
    # Released by the warp that took it, in every block.
    assert re.search(r"\n    if \(warp == 1\) \{\n\s+ptx::tmem_alloc\(", body) and re.search(r"\n    if \(warp == 1\) ptx::tmem_dealloc\(", body)
