"""Checks, from the sources of the KV-cache operators' tensor-core kernels, of rules that no run can be made to break
safely (as test_kernel_waits.py for the others)."""

import os
import re

import pytest

KV = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_12659_gb300", "csrc", "kv")
KERNELS = {"kv_attend_t5.cu": "k_kv_tiles_t5", "kv_weigh_t5.cu": "k_kv_weigh_t5"}


def kernel(name):
    with open(os.path.join(KV, name)) as f:
        text = f.read()
    start = text.index(f" {KERNELS[name]}(")
    return text[start:text.index("\ntemplate <int DP>\njpi_status launch_dim", start)]


@pytest.mark.parametrize("name", KERNELS)
def test_every_wait_is_bounded(name):
    body = kernel(name)
    assert "mbar_wait_bounded(" in body
    assert not re.search(r"mbar_wait(?!_bounded)\w*\(|try_wait|test_wait", body)


@pytest.mark.parametrize("name", KERNELS)
def test_errors_are_reported_and_tensor_memory_freed_after_the_last_barrier(name):
    body = kernel(name)
    last = max(body.rindex("__syncthreads()"), body.rfind("cluster_sync_all()"))
    assert body.rindex("atomicCAS(a.err, 0, *flag)") > body.rindex("__syncthreads()")
    assert body.index("tmem_dealloc(") > last
    assert "return;" not in body[body.index("tmem_alloc("):], "no role leaves the block early"


@pytest.mark.parametrize("name", KERNELS)
def test_a_wait_that_gave_up_is_noted(name):
    # The result of every wait is kept, and what is kept ends in the block's flag.
    body = kernel(name)
    for line in (x for x in body.splitlines() if "mbar_wait_bounded(" in x):
        assert "good = ptx::mbar_wait_bounded(" in line or "!ptx::mbar_wait_bounded(" in line, line.strip()
    assert body.count("if (!good) *flag = DEV_TIMEOUT") >= 3


def test_loaders_wait_for_their_last_copies():
    body = kernel("kv_attend_t5.cu")
    loaders = body[body.index("if (warp <= 1) {"):body.index("} else if (warp == 2) {")]
    assert "ring_drain(fullb, NS, issued," in loaders
    assert loaders.rindex("ring_drain(") > loaders.rindex("load(")
    # The key tile of the weights is one load, waited for by a thread of its own whatever the others do.
    weigh = kernel("kv_weigh_t5.cu")
    alone = weigh[weigh.index("if (warp == 0) {"):weigh.index("} else if (warp == 1) {")]
    assert "mbar_wait_bounded(kfull, 0," in alone


def test_the_last_products_have_a_barrier_of_one_phase():
    # A barrier that turns once a block cannot tell the last product from the one two phases before it.
    body = kernel("kv_attend_t5.cu")
    assert body.count("mbar_wait_bounded(alldone, 0,") == 1 and body.count("mma_commit(alldone)") == 1
    commit = body.index("mma_commit(alldone)")
    assert commit > body.index("mma_commit(&gdone[i % NG])") and commit < body.index("} else {", commit)


def test_clusters_meet_twice_around_the_sums_of_their_blocks():
    body = kernel("kv_weigh_t5.cu")
    reads = body.index("dsmem_ld_f32(")
    meets = [m.start() for m in re.finditer(r"if \(a\.ranks > 1\) ptx::cluster_sync_all\(\);", body)]
    assert len(meets) == 2 and meets[0] < reads < meets[1]


def test_a_wait_that_gave_up_in_any_block_of_a_cluster_keeps_its_keys_weights():
    # The block that writes reads the others' flags too, between the cluster's two meetings, and writes only if all are clear:
    # a sum that lacks a block's rows must not reach weights that are kept from call to call.
    body = kernel("kv_weigh_t5.cu")
    meets = [m.start() for m in re.finditer(r"if \(a\.ranks > 1\) ptx::cluster_sync_all\(\);", body)]
    part = body[meets[0]:meets[1]]
    own = re.search(r"bool whole = \*flag == 0;", part)
    loop = re.search(r"for \(int k = 1; k < a\.ranks; \+\+k\) \{(.*?)\n        \}", part, re.S)
    assert own and loop and own.start() < loop.start()
    assert re.search(r"whole = whole && __float_as_int\(ptx::dsmem_ld_f32\(ptx::dsmem_map\(ptx::smem_u32\(flag\), \(uint32_t\)k\)\)\) == 0;", loop[1])
    write = re.search(r"if \(([^{]*)\) \{[^}]*a\.out\[at\] =", part)
    assert write and "whole" in write[1] and write.start() > loop.end()
