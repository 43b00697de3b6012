"""Checks, from the source of the tensor-core tiles over windows and 8-bit caches, of rules that no run can be made to break safely
(as test_kernel_waits_kv.py for the other tiles)."""

import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_12659_gb300", "csrc", "kv", "kv_span_t5.cu")


def kernel():
    with open(SOURCE) as f:
        text = f.read()
    start = text.index(" k_kv_span_t5(")
    return text[start:text.index("\ntemplate <int DP>\njpi_status launch_dim", start)]


def test_every_wait_is_bounded_and_a_wait_that_gave_up_is_noted():
    body = kernel()
    assert not re.search(r"mbar_wait(?!_bounded)\w*\(|try_wait|test_wait", body)
    waits = [x.strip() for x in body.splitlines() if "mbar_wait_bounded(" in x]
    assert len(waits) >= 12 and all("good = ptx::mbar_wait_bounded(" in x for x in waits)
    assert len(re.findall(r"if \(!good\) \*flag = DEV_TIMEOUT", body)) == 5   # loaders, both products, codes, softmax


def test_errors_are_reported_and_tensor_memory_freed_after_the_last_barrier():
    body = kernel()
    last = body.rindex("__syncthreads()")
    assert body.index("tmem_dealloc(") > last and body.rindex("atomicCAS(a.err, 0, *flag)") > last
    # No role leaves the block early: the returns are those of lambdas.
    for x in re.findall(r"^.*\breturn\b.*$", body[body.index("tmem_alloc("):], re.M):
        assert re.search(r"auto \w+ = \[[^\]]*\]\([^)]*\) \{ return [^;]*; \};", x), x.strip()


def test_copies_have_landed_before_the_block_leaves():
    body = kernel()
    loaders = body[body.index("if (warp <= 1) {"):body.index("} else if (warp == 2) {")]
    assert loaders.rindex("ring_drain(fullb, NS, issued,") > loaders.rindex("load(is_v, i)")
    codes = body[body.index("} else if (Q8 && tid >= L::CONV) {"):]
    codes = codes[:codes.index("const int grp =")]
    assert codes.rindex("cp_async_wait_all()") > codes.rindex("fetch(")
    assert "break;" in codes and not re.search(r"\breturn\b", codes)


def test_the_last_products_have_a_barrier_of_one_phase():
    body = kernel()
    assert body.count("mbar_wait_bounded(alldone, 0,") == 1 and body.count("mma_commit(alldone)") == 1
    assert body.index("mma_commit(alldone)") > body.index("mma_commit(&gdone[i % NG])")


def test_barriers_of_a_ring_are_committed_only_where_a_block_follows():
    body = kernel()
    for ring, behind in (("kempty[sl]", "NS"), ("vempty[sl]", "NS"), ("odone[i % NB]", "NB"), ("gdone[i % NG]", "NG")):
        assert f"if (i + {behind} < nb) ptx::mma_commit(&{ring});" in body


def test_blocks_of_a_cluster_meet_before_their_parts_are_read_and_after():
    body = kernel()
    meets = [m.start() for m in re.finditer(r"ptx::cluster_sync_all\(\);", body)]
    read = body.index("join_tile<")
    assert len(meets) == 2 and meets[0] < read < meets[1] and "if constexpr (JOIN) {" in body[:meets[0]]
    # Nothing is written where a wait gave up in any block of the cluster.
    assert meets[0] < body.index("dsmem_map(ptx::smem_u32(flag)") < body.index("if (whole) join_tile<")
    with open(SOURCE.replace("kv_span_t5.cu", "kv_span.cu")) as f:
        rows = f.read()
    join = rows[rows.index("void join_cluster("):]
    join = join[:join.index("\n}\n")]
    meets = [m.start() for m in re.finditer(r"ptx::cluster_sync_all\(\);", join)]
    reads = [m.start() for m in re.finditer(r"ptx::dsmem_ld_", join)]
    assert len(meets) == 2 and all(meets[0] < r < meets[1] for r in reads) and len(reads) == 2
    assert join.count("return;") == 1 and "if (ranks == 1) return;" in join   # the same for all blocks
