"""Orders between the threads of the training operators' kernels that no run shows reliably: read from the kernels' text (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_08527_b200", "csrc")


def _body(file, head):
    """The text of the function whose declaration holds `head`, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    at = text.index("{", text.index(head))
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if depth == 0:
            return text[at:end]


def test_the_edges_of_the_first_row_are_there_before_it_is_read():
    # stored by the first warp, read by all: between them stands a barrier that releases the stores, for either owner
    body = _body("rocket_norm_backward.cuh", "block_rows_kernel(const Backward a")
    between = body[body.index("put_edges(0);"):body.index("for (int64_t row = owner")]
    cluster, block = re.search(r"if constexpr \(OWNER == kCluster\) \{(.*?)\} else \{(.*?)\}", between, re.S).groups()
    assert "__syncthreads()" in block
    assert "__syncthreads()" in cluster or ("barrier.cluster.arrive.release" in cluster and "barrier.cluster.wait.acquire" in cluster)
    body = _body("rocket_norm_forward.cuh", "rows_kernel(const Forward a")
    between = body[body.index("edge.put(ring);"):body.index("for (int turn = 0; row < a.N")]
    assert re.search(r"if constexpr \(OWNER != kWarp\) \{[^}]*__syncthreads\(\);", between)


def test_no_block_ends_while_another_reads_its_sums():
    # every value loaded from another block is used, and the last arrival releases, so that it stands behind the loads
    body = _body("rocket_norm_backward.cuh", "join_owners(const float* sums")
    loop, end = body[body.index("for (int i ="):body.rindex("store_typed")], body[body.rindex("store_typed"):]
    assert loop.index("if (!out) continue;") < loop.index("ld.shared::cluster")
    assert "leave_cluster" not in end and "barrier.cluster.arrive.release" in end and "barrier.cluster.wait.acquire" in end


def test_a_wait_that_gave_up_shows_in_every_sum_of_its_thread():
    body = _body("rocket_norm_backward.cuh", "block_rows_kernel(const Backward a")
    behind = body[body.index("m = next_m;"):body.index("float* out = a.joined")]
    assert re.search(r"if \(!ok\).*k < NV.*dg\[k\]\[j\] = db\[k\]\[j\] = __int_as_float\(0x7fc00000\)", behind, re.S)
