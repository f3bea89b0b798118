"""What the attention kernel waits on, by its source: barriers that count arrivals of all warps of a role end only if these agree on how many items there
are, which lengths that change during a step can undo.  So every wait of a role is a bounded one, and a barrier of the whole
block stands only where no role has begun, or every role has ended."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_22972_b200", "csrc")


def code(name):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, name)).read(), flags=re.S)


def kernel():
    text = code("attention_kernel.cuh")
    begin = text.index("attention_kernel(const __grid_constant__ CUtensorMap")
    return text[begin:text.index("__global__", begin)]


def test_no_wait_of_a_role_is_without_a_bound():
    text = kernel()
    for unbounded in ("bar.sync", "barrier.sync", "barrier.cta.sync", "barrier.red", "test_wait", "try_wait", "cp.async.wait", "nanosleep", "mbar_wait("):
        assert unbounded not in text, unbounded
    waits = re.findall(r"\bmbar_wait\w*", text)
    assert set(waits) == {"mbar_wait_suspended", "mbar_wait_quiet"} and waits.count("mbar_wait_suspended") == 1   # wait_warp, and the way out


def test_barriers_of_the_whole_block_stand_before_and_behind_the_roles():
    text = kernel()
    roles = text.index("Walk walk("), text.index("if (failed && !pending) misc[1] = 1;")
    at = [m.start() for m in re.finditer(r"__syncthreads\(\)", text)]
    assert at and all(x < roles[0] or x > roles[1] for x in at)


def test_loads_and_products_have_ended_before_the_block_does():
    text = kernel()
    ends = text.index("} else if (warp == S::kWarpQ) {"), text.index("} else if (warp == S::kWarpMma) {")
    loaders, queries, products = text[:ends[0]], text[ends[0]:ends[1]], text[ends[1]:]
    assert re.search(r"wait_warp\(!values \? k_full\(st\)", loaders[-300:])
    assert re.search(r"uses > 0\) wait_warp\(q_full\(s\)", queries)
    assert re.search(r"mma_commit\(drained\).*?wait_warp\(drained, 0\)", products, flags=re.S)
