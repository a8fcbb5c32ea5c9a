"""What the kernels of the single layers rely on, read from their source: conditions of the instructions that no run can be made to miss."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2206_08869_b200", "csrc")


def _text(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_a_warp_is_whole_where_an_instruction_wants_it_whole():
    """.aligned: every lane of the warp executes the same instruction. After code whose lanes may part (one thread sets barriers up, lanes
    store the rows that are theirs) only __syncwarp brings them together for certain."""
    functions = re.findall(r"__device__ __forceinline__ \w+ (cluster_\w+)\([^)]*\) \{\n(.*?)\n\}", _text("ptx_cluster.cuh"), flags=re.S)
    barriers = [(name, body) for name, body in functions if ".aligned" in body]
    assert len(barriers) == 2
    for name, body in barriers:
        assert body.strip().startswith("__syncwarp();"), name
    text = _text("proj_kernel.cu")
    loop = re.search(r"for \(int c = 0; c < cols; c \+= 32.*?done\(&sh\.tempty", text, flags=re.S).group(0)
    loop = loop[loop.index("transpose4(t1"):]                  # behind the loads and what every lane does
    parts = [m.start() for m in re.finditer(r"if \(rows32 >> \(|if \(n < a\.n\)", loop)]
    assert len(parts) == 3
    for at in parts:
        assert "__syncwarp();" in loop[at:], loop[at:]
    assert "__syncwarp();" in loop[parts[0]:parts[-1]]
    # no barrier of a cluster beside the two wrappers
    assert "barrier.cluster" not in text


def _kernels():
    """(name, body) of the projection's kernels that hand work to the tensor cores."""
    text = _text("proj_kernel.cu")
    for m in re.finditer(r"__global__ void [^(]*\([^)]*\) (\w+)\(.*?\n}\n", text, flags=re.S):
        if "umma" in m.group(0) or "mma(" in m.group(0):
            yield m.group(1), m.group(0)


def test_no_arrival_of_the_mmas_is_left_to_come_when_a_cta_leaves():
    """Every barrier that a commit arrives at is waited for after its last use: the full accumulators by the epilogue, the slots that
    are given back by whoever fills them."""
    kernels = dict(_kernels())
    assert len(kernels) == 3, list(kernels)
    for name, body in kernels.items():
        for ring in set(re.findall(r"commit\((?:ptx::smem_u32\()?&sh\.(\w*empty)\[", body)):
            if ring == "xempty" or ring == "aempty":
                loop = r"for \(int \w+ = 0; ok && \w+ < [\w.]+; [^)]*\) ok = wait\(&sh\.%s\[" % ring
                assert re.search(loop, body), (name, ring)
            else:
                assert "given_back(abort_flag, a.status, sh.%s," % ring in body, (name, ring)


def test_a_cta_that_gives_up_lets_its_copies_and_mmas_end():
    """Every wait of the projection's kernels, when it gives up, lets what its thread has asked for end before the thread stops: the CTA does
    not free its tensor memory or leave before all of them have stopped."""
    header, text = _text("ptx_cluster.cuh"), _text("proj_kernel.cu")
    body = {m.group(1): m.group(2) for m in re.finditer(r"bool (\w+_wait)\([^)]*\) \{\n(.*?)\n\}", header, flags=re.S)}
    assert set(body) == {"settled_wait", "quick_wait"}
    gave_up = body["settled_wait"].split("return true;")[1]
    assert "__nanosleep" in gave_up and re.search(r"i < \d+ &&", gave_up)              # and that ends, too
    assert "return settled_wait(" in body["quick_wait"] and "bounded_wait" not in body["quick_wait"]
    assert not re.search(r"bounded_wait|try_wait|test_wait", text)
    for name, kernel in _kernels():
        assert "__syncthreads();" in kernel[:kernel.index("tmem_dealloc")][-600:], name
