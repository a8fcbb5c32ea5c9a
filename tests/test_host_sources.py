"""What the host code does with the CUDA runtime, read from its source: orders that no run can be made to miss."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2206_08869_b200", "csrc")


def _functions():
    """(file, text) of every function of the host sources: from one closing brace in the first column to the next."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*_api.cu"))):
        with open(path) as f:
            for part in re.split(r"^}", f.read(), flags=re.M):
                yield os.path.basename(path), part


def test_what_a_handle_is_made_of_has_arrived_when_it_is_handed_out():
    """cudaMemcpy from pageable memory returns when the memory may be reused, not when the device holds the data, and a stream
    made with cudaStreamNonBlocking (every side stream of torch) does not wait for the default stream."""
    seen = 0
    for name, text in _functions():
        copies = [m.start() for m in re.finditer(r"\bcudaMemcpy\([^;]*cudaMemcpyHostToDevice\)", text)]
        if copies:
            seen += 1
            assert re.search(r"\b(cudaStreamSynchronize\(0\)|cudaDeviceSynchronize\(\))", text[copies[-1]:]), (name, text[copies[-1]:][:200])
    assert seen >= 5                                  # models, codecs, projections, norms, refinements
