"""Rules of the paged cache's kernels that no run on a GPU shows broken on demand, checked where they are written."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2412_04757_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_what_an_arrival_has_acquired_is_ordered_for_the_threads_that_read_it():
    # one thread arrives, and with it sees the other CTAs' parts; the others of its warp or CTA read them only behind a barrier,
    # since exchanging registers orders no memory
    text = source("kernels_paged_decode.cu")
    arrivals = [m.end() for m in re.finditer(r"paged_arrive\(", text)]
    assert len(arrivals) == 2
    for at in arrivals:
        rest = text[at:]
        read = re.search(r"wk\.part \+", rest).start()
        assert re.search(r"__sync(warp|threads)\(\)", rest[:read]), rest[:200]
