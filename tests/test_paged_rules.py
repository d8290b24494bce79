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


def test_what_an_eviction_has_read_again_is_bounded_before_it_is_an_index():
    # the keys of long rows are read several times, and rows that share pages change them in between: the candidates, the words
    # of the lists and the slots that they name are compared with their arrays' sizes
    text = re.sub(r"\s+", " ", source("kernels_paged_evict.cu"))
    assert not re.search(r"s_cand\[\s*atomicAdd", text) and re.search(r"if \((\w+) < kEvCand\) s_cand\[\1\]", text)
    assert re.search(r"min\(__shfl_sync\(0xffffffffu, count, warp\), kEvCand - before\)", text)
    assert "h < n - budget ? word(budget + h) : -1" in text
    moves = text[text.index("__ldcg(&c.list["):]
    assert moves.index("(unsigned)src < (unsigned)n") < moves.index("paged_nth(c, src)")
    assert moves.index("(unsigned)dst < (unsigned)n") < moves.index("paged_nth(c, dst)")


def test_an_eviction_takes_a_bin_whatever_the_histogram_holds():
    # s_bin, s_above and s_in are set in every round, by the thread of the lowest bins if no bin reaches the sum
    text = re.sub(r"\s+", " ", source("kernels_paged_evict.cu"))
    assert "const bool lowest = tid == kEvThreads - 1;" in text and "(need <= to || lowest)" in text
    assert "(lowest && b == 3)" in text


def test_no_cta_of_an_evicting_cluster_leaves_while_another_may_ask_for_its_length():
    # lengths that change while they are read: who returns early passes the two barriers between which the others compare theirs
    text = re.sub(r"\s+", " ", source("kernels_paged_evict.cu"))
    early = text.index("if (n <= budget) {")
    assert text[early:].startswith("if (n <= budget) { if (C > 1) { cluster.sync(); cluster.sync(); } return; }")
    rest = text[early:][len("if (n <= budget) { if (C > 1) { cluster.sync(); cluster.sync(); } return; }"):]
    first = rest.index("cluster.sync();")
    second = rest.index("cluster.sync();", first + 1)
    assert "map_shared_rank(x, lane)" in rest[:first] and "ask(&" not in rest[:first]
    assert first < rest.index("ask(&s_n, n) == n") < second
    assert rest[second:].startswith("cluster.sync(); if (!agreed) { paged_status(c, row); return; }")
