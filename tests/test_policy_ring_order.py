"""Ordering of the shared places of the policy loss's ring kernel, shown on the
CPU: what its barriers and its warps' programs order after what, in every CTA of
a cluster, with the numbers of stages and places read from its source.

A place that is written again (a stage, the parts of a CTA or of the cluster, the
gradient's coefficients) has to have been read; a barrier's phase has to have
completed before an arrival of the next one; and a wait for a phase has to be over
before the next phase of its barrier completes, or its parity would be met again."""
import os
import re

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2609_34325_gb300", "csrc", "policy.cu")
ROWS = 14


def _kernel():
    src = open(SRC).read()
    start = src.index("policy_ring_kernel(Rows<T> r, Actions p) {")
    return src[start:src.index("finish_totals<3 +", start)]


def _size(src, name):
    """The first dimension of a shared array, a number or a constant of the kernel."""
    dim = re.search(r"\b%s\[(\w+)\]" % name, src).group(1)
    return int(dim if dim.isdigit() else re.search(r"\b%s = (\d+)" % dim, src).group(1))


class _Order:
    """Events and what is ordered after them, for `ctas` CTAs over ROWS rows."""

    def __init__(self, ctas, stages, places):
        self.ctas, self.stages, self.places = range(ctas), stages, places
        self.after, self.reach = {}, {}
        for c in self.ctas:
            self._cta(c)

    def edge(self, a, b):
        if a[-1] >= 0:
            self.after.setdefault(a, set()).add(b)

    def chain(self, *events):
        for a, b in zip(events, events[1:]):
            self.edge(a, b)

    def _cta(self, c):
        copies, sums, grads, joins = [], [], [], ([], [])
        for n in range(ROWS):
            # the producer: a stage that has been freed is filled
            self.edge(("empty", c, n - self.stages), ("copy", c, n))
            self.edge(("copy", c, n), ("full", c, n))
            copies.append(("copy", c, n))
            # the sum warps: the granules, then a part where the last has been taken
            sums += [("sum_full", c, n), ("sum", c, n), ("sum_ready", c, n), ("part", c, n)]
            self.edge(("full", c, n), ("sum_full", c, n))
            self.edge(("ready", c, n - 2), ("sum_ready", c, n))
            self.edge(("part", c, n), ("summed", c, n))
            # a joining warp has every other row
            joins[n % 2].extend([("join_summed", c, n), ("take", c, n), ("send", c, n),
                                 ("join_joined", c, n), ("read", c, n), ("join_taken", c, n),
                                 ("write_grad", c, n), ("hand", c, n)])
            self.edge(("summed", c, n), ("join_summed", c, n))
            for d in self.ctas:
                self.edge(("send", c, n), ("joined", d, n))
            self.edge(("joined", c, n), ("join_joined", c, n))
            self.edge(("taken", c, n - 2), ("join_taken", c, n))
            self.edge(("hand", c, n), ("ready", c, n))
            # the gradient warps
            grads += [("grad_full", c, n), ("grad_ready", c, n), ("read_grad", c, n),
                      ("free_grad", c, n), ("gradient", c, n), ("free", c, n)]
            self.edge(("full", c, n), ("grad_full", c, n))
            self.edge(("ready", c, n), ("grad_ready", c, n))
            self.edge(("free_grad", c, n), ("taken", c, n))
            self.edge(("free", c, n), ("empty", c, n))
        for program in (copies, sums, grads) + joins:
            self.chain(*program)

    def before(self, a, b):
        if a not in self.reach:
            seen, todo = set(), [a]
            while todo:
                for e in self.after.get(todo.pop(), ()):
                    if e not in seen:
                        seen.add(e)
                        todo.append(e)
            self.reach[a] = seen
        return b in self.reach[a]

    def faults(self):
        """(what, CTA, row, later row) of places and phases that are not in order."""
        out = []

        def need(what, c, n, m, first, then):
            if m < ROWS and not self.before(first, then):
                out.append((what, c, n, m))

        for c in self.ctas:
            for n in range(ROWS):
                m = n + self.stages
                need("stage", c, n, m, ("sum", c, n), ("copy", c, m))
                need("stage", c, n, m, ("gradient", c, n), ("copy", c, m))
                for wait in ("sum_full", "grad_full"):
                    need("full", c, n, m, (wait, c, n), ("copy", c, m))
                need("empty", c, n, m, ("copy", c, m), ("free", c, m))
                m = n + 2
                need("parts", c, n, m, ("take", c, n), ("part", c, m))
                need("summed", c, n, m, ("join_summed", c, n), ("part", c, m))
                need("coefficients", c, n, m, ("read_grad", c, n), ("write_grad", c, m))
                need("ready", c, n, m, ("grad_ready", c, n), ("hand", c, m))
                need("ready", c, n, m, ("sum_ready", c, m), ("hand", c, m))
                need("taken", c, n, m, ("join_taken", c, m), ("free_grad", c, m))
                m = n + self.places
                for d in self.ctas:
                    need("cluster's parts", c, n, m, ("read", c, n), ("send", d, m))
                    need("joined", c, n, m, ("joined", c, n), ("send", d, m))
                    need("joined", c, n, m, ("join_joined", c, n), ("send", d, m))
        return out


@pytest.mark.parametrize("ctas", [2, 3, 4])
def test_places_of_the_ring_are_read_before_they_are_written_again(ctas):
    src = _kernel()
    assert _size(src, "slots") == _size(src, "grads") == 2
    places = _size(src, "ctas")
    assert places == _size(src, "joined")
    assert _Order(ctas, _size(src, "full"), places).faults() == []


def test_the_model_tells_one_place_a_joining_warp_from_two():
    one = _Order(2, 3, 2).faults()
    assert {what for what, *_ in one} == {"cluster's parts", "joined"}
    assert _Order(2, 3, 4).faults() == []


def test_no_copy_follows_a_wait_that_ran_out():
    # warps that give up arrive like those that are done, so the copying warp's own wait
    # may succeed: it has to look at the CTA's flag before each copy into a used stage
    src = _kernel()
    producer = src[src.index("if (warp == 2) {"):src.index("bulk_load(")]
    assert producer.count("wait(") == 1
    assert "if (abort) break;" in producer[producer.index("wait(&empty[stage], lap - 1)"):]
