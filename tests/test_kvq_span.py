"""Which rows and keys of a batch are a sequence's (csrc/remp_kvq_span.h): compiled for the host with a trap on every signed overflow,
against Python's whole numbers, at the ends of 32 bits."""
import itertools
import os
import subprocess

import paper_2606_18741_b200 as remp  # noqa: F401
from paper_2606_18741_b200.build import CSRC

MOST, LEAST = 2 ** 31 - 1, -2 ** 31
PROGRAM = r"""
#include <cstdio>
#include "remp_kvq_span.h"
int main() {
    int s, e, l, n, r, w;
    while (std::scanf("%d %d %d %d %d %d", &s, &e, &l, &n, &r, &w) == 6) {
        const remp::KvqSpan x = remp::kvq_span(s, e, l, n, r);
        std::printf("%d %d %d %d %d %d %d\n", x.q0, x.queries, x.len, x.first_pos, remp::kvq_first_key(x.first_pos, w),
                    remp::kvq_first_key(x.first_pos + (x.queries ? x.queries - 1 : 0), w), (int)remp::kvq_span_bad(x, l));
    }
}
"""


def test_spans_at_the_ends_of_32_bits(tmp_path):
    source, program = tmp_path / "span.cpp", tmp_path / "span"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-I", os.path.abspath(CSRC),
                    str(source), "-o", str(program)], check=True)
    ends = (LEAST, -1, 0, 1, 17, 2 ** 20, MOST - 1, MOST)
    most = 0x7fff0000  # of tokens and of a table's row
    cases = [c for c in itertools.product(ends, ends, ends, (1, 17, most), (0, 16, 2 ** 20, most), (0, 1, 16, MOST - 2, MOST))]
    run = subprocess.run([str(program)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True)
    rows = [tuple(map(int, line.split())) for line in run.stdout.splitlines()]
    assert len(rows) == len(cases)
    for (start, end, length, tokens, room, window), got in zip(cases, rows):
        q0 = min(max(start, 0), tokens)
        queries = max(0, min(end, tokens) - q0)
        first = max(length, 0) - queries
        last = first + max(0, queries - 1)
        keys = [max(0, p - window + 1) if window else 0 for p in (first, last)]
        assert got == (q0, queries, min(max(length, 0), room), first, *keys, int(not 0 <= length <= room or (queries > 0 and first < 0)))
