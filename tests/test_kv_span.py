"""Which tiles and keys rows see with a window and first tokens (csrc/remp_kvq_span.h): compiled for the host with a trap on every signed
overflow, against the plain rule key by key."""
import itertools
import os
import subprocess

from paper_2606_18741_b200.build import CSRC

MOST = 2 ** 31 - 1
PROGRAM = r"""
#include <cstdio>
#include "remp_kvq_span.h"
int main() {
    int len, pos, w, f, key;
    while (std::scanf("%d %d %d %d %d", &len, &pos, &w, &f, &key) == 5) {
        const remp::KvqSpan x{0, 1, len, pos};
        const remp::KvTiles t = remp::kv_tiles(x, pos, w, f);
        std::printf("%d %d %d %d\n", t.sinks, t.tile0, t.rest, (int)remp::kv_sees(pos, key, w, f));
    }
}
"""


def test_tiles_and_keys(tmp_path):
    source, program = tmp_path / "tiles.cpp", tmp_path / "tiles"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-I", os.path.abspath(CSRC),
                    str(source), "-o", str(program)], check=True)
    small = [c for c in itertools.product((0, 1, 15, 16, 17, 40, 100), (-5, 0, 1, 16, 39, 99, 120), (0, 1, 2, 16, 17, 50, MOST), (0, 1, 4, 16, 17, 90, MOST), (0, 3, 16, 33, 99))]
    large = [c for c in itertools.product((0, 0x7fff0000), (-2 ** 31 + 1, -1, 0x7fff0000, MOST), (0, 1, MOST), (0, 1, MOST), (0, 0x7ffeffff))]
    run = subprocess.run([str(program)], input="\n".join(" ".join(map(str, c)) for c in small + large), capture_output=True, text=True, check=True)
    rows = [tuple(map(int, line.split())) for line in run.stdout.splitlines()]
    assert len(rows) == len(small) + len(large)
    for (length, pos, window, first, key), (sinks, tile0, rest, seen) in zip(small + large, rows):
        assert seen == int(key <= pos and (window == 0 or key > pos - window or key < first))
        assert 0 <= sinks <= tile0 and rest >= 0 and tile0 + rest == -(-length // 16)
        if length <= 100:
            tiles = set(range(sinks)) | set(range(tile0, tile0 + rest))
            # a row at `pos` or behind it sees no key outside these tiles
            for k in range(length):
                for p in (pos, pos + 1, pos + 30):
                    if k <= p and (window == 0 or k > p - window or k < first):
                        assert k // 16 in tiles
