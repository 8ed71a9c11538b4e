"""The tile kernel's ring as the memory of small tiles (csrc/lh_paged_lds.h), compiled for the host and gone through word by
word: a wave that is done writes its part while others still use their words, unless a barrier parts the two."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_06554_amd", "csrc")
SHAPES = [(D, NW) for D in (64, 128) for NW in (4, 8, 12)]


def clashes(D, NW, per, own, part, words):
    """What is wrong with a map: lists of (array, offset) by wave."""
    span = lambda at, n: {(at[0], at[1] + i) for i in range(n)}  # noqa: E731
    parts, mine = [span(a, 16 * D) for a in part[:per]], [span(a, 8 * D) for a in words]
    room = {(a, i) for a in range(4) for i in range(32 * D)}
    out = [f"wave {w} outside" for w in range(NW) if not mine[w] <= room or (w < per and not parts[w] <= room)]
    for w in range(NW):
        for y in range(NW):
            if w == y:
                continue
            if mine[w] & mine[y]:
                out.append(f"words {w}, words {y}")
            if w < per and y < per and parts[w] & parts[y]:
                out.append(f"part {w}, part {y}")
            if own and y < per and mine[w] & parts[y]:
                out.append(f"words {w}, part {y}, no barrier")
    return out


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not installed")
def test_words_and_parts_do_not_meet(tmp_path):
    src, exe = tmp_path / "map.cpp", str(tmp_path / "map")
    show = "".join(f"show<{D}, {NW}>();" for D, NW in SHAPES)
    src.write_text("""#include <cstdio>
#include "lh_paged_lds.h"
template <int D, int NW> void show() {
  using M = lh::TileLdsMap<D, NW>;
  std::printf("%d %d %d %d %d", D, NW, M::PER, (int)M::kOwnWords, (int)M::sound());
  for (int w = 0; w < NW; ++w) std::printf(" %d %d %d %d", M::part_array(w), M::part_off(w), M::words_array(w), M::words_off(w));
  std::printf("\\n");
}
int main() { SHOW }
""".replace("SHOW", show))
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", exe], check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(lines) == len(SHAPES)
    for line, shape in zip(lines, SHAPES):
        D, NW, per, own, sound, *at = map(int, line.split())
        assert (D, NW) == shape and sound == 1 and (per == NW or not own)
        at = [at[4 * w:4 * w + 4] for w in range(NW)]
        assert clashes(D, NW, per, own, [(a, b) for a, b, _, _ in at], [(c, d) for _, _, c, d in at]) == []


def test_the_check_finds_words_in_another_waves_part():
    """Eight waves whose words fill the arrays in order while their parts take the arrays in turn."""
    D, part, words = 128, [(w & 3, (w >> 2) * 2048) for w in range(8)], [(w >> 2, (w & 3) * 1024) for w in range(8)]
    assert "words 2, part 4, no barrier" in clashes(D, 8, 8, True, part, words)
    assert clashes(D, 8, 8, False, part, words) == []
