"""Where the parts of attention's gradients lie: none shares a place with another, and none is lost to 32 bits where first tokens are many."""
import json
import os
import random
import subprocess

import pytest

from paper_1606_05688_amd import build

PROGRAM = """
#include <stdio.h>
#include "back_parts.h"
int main()
{
    znni::BackParts p;
    int bh, tile, split;
    while (scanf("%d %d %d %d %d %d %d %d", &p.tiles, &p.splits, &p.first_tiles, &p.far_tiles, &p.far, &bh, &tile, &split) == 8)
        printf("[%lld, %lld, %lld]\\n", p.per_head(), p.own_part(bh, tile, split), p.far_part(bh, tile, split));
}
"""


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    """[per_head, own_part, far_part] of each (tiles, splits, first_tiles, far_tiles, far, bh, tile, split), by the library's own header."""
    folder = tmp_path_factory.mktemp("parts")
    (folder / "main.hip").write_text(PROGRAM)
    program = str(folder / "main")
    subprocess.run([build.HIPCC, "--offload-host-only", "-std=c++17", "-I", build.CSRC, str(folder / "main.hip"), "-o", program], check=True, capture_output=True)

    def ask(asked):
        text = "\n".join(" ".join(map(str, a)) for a in asked)
        r = subprocess.run([program], input=text, capture_output=True, text=True, check=True)
        return [json.loads(line) for line in r.stdout.splitlines()]

    return ask


def test_parts_have_places_of_their_own(places):
    rng = random.Random(3)
    for _ in range(20):
        tiles, splits, heads = rng.randint(1, 5), rng.choice((1, 1, 2, 5)), rng.randint(1, 3)
        first = rng.randint(0, tiles)
        far_tiles = rng.randint(4 * first - 3, 4 * first) if first else 0
        plan = (tiles, splits, first, far_tiles, rng.randint(1, 6) if first else 0)
        own = [(bh, t, s) for bh in range(heads) for t in range(tiles if splits > 1 else first) for s in range(splits)]
        far = [(bh, t, s) for bh in range(heads) for t in range(far_tiles) for s in range(plan[4])]
        got = places([(*plan, *x) for x in own + far])
        spans = sorted([(g[1], g[1] + 128) for g in got[:len(own)]] + [(g[2], g[2] + 32) for g in got[len(own):]])
        # one behind the other, without a gap, as many as the workspace is made for
        assert [a for a, _ in spans] == [0, *(b for _, b in spans[:-1])][:len(spans)]
        assert not spans or spans[-1][1] == got[0][0] * heads


@pytest.mark.parametrize("tokens,far", [((1 << 25) - 31, 64), (1 << 25, 64), (1 << 27, 64), ((1 << 31) - 300, 5)])
@pytest.mark.parametrize("bh", [0, 3])
def test_parts_of_many_first_tokens(places, tokens, far, bh):
    first, far_tiles = (tokens + 127) // 128, (tokens + 31) // 32
    per_head = first * 128 + far_tiles * far * 32
    last = [first, 1, first, far_tiles, far, bh]
    (a, own, _), (_, _, there) = places([(*last, first - 1, 0), (*last, far_tiles - 1, far - 1)])
    assert a == per_head and own == bh * per_head + (first - 1) * 128 and there == bh * per_head + first * 128 + (far_tiles * far - 1) * 32


def test_parts_of_walks_that_are_split(places):
    (a, own, _), = places([(511, 64, 0, 0, 0, 65534, 510, 63)])
    assert a == 511 * 64 * 128 and own == 65534 * a + (510 * 64 + 63) * 128
