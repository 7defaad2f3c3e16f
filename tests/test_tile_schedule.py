"""Copies into LDS ahead of their use: what is read has arrived, and nothing is overwritten that is still to be read (CPU: the rules are plain C++)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# A wave's copies in order of issue, each (tile, K-tile, buffer); a wait with N in flight means that all but the last N have arrived.
# All waves run the same schedule and meet behind each wait, so what one of them has waited for is there for all.
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "tile_schedule.h"
using namespace dcnn;
struct Copy { int tile, kt, buf; };
int main() {
    int bad = 0;
    for (int nb = 2; nb <= 4; ++nb)
        for (int kts = 1; kts <= 3 * nb + 1; ++kts)
            for (int tiles = 1; tiles <= 4; ++tiles) {
                std::vector<Copy> issued;
                size_t arrived = 0;
                auto wait = [&](int in_flight) { if (issued.size() - in_flight > arrived && (int)issued.size() >= in_flight) arrived = issued.size() - in_flight; };
                auto holds = [&](int tile, int kt) {             // the last copy into the buffer of K-tile kt is that one, and it has arrived
                    for (size_t i = issued.size(); i-- > 0;)
                        if (issued[i].buf == kt % nb) return issued[i].tile == tile && issued[i].kt == kt && i < arrived;
                    return false;
                };
                auto wrong = [&](int tile, int kt) {
                    if (bad++ < 20) printf("%d buffers, %d K-tiles, %d tiles: tile %d K-tile %d is not there\n", nb, kts, tiles, tile, kt);
                };
                int ahead = 0;
                for (int kt = 0; kt < nb && kt < kts; ++kt) issued.push_back({0, kt, kt});
                wait((kts < nb ? kts : nb) - 1);
                for (int tile = 0; tile < tiles; ++tile) {
                    const int there = tile == 0 ? 1 : nb;          // K-tiles that have been waited for before the tile begins
                    if (!holds(tile, 0)) wrong(tile, 0);
                    for (int kt = 0; kt < kts; ++kt) {
                        if (kt + 1 >= there) wait(may_be_in_flight(kt, kts, nb, ahead < tiles));
                        if (kt + 1 < kts && !holds(tile, kt + 1)) wrong(tile, kt + 1);
                        if (turns_to_next(kt, kts, nb)) ++ahead;
                        if (ahead < tiles) issued.push_back({ahead, copied_behind(kt, kts, nb), kt % nb});
                    }
                    wait(0);
                }
                if ((int)issued.size() != tiles * kts) {           // each once
                    ++bad;
                    printf("%d buffers, %d K-tiles, %d tiles: %zu copies\n", nb, kts, tiles, issued.size());
                }
            }
    return bad != 0;
}
"""


def test_k_tiles_are_there_when_they_are_read(tmp_path):
    src = tmp_path / "schedule.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "schedule"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2203_03996_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


ROWS = r"""
#include <cstdio>
#include <initializer_list>
#include "tile_schedule.h"
using namespace dcnn;
int main() {
    int bad = 0;
    const int tops[] = {0, 1, 2, 31, 32, 63, 64, 65, 127, 128, 255, 256, 257, 1 << 24, 0x7ffffeff, 0x7fffff00, 0x7fffff01, 0x7fffff80, 0x7fffff81, 0x7fffffc1, 0x7ffffffe, 0x7fffffff};
    for (int per : {32, 64, 128, 256})
        for (int rows : tops) {
            const long long tiles = tiles_of(rows, per);
            if (tiles * per < rows || (tiles - 1) * per >= rows) ++bad, printf("%d rows in tiles of %d: %lld\n", rows, per, tiles);
            if (rows == 0) continue;
            const int t0 = (int)((tiles - 1) * per);             // the last tile
            for (int r = 0; r < per; ++r)
                if (in_rows(t0, r, rows) != ((long long)t0 + r < rows)) ++bad, printf("%d rows: row %d of the tile at %d\n", rows, r, t0);
        }
    return bad != 0;
}
"""


def test_tiles_of_the_longest_calls(tmp_path):
    """Up to 2^31 - 1 rows: sums that pass 32 bits would leave a call without tiles, or its last rows' scales to be read from elsewhere."""
    src = tmp_path / "rows.cpp"
    src.write_text(ROWS)
    exe = tmp_path / "rows"
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2203_03996_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
