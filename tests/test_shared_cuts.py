"""How the blocks of both lines of shared prefixes are cut into workgroups' pieces, in the source's own lines compiled for the CPU: each block in one piece, and found again by
its number."""
from tests import host_code

SOURCE = "bcq_attend_shared.hip"
PROGRAM = """
void check(const Cut &c, int total, int most0, int most1)
{
    const int pieces = c.w0 + c.w1;
    CHECK(c.total == total && c.w0 <= std::max(most0, 1) && c.w1 <= std::max(most1, 1));
    int at = 0;
    for (int i = 0; i < pieces; ++i) {
        if (i < c.w0 ? most0 == 0 : most1 == 0) {
            CHECK(c.end(i) == c.begin(i));
            continue;
        }
        CHECK(c.begin(i) == at && c.end(i) >= at);
        at = c.end(i);
        for (int b : {c.begin(i), (c.begin(i) + c.end(i)) / 2, c.end(i) - 1})
            if (b >= c.begin(i) && b < c.end(i)) CHECK(c.piece_of(b) == i);
    }
    CHECK(at == total);
}

int main()
{
    const int blocks[] = {0, 1, 2, 3, 5, 15, 16, 17, 31, 32, 33, 44, 63, 64, 65, 100, 127, 128, 129, 208, 500, 1000, 4097, 33333, 1000003, 1 << 30, 0x7fffffff};
    for (int workers = 1; workers <= 512; workers += workers < 70 ? 1 : 17) {
        const int half = workers / 2, rest = workers - half;
        for (int tiles : blocks)
            for (int few : blocks) {
                const Cuts c(half, rest, tiles, few);
                check(c.tiles, tiles, half, rest);
                check(c.few, few, kTileWaves * rest, kTileWaves * half);
            }
    }
}
"""


def test_pieces(tmp_path):
    parts = [host_code.part("bcq_attend_tile.h", "kTileWaves = 4"), host_code.part(SOURCE, "struct Cut {"), host_code.part(SOURCE, "struct Cuts {")]
    host_code.run(tmp_path, *parts, PROGRAM)
