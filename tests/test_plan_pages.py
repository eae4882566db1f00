"""Which pages a thread of the plan's kernel moves, in the source's own lines compiled for the CPU: each page once and none else, up to the most that a call may hold."""
import pytest

from tests import host_code

SOURCE = "bcq_plan.hip"
# `upto` of 1024 requests with `many` pages each (the last ones' sum cut to `all`); every page that is loaded is noted
PROGRAM = """
int main()
{
    const int all = ALL, many = MANY;
    static int upto[kThreads];
    for (int r = 0; r < kThreads; ++r) upto[r] = (int)std::min<i64>((i64)many * (r + 1), all);
    const int threads[] = {0, 1, 511, kThreads - 1};
    for (int t : threads) {
        threadIdx.x = t;
        i64 turns = 0, stored = 0;
        const auto check = [&](int k, int i, int j) {
            CHECK(k >= 0 && k < all);
            CHECK(i >= 0 && i < kThreads && k < upto[i] && (i == 0 || k >= upto[i - 1]));
            CHECK(j == k - (i ? upto[i - 1] : 0) && j < many);
        };
        move_pages(upto, all,
                   [&](int k, int i, int j) {
                       CHECK(++turns <= (i64)all / kThreads + 2 * kAtOnce);
                       check(k, i, j);
                       return k;
                   },
                   [&](int k, int i, int j, int page) {
                       check(k, i, j);
                       CHECK(page == k && k == t + stored * kThreads);
                       ++stored;
                   });
        CHECK(stored == (all > t ? ((i64)all - t - 1) / kThreads + 1 : 0));
    }
}
"""


# (the largest of a call: 1024 requests of 2097151 pages, one less than 2^31 in all)
@pytest.mark.parametrize("all_pages,many", [(0, 1), (1, 1), (1023, 1), (1024, 1), (1025, 2), (4095, 4), (4096, 4), (4097, 5), (100000, 98), (1024 * 2097151, 2097151), (2 ** 31 - 1, 2097152),
                                            (2 ** 31 - 4096, 2097152), (2 ** 31 - 4097, 2097152), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_each_page_once(all_pages, many, tmp_path):
    parts = [host_code.part(SOURCE, "kThreads = 1024"), host_code.part(SOURCE, "kAtOnce"), host_code.part(SOURCE, "__device__ __forceinline__ void first_beyond"),
             host_code.part(SOURCE, "__device__ __forceinline__ void move_pages")]
    host_code.run(tmp_path, *parts, PROGRAM.replace("ALL", str(all_pages)).replace("MANY", str(many)))
