// Blocks of the feed-forward unit's products over what its description allows: every
// axis below 2^32 threads, all blocks covered, numbers of blocks below 2^31.  Built and
// run by tests/test_ffn_launches.py.
#include <cstdio>

#include "../../paper_2608_08330_amd/csrc/kernels/token_ops.hpp"

using namespace rtcc::kern;

int main() {
    int bad = 0;
    const int64_t most_rows = 2147483648 - 256;
    for (int64_t width : {int64_t(8), int64_t(72), int64_t(512), int64_t(4096), int64_t(65536)})
        for (int64_t rows : {int64_t(1), int64_t(65), most_rows}) {
            const int64_t n = rows * width <= kMaxFfnValues ? rows : kMaxFfnValues / width;
            for (int cols : {32, 64, 128, 256}) {  // 32: half a tile of 64, of a gated product
                const int tall = cols < 64 ? 64 : cols;
                const int64_t blocks = row_tiles(n, tall) * row_tiles(width, cols);
                const Fold f = fold(blocks, 256);
                const int64_t all = int64_t(f.x) * f.z;
                if (blocks >= (int64_t(1) << 31) || int64_t(f.x) * 256 >= (int64_t(1) << 32) || f.z > 65535 || all < blocks ||
                    all >= (int64_t(1) << 31) || row_tiles(n, tall) * tall - 1 > 2147483647) {
                    std::printf("%lld x %lld by %d: %lld blocks, %u x %u\n", (long long)n, (long long)width, cols,
                                (long long)blocks, f.x, f.z);
                    ++bad;
                }
            }
        }
    std::printf("%d\n", bad);
    return bad != 0;
}
