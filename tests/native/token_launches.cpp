// The token operators' launch sizes over what their descriptions allow: every
// axis below 2^32 threads, all blocks covered, numbers of blocks below 2^31.
// Built and run by tests/test_token_launches.py.
#include <cstdio>

#include "../../paper_2608_08330_amd/csrc/kernels/token_ops.hpp"

using namespace rtcc::kern;

namespace {

int bad = 0;

void check(const char *what, int64_t blocks, int threads) {
    const Fold f = fold(blocks, threads);
    const int64_t all = int64_t(f.x) * f.z;
    const bool ok = blocks > 0 && blocks < (int64_t(1) << 31) && int64_t(f.x) * threads < (int64_t(1) << 32) && f.z >= 1 &&
                    f.z <= 65535 && all >= blocks && all - blocks < f.z && (blocks * threads >= (int64_t(1) << 32) || f.z == 1);
    if (!ok) {
        std::printf("%s: %lld blocks of %d threads: %u x %u\n", what, (long long)blocks, threads, f.x, f.z);
        ++bad;
    }
}

}  // namespace

int main() {
    const int64_t kMax = 2147483647;  // past all the limits of rows and q_rows * q_heads
    for (int heads : {1, 3, 256, 1024})
        for (int group : {1, 4, 1024}) {
            if (int64_t(heads) * group > 1024) continue;
            for (int seqs : {1, 1000, 65536})
                for (int64_t rows : {int64_t(1), int64_t(65536), kMax / 2, kMax}) {
                    AttnArgs a{};
                    a.kv_heads = heads, a.group = group, a.q_heads = heads * group, a.n_seqs = seqs;
                    a.q_rows = int32_t(rows < kMax / a.q_heads ? rows : kMax / a.q_heads);
                    a.k_rows = int32_t(rows < (kMaxGradKeys - 1) / heads ? rows : (kMaxGradKeys - 1) / heads);
                    check("tiles", column_blocks(a, 128), 256);
                    check("few", column_blocks(a, 32), 128);
                    check("few", column_blocks(a, 32), 256);
                    check("join", column_blocks(a, 16), 256);
                    check("dq", column_blocks(a, 64), 256);
                    check("dkv", key_blocks(a, 64), 256);
                    // tiles of 64 sequences of the whole batch each, in 32 bits
                    if (64 * row_tiles(int64_t(a.q_rows) * group, 64) > (int64_t(1) << 31) ||
                        64 * row_tiles(a.k_rows, 64) > (int64_t(1) << 31))
                        ++bad;
                }
        }
    for (int per : {32, 64, 128, 256})
        for (int64_t rows : {int64_t(1), int64_t(255), kMax - 255, kMax}) {
            const int64_t tiles = row_tiles(rows, per);
            check("rows", tiles, 256);
            if (tiles * per < rows || (tiles - 1) * per >= rows) ++bad;
            // a thread's row, counted in 32 bits without a sign
            const Fold f = fold(tiles, 256);
            if (int64_t(f.x) * f.z * per > (int64_t(1) << 32)) ++bad;
        }
    std::printf("%d\n", bad);
    return bad != 0;
}
