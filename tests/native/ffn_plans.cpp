// Prints the plans of the feed-forward unit's products on a device of 256 compute
// units: for bf16 or not, rows, channels, hidden and the strides of w_gate and w_up
// (the arguments) a line "product tile slices blocks" each.  Without arguments: the
// largest number of tiles that a product over the description's rows can have.  Built
// and run by tests/test_ffn_plans.py.
#include <cstdio>
#include <cstdlib>

#include "../../paper_2608_08330_amd/csrc/kernels/ffn_plan.hpp"

using namespace rtcc::kern;

int main(int argc, char **argv) {
    if (argc == 1) {
        int64_t most = 0;
        for (int64_t n = 8; n <= 65536; n += 8)
            for (Epilogue epi : {kPlain, kGated, kGatedGrad})
                for (Tiles kind : {kTiles256, kTiles128, kTiles64, kTiles64Deep})
                    most = std::max(most, tiles_of({std::min<int64_t>(2147483648 - 256, kMaxFfnValues / n), n}, kind, epi));
        std::printf("%lld\n", (long long)most);
        return 0;
    }
    if (argc != 7) return 2;
    FfnArgs a{};
    a.bf16 = std::atoi(argv[1]);
    a.rows = std::atoi(argv[2]);
    a.channels = std::atoi(argv[3]);
    a.hidden = std::atoi(argv[4]);
    a.w_gate_s = std::atoi(argv[5]);
    a.w_up_s = std::atoi(argv[6]);
    char any;
    auto say = [&](const char *product, const Plan &p, int64_t tiles) {
        std::printf("%s %d %d %lld\n", product, kSizeOf[p.kind], p.slices, (long long)tiles * p.slices);
    };
    const Size hidden{a.rows, a.hidden}, outer{a.rows, a.channels}, weight{a.hidden, a.channels}, down{a.channels, a.hidden};
    const int64_t cus = 256;
    Plan p = plan_gated(a, cus);
    say("gated", p, tiles_of(hidden, p.kind, kGated));
    a.gate = a.up = a.act = &any;
    p = plan_gated(a, cus);
    say("gated_saved", p, tiles_of(hidden, p.kind, kGated));
    p = plan_down(a, cus);
    say("down", p, tiles_of(outer, p.kind, kPlain));
    p = plan_dhidden(a, cus);
    say("dhidden", p, tiles_of(hidden, p.kind, kGatedGrad));
    a.dx = a.dw_gate = a.dw_up = a.dw_down = &any;
    const Backward b = plan_backward(a, cus);
    say(b.both ? "dx_shared" : "dx", b.x, tiles_of(outer, b.x.kind, kPlain));
    say(b.both ? "weights_shared" : "weights", b.w, 2 * tiles_of(weight, b.w.kind, kPlain) + tiles_of(down, b.w.kind, kPlain));
    return 0;
}
