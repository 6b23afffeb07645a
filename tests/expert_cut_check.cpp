// The cut of the experts' factors (expert_cut.h), on the CPU: whatever rows the experts get, their ranges, partial sums and experts of several
// ranges are no more than the launch and the scratch are made for, no range is empty or longer than rows_per, and a range's bytes fit 32 bits.
#include <cstdio>
#include <random>
#include <vector>

#include "../paper_1811_12019_amd/csrc/expert_cut.h"

using namespace kfac;

int main() {
    std::mt19937 rng(1);
    auto up_to = [&](long long n) { return (long long)(rng() % (unsigned long long)n); };
    auto spread = [&](double lo, double hi) { return (int)std::exp(std::log(lo) + (std::log(hi) - std::log(lo)) * (rng() / 4294967296.0)); };
    int faults = 0;
    long long checked = 0;
    for (int trial = 0; trial < 20000; ++trial) {
        kfac_expert_factor_desc d = {};
        d.rows = trial % 10 == 0 ? (int)up_to(4) : trial % 10 == 1 ? spread(1e5, 2e9) : spread(1, 2e5);
        d.experts = trial % 7 == 0 ? 1 : spread(1, 1024.9);
        d.dim = trial % 5 == 0 ? spread(1, 32766) : spread(1, 4096);
        d.dtype = (int)up_to(3);
        d.has_bias = (int)up_to(2);
        if (up_to(3) == 0) d.ld = d.dim + up_to(40);
        if (up_to(50) == 0) d.ld = std::max((long long)d.dim, (1ll << 18) - 8 + up_to(17));
        if (!expert_factor_ok(&d)) { ++faults; continue; }
        const ExpertCut c = expert_cut(d);
        const int es = d.dtype == KFAC_F32 ? 4 : 2, most_rows = d.dtype == KFAC_F32 ? ROWS_PER_WG_MAX_F32 : ROWS_PER_WG_MAX;
        auto want = [&](bool ok, const char* what) {
            if (!ok && ++faults <= 20)
                printf("%s: rows %d experts %d dim %d dtype %d ld %lld: rows_per %d tw %d\n", what, d.rows, d.experts, d.dim, d.dtype, (long long)d.ld, c.rows_per, c.tw);
        };
        want(c.rows_per >= 64 && c.rows_per % 64 == 0 && c.rows_per <= (most_rows + 63) / 64 * 64, "rows of a range");
        want((c.tw == 64 || c.tw == 128 || (c.tw == 256 && es == 2)) && (long long)c.tiles_dim * c.tw >= d.dim && (long long)(c.tiles_dim - 1) * c.tw < d.dim, "width");
        want(c.ntiles == c.tiles_dim * (c.tiles_dim + 1) / 2 && c.tile_floats == tile_floats(c.tw, c.ntiles), "tiles");
        want(c.ld % (16 / es) == 0 && c.ld >= d.dim && c.ld <= EXPERT_LD_MAX, "distance of rows");
        want((long long)(c.rows_per + 512) * c.ld * es < 0xFFFFFFF0ll || es == 4, "bytes of a range");      // (512: slabs fetched ahead)
        want(!c.pad || c.pad_bytes >= (size_t)d.rows * c.ld * es, "copy");
        want(c.tile_bytes >= (size_t)c.parts * c.ntiles * c.tile_floats * 4 && (!d.has_bias || c.sum_bytes >= (size_t)c.parts * c.tiles_dim * c.tw * 4), "scratch");
        // Rows of the experts: equal, one's, as few as make a second range, one more than whole ranges, any.
        for (int how = 0; how < 6; ++how) {
            long long left = d.rows, ranges = 0, parts = 0, splits = 0;
            for (int e = 0; e < d.experts; ++e) {
                long long rows = how == 0 ? (long long)d.rows * (e + 1) / d.experts - (long long)d.rows * e / d.experts
                               : how == 1 ? (e == d.experts / 2 ? left : 0)
                               : how == 2 ? c.rows_per + 1
                               : how == 3 ? c.rows_per * (1 + up_to(5)) + 1
                               : how == 4 ? up_to(2ll * d.rows / d.experts + 1)
                                          : c.rows_per * up_to(4) + up_to(3);
                rows = std::min(rows, left);
                if (how >= 2 && e == d.experts - 1) rows = left;
                left -= rows;
                const long long n = (rows + c.rows_per - 1) / c.rows_per;
                ranges += std::max(n, 1ll);
                parts += n > 1 ? n : 0;
                splits += n > 1;
                if (n > 0) {                                             // as the tile kernel cuts an expert's rows
                    const long long each = ((rows + n - 1) / n + 63) / 64 * 64;
                    want(each <= c.rows_per && (n - 1) * each < rows, "an expert's ranges");
                }
            }
            want(ranges <= c.ranges && parts <= c.parts && splits <= c.splits, "ranges, partial sums");
            ++checked;
        }
    }
    printf("%lld cuts, %d faults\n", checked, faults);
    return faults != 0;
}
