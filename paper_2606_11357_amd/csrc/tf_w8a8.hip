// Which kernel an 8-bit matrix product runs on: the one expected to be done first.
#include <algorithm>

#include "tf_w8a8.h"

namespace tf {

int launch_w8a8_direct(const W8Args& a, hipStream_t s);
int launch_w8a8_tile(const W8Args& a, int form, hipStream_t s);

namespace {

// Expected times, us, fitted to K = 4096 and 14336 with N = 4096, 6144 and 28672 on
// MI355X, weights from memory; measured / expected for some of them, M x K x N:
//   direct       16 x 14336 x 4096     17.3 / 17.4   (tiles of 64 x 64: 26)
//   64 x 64      256 x 4096 x 4096      9.7 / 11     (64 x 128: 12.1)
//   64 x 128     400 x 4096 x 4096     11.7 / 14     (64 x 64: 14.6, 128 x 128: 16.0)
//   128 x 128    400 x 4096 x 6144     17.6 / 18     (64 x 128: 20.0, 128 x 256: 25.8)
//   128 x 256    1500 x 14336 x 4096   97.0 / 100    (256 x 256: 129, 128 x 128: 121)
//   256 x 256    1500 x 4096 x 28672   171 / 129     (128 x 256: 190, 128 x 128: 223)
// A tile's step of 64 of K takes what its operands take through a compute unit's L1, some
// 25 bytes a cycle (misses in the L2 bound it, not the number of loads on their way:
// twice the depth changes nothing); 256 x 256 is the one that the matrix cores bound.
// Its step is that of few tiles: with all compute units at work the power's limit on the
// clock makes it a third longer (171 us of 129 above), which the rule leaves out.
constexpr int kForms = 5;
struct FormCost {
    int bm, bn, wgs;
    double start, step, rows;      // a tile's start; a step's time without A, and A's share of it
};
constexpr FormCost kForm[kForms] = {{256, 256, 1, 7.0, 0.56, 0.0},
                                    {128, 256, 1, 0.0, 0.31, 0.13},
                                    {128, 128, 1, 0.0, 0.18, 0.09},
                                    {64, 128, 2, 0.0, 0.15, 0.06},
                                    {64, 64, 2, 0.0, 0.10, 0.06}};

}  // namespace

namespace {

struct Plan {
    int kernel;              // a form, or kForms: the direct one
    int splits;
    double expected;
};

// K is split for 64 x 64 tiles, into 2 or 4 parts where `ws_bytes` hold their sums: few
// rows by few columns with long K, whose tiles leave most compute units idle (64 x 14336
// x 4096 35.7 -> 18.7 us, 128 rows 35.1 -> 25.2; K = 4096 9.1 -> 10.1, so not there; up to
// 16 rows the direct kernel, 17.9 us with its codes, 21.3 split).  The sums' way through
// memory and the launch that adds them take some 8 us, more where calls are short.
Plan plan_w8a8(int64_t M, int64_t K, int64_t N, int64_t experts, double cus, int64_t ws_bytes) {
    const int64_t weights = experts ? std::min(experts, M) : 1;
    const int64_t rows = (M + weights - 1) / weights;        // of one weight, on average
    const double memory = (double)weights * (double)K * (double)N / 5.0e6;
    const double steps = (double)((K + 127) / 128 * 2);
    // Where the memory's rate decides, the smallest tiles that leave it some room: their
    // loads come from more places at once (500 tokens, 6 of 64 experts, 2048 x 2000: 64 x
    // 128 56 us, 128 x 256 70; one row, 4096 x 28672: 64 x 64 22.7, 128 x 128 29.7).
    const double floor = 3.0 + memory;
    double least = 1e30;
    Plan best{0, 1, 0.0};
    auto offer = [&](int kernel, int splits, double alone) { // `alone`: were it not for the memory's rate
        const double t = alone <= 0.8 * floor ? 0.8 * floor : alone;
        if (t <= least) best = {kernel, splits, std::max(t, floor)}, least = t;
    };
    for (int f = 0; f < kForms; ++f) {
        const FormCost& c = kForm[f];
        // experts' rows are ragged: half a tile more of each
        const double tiles_m = experts ? (double)weights * std::max(1.0, (double)rows / c.bm + 0.5)
                                       : (double)((rows + c.bm - 1) / c.bm);
        const double tiles = tiles_m * (double)((N + c.bn - 1) / c.bn);
        const double step = c.step + c.rows * std::min<double>((double)rows, c.bm) / c.bm;
        double rounds = std::max(1.0, (double)(int64_t)((tiles + cus - 1) / cus));
        if (c.wgs == 2 && rounds > 1) rounds -= 0.4;         // two at a time hide part of each other
        offer(f, 1, 1.0 + rounds * (c.start + steps * step));
    }
    if (rows <= 48)
        offer(kForms, 1, 2.6 + memory * (rows <= 16 ? 0.95 + 0.02 * (double)rows : 0.85 * (double)((rows + 15) / 16)));
    if (!experts && M > 16) {
        const FormCost& c = kForm[kForms - 1];
        const double tiles = (double)((M + c.bm - 1) / c.bm * ((N + c.bn - 1) / c.bn));
        for (const int splits : {2, 4}) {
            const int64_t bytes = splits * M * N * 4;
            if (bytes > ws_bytes || steps < 32.0 * splits) continue;
            const double rounds = std::max(1.0, (double)(int64_t)((tiles * splits + cus - 1) / cus));
            const double step = c.step + c.rows * std::min<double>((double)M, c.bm) / c.bm;
            const double alone = 11.0 + rounds * steps / splits * step + (double)bytes / 2.0e6;
            if (alone < least) offer(kForms - 1, splits, alone);
        }
    }
    return best;
}

constexpr double kCus = 256;

}  // namespace

int64_t w8a8_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    const Plan p = plan_w8a8(M, K, N, 0, kCus, INT64_MAX);
    return p.splits > 1 ? p.splits * M * N * 4 : 0;
}

int launch_w8a8(W8Args a, void* ws, int64_t ws_bytes, hipStream_t s) {
    const Plan p = plan_w8a8(a.M, a.K, a.N, a.experts, (double)device_cus(s), ws ? ws_bytes : 0);
    a.splits = p.splits;
    a.parts = static_cast<int32_t*>(ws);
    if (log_enabled())
        log_plan("w8a8 M=%lld K=%lld N=%lld experts=%d%s: %s, %d x %d tiles, K in %d, expected %.1f us", (long long)a.M,
                 (long long)a.K, (long long)a.N, a.experts, a.rows ? " gathered" : "",
                 p.kernel < kForms ? "w8a8_tile_kernel" : "w8a8_direct_kernel", p.kernel < kForms ? kForm[p.kernel].bm : 16,
                 p.kernel < kForms ? kForm[p.kernel].bn : 16, p.splits, p.expected);
    return p.kernel < kForms ? launch_w8a8_tile(a, p.kernel, s) : launch_w8a8_direct(a, s);
}

}  // namespace tf
