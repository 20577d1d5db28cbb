// Host arithmetic of mpt_distill_topk's kernel for long rows, free of CUDA so that it can be tested without a device.
#pragma once

namespace mpt {

constexpr int kDistillClusters = 4;       // clusters of 1, 2, 4 or 8 CTAs

// log2 of the CTAs of a cluster that share a row of C classes, B rows; -1: no cluster fits the device.  known: clusters of each
// size that are resident at once, one CTA on an SM, of ONE kernel on ONE device (0: not asked yet, -1: none).  resident(ctas)
// asks for that number: below 0 for an error, which is asked again the next time.  Sizes that do not fit are left out.
// Chosen is the least of rounds of rows times what a row takes, in classes: its share of a CTA and what it costs besides
// (measured with 131072 classes: 0.138 ns a class and 0.3, 1.0, 1.8 and 2.5 us a row; 512 x 793471 takes 434, 366 and 418 us in
// clusters of 1, 2 and 4, 700 x 131072 takes 90, 102 and 137, 10 x 250000 takes 22, 15 and 12 us in clusters of 2, 4 and 8).
template <typename Resident>
inline int distill_cluster_log2(int (&known)[kDistillClusters], int B, int C, Resident resident)
{
    constexpr int besides[kDistillClusters] = {2000, 7000, 13000, 18000};
    double least = 0.0;
    int best = -1;
    for (int i = 0; i < kDistillClusters; i++) {
        if (known[i] == 0) {
            const int n = resident(1 << i);
            if (n >= 0) known[i] = n > 0 ? n : -1;
        }
        if (known[i] <= 0) continue;
        const double cost = (double)((B - 1) / known[i] + 1) * ((double)C / (1 << i) + besides[i]);
        if (best < 0 || cost < least) {
            least = cost;
            best = i;
        }
    }
    return best;
}

}  // namespace mpt
