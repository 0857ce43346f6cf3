// How many CTAs share the rows of a unit in the single-token kernels: plain host arithmetic.
#pragma once
#include <algorithm>

namespace shwin {

// How a launch is laid out: S CTAs (a cluster) share the rows of a unit.  A CTA of a kernel draws at most `rate`
// bytes/us, whatever bandwidth is left.
struct Shape {
    int S;
    double us;      // what the launch is expected to take
};
// CTAs run in waves of slots_of[log2 S], what the device holds at once of such clusters; those of a wave share the memory bandwidth (6.4 MB/us), and each costs about 2.5 us to start and to
// merge, half a microsecond more with each doubling of the cluster.  rows * row_bytes is what a unit may have to read.  The number of rows that a sequence really holds is known on the device
// only, so it is the cache's size that counts here.  A size of cluster that the device has no place for is left out; single CTAs always can be launched.
inline Shape best_split(long long units, long long rows, int row_bytes, const int (&slots_of)[4], double rate) {
    Shape best = {1, 1e300};
    for (int S = 1, i = 0; S <= 8 && (S == 1 || rows >= 64ll * S); S *= 2, ++i) {
        if (S > 1 && slots_of[i] < S) continue;
        const long long ctas = units * S, slots = std::max(slots_of[i], S), full = (ctas - 1) / slots, rest = ctas - full * slots;
        const double bytes = (double)rows * row_bytes / S;
        auto wave = [&](long long n) { return bytes / std::min(6.4e6 / (double)n, rate) + 2.5 + 0.5 * (S > 1) + 0.5 * (S > 2) + 0.5 * (S > 4); };
        const double us = (full ? full * wave(slots) : 0.0) + wave(rest);
        if (us < best.us) best = {S, us};
    }
    return best;
}

}  // namespace shwin
