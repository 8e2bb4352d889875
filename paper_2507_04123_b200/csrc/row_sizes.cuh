// How the operators on dispatched rows divide a row over lanes, and how large the scratch of the lookup's gradient is.  Host
// arithmetic without CUDA, so that the CPU tests exercise these lines and not a copy of them.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace emc2 {

constexpr int kLookupThreads = 256;
constexpr int kRunItems = 16;                 // sorted places per group of lanes, at least
constexpr int kSortItems = 2048;              // ids of a tile of the sort
constexpr int kMaxDigits = 1024;

// A row of nvec vectors of four elements is spread over 1 << log lanes that hold up to `per` vectors each (vector
// lane + i * lanes): the split that leaves fewest places empty with at most `most` vectors per lane (or what 32 lanes need),
// and of those the one with fewest lanes, since the more a lane loads at once, the more is in flight.
struct RowSplit {
    int log, per;
};
inline RowSplit row_split(int nvec, int most) {
    RowSplit best = {5, (nvec + 31) / 32};
    for (int log = 4; log >= 0; --log) {
        const int lanes = 1 << log, per = (nvec + lanes - 1) / lanes;
        if (per <= most && per * lanes <= best.per << best.log) best = {log, per};
    }
    return best;
}

// What a part of the sorted list leaves of the runs that its ends divide.
struct RunEnds {
    int head;                   // id of a run that begins before the part, or -1
    int through;                // that run also goes on behind the part
    int tail;                   // id of a run that begins in the part and goes on behind it, or -1
    int pad;
};

// How the sum over the sorted list is divided: groups of lanes in a CTA, places of a group (a multiple of kRunItems), CTAs.
// As many places as make about four CTAs per SM, so that their ends do not weigh.
struct LookupParts {
    int groups, items, ctas;
};
inline LookupParts lookup_parts(int num_sms, long long n, int nvec) {
    LookupParts p;
    p.groups = kLookupThreads >> row_split(nvec, 3).log;
    const long long most = (long long)p.groups * 4 * num_sms;
    p.items = (int)(std::max<long long>(1, (n + most * kRunItems - 1) / (most * kRunItems)) * kRunItems);
    p.ctas = (int)((n + (long long)p.items * p.groups - 1) / ((long long)p.items * p.groups));
    return p;
}

// Scratch of the gradient for n ids and rows of nvec vectors, as offsets.
struct LookupScratch {
    size_t keys[2], vals[2], counts, row_tot, ends, partial, bytes;
};
inline LookupScratch lookup_scratch(long long n, int ctas, int nvec) {
    LookupScratch s;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += (bytes + 255) & ~(size_t)255; return o; };
    for (int k = 0; k < 2; ++k) { s.keys[k] = take((size_t)n * 4); s.vals[k] = take((size_t)n * 4); }
    s.counts = take((size_t)kMaxDigits * ((n + kSortItems - 1) / kSortItems + 3) * 4);
    s.row_tot = take(kMaxDigits * 4);
    s.ends = take((size_t)ctas * sizeof(RunEnds));
    s.partial = take((size_t)ctas * 2 * nvec * 16);
    s.bytes = off;
    return s;
}

// The most CTAs that a call of up to n ids has.  Their number falls wherever n is large enough for more places per group, so
// the handle's own n is not the one that has most; but there are never more than four per SM, nor fewer places than kRunItems.
inline int most_lookup_ctas(int num_sms, long long n, int nvec) {
    const long long per_cta = (long long)lookup_parts(num_sms, n, nvec).groups * kRunItems;
    return (int)std::min<long long>(4LL * num_sms, (n + per_cta - 1) / per_cta);
}

// What every call of up to n ids and max_channels channels fits in.
inline size_t lookup_scratch_most(int num_sms, long long n, int max_channels) {
    size_t most = 0;
    // Narrower rows have more groups per CTA, so fewer CTAs: which width needs most depends on n.
    for (int c = 4; c <= max_channels; c += 4) most = std::max(most, lookup_scratch(n, most_lookup_ctas(num_sms, n, c / 4), c / 4).bytes);
    return most;
}

}  // namespace emc2
