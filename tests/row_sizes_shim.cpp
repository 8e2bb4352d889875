// csrc/row_sizes.cuh for the CPU tests: its functions behind a C interface.
#include "row_sizes.cuh"

using namespace emc2;

extern "C" {

int parts(int num_sms, int64_t n, int channels, int* items) {
    const LookupParts p = lookup_parts(num_sms, n, channels / 4);
    *items = p.items;
    return p.ctas;
}
int groups(int channels) { return lookup_parts(1, 1, channels / 4).groups; }
uint64_t need(int num_sms, int64_t n, int channels) {
    return lookup_scratch(n, lookup_parts(num_sms, n, channels / 4).ctas, channels / 4).bytes;
}
uint64_t most(int num_sms, int64_t n, int max_channels) { return lookup_scratch_most(num_sms, n, max_channels); }

// Largest need of calls of n0 .. n1 ids and up to max_channels channels, over every number of ids.
uint64_t largest_need(int num_sms, int64_t n0, int64_t n1, int channels) {
    uint64_t m = 0;
    for (int64_t n = n0; n <= n1; ++n) m = std::max(m, need(num_sms, n, channels));
    return m;
}

}
