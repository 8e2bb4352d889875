// The same call of the library from two host threads at once, each with its own handle: for tests/test_gpu_two_threads.py.
#include <atomic>
#include <cstdint>
#include <thread>

extern "C" {

struct FfnCall {
    void* bridge;
    int32_t B, N, channels, hidden, type, act;
    const void *x, *offsets, *gate, *up, *down;
    void *y, *stream;
};
using Ffn = int (*)(void*, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, const void*, const void*, const void*, const void*, const void*, void*, void*);

struct NormGradCall {
    void* bridge;
    int32_t B, N, channels, type_x, type_y;
    const void *x, *offsets, *weight, *mean, *rstd, *dy;
    void *dx, *dweight, *dbias, *stream;
};
using NormGrad = int (*)(void*, int32_t, int32_t, int32_t, int32_t, int32_t, const void*, const void*, const void*, const void*, const void*, const void*, void*, void*,
                         void*, void*);

struct LookupGradCall {
    void* bridge;
    int32_t n, rows, channels, type;
    const void *ids, *dout;
    float scale;
    void *dtable, *stream;
};
using LookupGrad = int (*)(void*, int32_t, int32_t, int32_t, int32_t, const void*, const void*, float, void*, void*);

}

namespace {

// `times` calls in each thread; the first that failed, or 0.
template <typename Call>
int both(const Call& a, const Call& b, int times) {
    std::atomic<int> first{0}, ready{0};
    auto run = [&](const Call& call) {
        ++ready;
        while (ready < 2) {}
        for (int i = 0; i < times && first == 0; ++i)
            if (const int rc = call()) { int none = 0; first.compare_exchange_strong(none, rc); }
    };
    std::thread other([&] { run(b); });
    run(a);
    other.join();
    return first;
}

template <typename C, typename F>
int two(const C* c, int times, const F& call) {
    struct Bound {
        const C* c;
        const F* f;
        int operator()() const { return (*f)(*c); }
    };
    return both(Bound{c, &call}, Bound{c + 1, &call}, times);
}

}  // namespace

extern "C" {

int two_ffn(void* f, const FfnCall* c, int times) {
    return two(c, times, [f](const FfnCall& a) {
        return reinterpret_cast<Ffn>(f)(a.bridge, a.B, a.N, a.channels, a.hidden, a.type, a.act, a.x, a.offsets, a.gate, a.up, a.down, a.y, a.stream);
    });
}
int two_norm_grad(void* f, const NormGradCall* c, int times) {
    return two(c, times, [f](const NormGradCall& a) {
        return reinterpret_cast<NormGrad>(f)(a.bridge, a.B, a.N, a.channels, a.type_x, a.type_y, a.x, a.offsets, a.weight, a.mean, a.rstd, a.dy, a.dx, a.dweight, a.dbias, a.stream);
    });
}
int two_lookup_grad(void* f, const LookupGradCall* c, int times) {
    return two(c, times, [f](const LookupGradCall& a) {
        return reinterpret_cast<LookupGrad>(f)(a.bridge, a.n, a.rows, a.channels, a.type, a.ids, a.dout, a.scale, a.dtable, a.stream);
    });
}

}
