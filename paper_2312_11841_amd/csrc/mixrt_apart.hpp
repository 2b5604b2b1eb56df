// Whether two arrays of a call share memory: pure host arithmetic on their addresses.
#pragma once

#include <stdint.h>

namespace mixrt {

// Runs of `run` bytes from address `at` on, repeated n[j] times `step[j]` bytes (at
// least 0) apart in each of three dimensions.
struct Extent {
    uint64_t at;
    int64_t run;
    int64_t n[3], step[3];
};

inline Extent flat_extent(const void *p, int64_t bytes)
{
    return Extent{(uint64_t)(uintptr_t)p, bytes, {1, 1, 1}, {0, 0, 0}};
}

inline bool empty_extent(const Extent &e)
{
    return e.at == 0 || e.run <= 0 || e.n[0] <= 0 || e.n[1] <= 0 || e.n[2] <= 0;
}

// Whether two arrays certainly share no byte: one lies behind the other, or both
// repeat with some step and take other parts of it (slices of one joint array).
inline bool apart(const Extent &a, const Extent &b)
{
    if (empty_extent(a) || empty_extent(b)) return true;
    const Extent *both[2] = {&a, &b};
    int64_t span[2];
    for (int i = 0; i < 2; ++i) {
        span[i] = both[i]->run;
        for (int j = 0; j < 3; ++j) span[i] += (both[i]->n[j] - 1) * both[i]->step[j];
    }
    if (a.at < b.at ? b.at - a.at >= (uint64_t)span[0] : a.at - b.at >= (uint64_t)span[1])
        return true;
    const int64_t diff = (int64_t)(b.at - a.at);
    for (int c = 0; c < 6; ++c) {
        const int64_t s = both[c / 3]->step[c % 3];
        if (s <= 0 || both[c / 3]->n[c % 3] == 1) continue;
        int64_t part[2];        // of a repetition
        for (int i = 0; i < 2; ++i) {
            part[i] = both[i]->run;
            for (int j = 0; j < 3; ++j)
                if (both[i]->step[j] % s) part[i] += (both[i]->n[j] - 1) * both[i]->step[j];
        }
        const int64_t m = (diff % s + s) % s;
        if (m >= part[0] && m + part[1] <= s) return true;
    }
    return false;
}

// The arrays of a call, to find outputs that share memory with another.
struct Arrays {
    struct One {
        Extent e;
        const char *name;
        bool out;
    };
    One a[20];
    int n = 0;
    void add(const Extent &e, const char *name, bool out = false)
    {
        if (!empty_extent(e)) a[n++] = One{e, name, out};
    }
    // an array that an output shares memory with, or NULL
    const One *shared() const
    {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j)
                if (i != j && a[i].out && !apart(a[i].e, a[j].e)) return &a[i];
        return nullptr;
    }
};

}  // namespace mixrt
