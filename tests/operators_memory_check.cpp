// The operators' C entry points while host memory is short: one allocation after the other fails, and each call has to come back with a
// status.  Calls that are refused before anything is launched, so that no GPU is needed.
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <new>

#include "../include/klay.h"

static long countdown = -1;         // allocations until one fails; < 0: none does

void* operator new(std::size_t n) {
    if (countdown >= 0 && countdown-- == 0) throw std::bad_alloc();
    if (void* p = std::malloc(n ? n : 1)) return p;
    throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main() {
    klay_tokens_args t = {};
    t.dtype = 9;
    klay_tokens_args many = {};
    many.vocab = 10;
    many.num_tokens = 5000;
    klay_scan_args s = {};
    s.semiring = 7;
    float x[8] = {};
    const struct { const char* name; std::function<klay_status()> call; } calls[] = {
        {"tokens_forward", [&] { return klay_tokens_forward(&t, x, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr); }},
        {"tokens_forward, 5000 tokens", [&] { return klay_tokens_forward(&many, x, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr); }},
        {"tokens_backward", [&] { return klay_tokens_backward(&t, x, x, nullptr, nullptr, x, nullptr); }},
        {"scan_forward", [&] { return klay_scan_forward(&s, x, nullptr, nullptr, 0, nullptr); }},
        {"scan_backward", [&] { return klay_scan_backward(&s, x, x, nullptr, x, x, nullptr, nullptr, 0, nullptr); }},
        {"scan_step", [&] { return klay_scan_step(0, 5, 0, 1, 1, x, 1, x, 1, x, 1, x, 1, nullptr); }},
    };
    int bad = 0;
    for (const auto& c : calls) {
        bool failed = false;
        for (long n = 0; n < 8; ++n) {
            klay_status st = KLAY_OK;
            try {
                countdown = n;
                st = c.call();
                failed = failed || countdown < 0;
            } catch (...) {
                std::printf("%s: an exception came out of the call (allocation %ld)\n", c.name, n);
                ++bad;
            }
            countdown = -1;
            if (st != KLAY_EINVAL && st != KLAY_ENOMEM && !bad) {
                std::printf("%s: status %d (allocation %ld)\n", c.name, (int)st, n);
                ++bad;
            }
        }
        if (!failed) {
            std::printf("%s: no allocation failed\n", c.name);
            ++bad;
        }
        if (c.call() != KLAY_EINVAL) ++bad;
    }
    std::printf(bad ? "%d bad\n" : "ok\n", bad);
    return bad ? 1 : 0;
}
