// OncePerDevice on the host: each device is set for itself, a failure is tried again,
// and threads that begin together all come out with their device set.
#include <cstdio>
#include <thread>
#include <vector>

#include "once_per_device.h"

static int failures = 0;
static void expect(bool ok, const char *what)
{
    if (!ok) ++failures, printf("%s\n", what);
}

int main()
{
    ar::OncePerDevice once;
    int set[66] = {}, failing = 0;
    auto call = [&](int device) { return once(device, [&] { return ++set[device], failing == 0; }); };
    expect(call(0) && call(0) && set[0] == 1, "the first device, once");
    expect(call(1) && call(1) && set[1] == 1, "the second device, for itself");
    failing = 1;
    expect(!call(2) && !call(2) && set[2] == 2, "a failure is reported, and tried again");
    expect(call(0) && set[0] == 1, "another device's failure changes nothing");
    failing = 0;
    expect(call(2) && call(2) && set[2] == 3, "and not after it has succeeded");
    expect(call(63) && call(63) && set[63] == 1, "the last one that is remembered");
    expect(call(65) && call(65) && set[65] == 2, "one beyond");
    ar::OncePerDevice shared;
    std::atomic<int> ready{0}, sets{0}, good{0};
    std::vector<std::thread> threads;
    for (int t = 0; t < 8; ++t)
        threads.emplace_back([&, t] {
            for (++ready; ready < 8;) {}
            for (int k = 0; k < 1000; ++k) good += shared(t % 2, [&] { return ++sets, true; });
        });
    for (auto &t : threads) t.join();
    expect(good == 8000 && sets >= 2 && sets <= 8, "threads");
    printf("once per device: %s\n", failures ? "FAILED" : "ok");
    return failures != 0;
}
