// Several threads that make failing calls of the dense layers on one context, each of which has to get its own messages.  All of it
// is refused on the host before a device is needed, so the context is put together here.
#include <atomic>
#include <cstdio>
#include <cstring>
#include <thread>
#include <vector>

#include "common.cuh"

int main() {
    tfjsb_ctx* ctx = new tfjsb_ctx;  // not one of tfjsb_init, which wants a device
    if (strcmp(tfjsb_last_error(ctx), "")) return printf("a new context has a message\n"), 1;
    const int64_t dims[1] = {8}, wrong[1] = {3};
    std::atomic<int> waiting{4}, bad{0};
    auto call = [&](int which) -> tfjsb_status {
        switch (which) {
            case 0: return tfjsb_dropout(ctx, (tfjsb_dtype)7, nullptr, nullptr, nullptr, 1, dims, nullptr, 0.5, 0, 0, nullptr);
            case 1: return tfjsb_dropout(ctx, TFJSB_DTYPE_F32, nullptr, nullptr, nullptr, 1, dims, nullptr, 1.5, 0, 0, nullptr);
            case 2: return tfjsb_dropout(ctx, TFJSB_DTYPE_F32, nullptr, nullptr, nullptr, 1, dims, wrong, 0.5, 0, 0, nullptr);
            default: return tfjsb_quantize_int8(ctx, TFJSB_DTYPE_F32, nullptr, 1, 131073, nullptr, nullptr, nullptr);
        }
    };
    const char* text[4] = {"unknown dtype", "rate must be in [0, 1)", "each dimension of the mask must be that of x or 1", "more than 131072 columns"};
    std::vector<std::thread> threads;
    for (int t = 0; t < 4; ++t)
        threads.emplace_back([&, t] {
            --waiting;
            while (waiting > 0) {}
            for (int i = 0; i < 20000; ++i) {
                if (call(t) == TFJSB_OK) ++bad;
                if (strcmp(tfjsb_last_error(ctx), text[t])) ++bad;
            }
        });
    for (auto& t : threads) t.join();
    if (bad) return printf("%d calls got another thread's message\n", bad.load()), 1;
    // one thread at a time: a message may be asked for by another thread than the one whose call failed
    call(1);
    bool same = false, later = false;
    std::thread([&] { same = !strcmp(tfjsb_last_error(ctx), text[1]); call(3); }).join();
    if (!same || strcmp(tfjsb_last_error(ctx), text[1])) return printf("the message went away with the thread\n"), 1;
    later = !strcmp(tfjsb_last_error(ctx), text[3]);  // asked for its own, so the last one of all
    if (!later) return printf("the last failing call's message is not found\n"), 1;
    delete ctx;
    printf("ok\n");
    return 0;
}
