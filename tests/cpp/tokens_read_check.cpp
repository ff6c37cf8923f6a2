// tokens_read (csrc/kvbfp_internal.h) against 64-bit arithmetic, up to the largest lengths, windows and prefixes (built with the sanitizer for
// undefined behaviour: no sum may pass 32 bits).
#include <algorithm>
#include <cstdio>
#include <initializer_list>

#include "kvbfp_internal.h"

int main() {
    const int32_t top = 1 << 30;
    const std::initializer_list<int32_t> sizes = {0, 1, 2, 63, 64, 65, 1000, top / 2 - 1, top / 2, top / 2 + 64, top - 128, top - 64, top - 1, top};
    for (int32_t len : sizes)
        for (int32_t prefix : sizes)
            for (int32_t window : sizes)
                for (int32_t more : {0, 1, 63})
                    for (int32_t n_tok : {1, 5, 64}) {
                        if (prefix > len) continue;
                        const int64_t want = std::min<int64_t>(len, (int64_t)window + more + n_tok + prefix);
                        const int32_t got = kvbfp::tokens_read(len, window + more, n_tok, prefix);
                        if (got != want) {
                            std::printf("len %d window %d n_tok %d prefix %d: %d, not %lld\n", len, window + more, n_tok, prefix, got, (long long)want);
                            return 1;
                        }
                    }
    std::printf("tokens_read ok\n");
    return 0;
}
