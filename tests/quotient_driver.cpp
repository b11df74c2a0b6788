// Every (divisor, multiple) that the paged attention's limits allow, at the two
// places where a quotient that is not exact shows: a multiple and the number before it.
#include <stdio.h>

#include "cas_internal.h"

int main() {
    for (int d = 1; d <= 4096; ++d) {
        const cas::Quotient q(d);
        for (int k = 0, x = 0; x < 1 << 24; ++k, x += d)
            if (q(x) != k || q(x + d - 1) != k) {
                printf("%d or %d by %d\n", x, x + d - 1, d);
                return 1;
            }
    }
    for (const int d : {1, 2, 3, 501, 2046, 4092, 65535, 65536})
        for (int64_t x = INT32_MAX; x > INT32_MAX - 70000; --x)
            if (cas::Quotient(d)((int)x) != (int)(x / d)) {
                printf("%lld by %d\n", (long long)x, d);
                return 1;
            }
    puts("exact");
    return 0;
}
