// The scratch that the log probabilities report against what their plans take, over rows
// of every size around the borders of the rules.
#include <stdio.h>

#include <set>

#include "logprob_plan.h"

int main() {
    std::set<int> rows, lengths;
    for (int p = 0; p <= 21; ++p)
        for (const int d : {-1, 0, 1}) rows.insert((1 << p) + d);
    for (int n = 1; n <= 700; ++n) rows.insert(n);
    for (const int n : {1000, 1100, 1501, 1600, 1999, 2500, 3000, 5000, 100000, 1500000}) rows.insert(n);
    for (int p = 0; p <= 20; ++p)
        for (const int d : {-1, 0, 1}) lengths.insert((1 << p) + d);
    for (int v = 2048; v <= 1 << 20; v += 2048)
        for (const int d : {-1, 0, 1}) lengths.insert(v + d);
    for (const int n : rows)
        for (const int V : lengths) {
            if (n < 1 || n > 1 << 21 || V < 1 || V > 1 << 20) continue;
            const cas::LpPlan p = cas::lp_plan(n, V);
            const int chunk = p.threads * p.each;
            if (p.span < 1 || p.span > cas::LP_SPAN || p.parts < 1 || p.parts > cas::LP_PARTS ||
                (int64_t)p.parts * p.span * chunk < V || (int64_t)(p.parts - 1) * p.span * chunk >= V) {
                printf("%d rows of %d: %d parts of %d chunks of %d\n", n, V, p.parts, p.span, chunk);
                return 1;
            }
            for (const int K : {0, 1, 20, 32})
                if (p.parts > 1 && cas::lp_work_bytes(n, V, K) < (size_t)n * p.parts * cas::lp_words(K) * 4) {
                    printf("%d rows of %d, K = %d: scratch of %zu bytes\n", n, V, K, cas::lp_work_bytes(n, V, K));
                    return 1;
                }
        }
    puts("enough");
    return 0;
}
