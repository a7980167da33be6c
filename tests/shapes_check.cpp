// Which kernels products take (tq_shapes.h, the header that the library itself asks): lines "i8 m n k" or "orth pairs m n k below count" from the
// standard input, one answer a line: the shape's name, for 8-bit integers with the parts of k.
#include <cstdio>
#include <cstring>

#include "tq_shapes.h"

int main()
{
    static const char* const kI8[] = {"few", "256", "192", "192x256", "256x128", "128x256", "128x320", "128", "64"};
    static const char* const kOrth[] = {"256", "192", "128", "128 alone", "64"};
    char what[8];
    while (scanf("%7s", what) == 1) {
        unsigned long long a, m, n, k, below, count;
        if (!strcmp(what, "i8")) {
            if (scanf("%llu %llu %llu", &m, &n, &k) != 3) return 1;
            const unsigned long long groups = (k + 127) / 128;
            printf("%s %u\n", kI8[tq::i8::shape_of(m, n, groups)], tq::i8::splits_of(m, n, groups));
        } else {
            if (scanf("%llu %llu %llu %llu %llu %llu", &a, &m, &n, &k, &below, &count) != 6) return 1;
            printf("%s\n", kOrth[tq::orth::shape_of(a ? tq::kHalfPair : tq::kHalf, m, n, k, below != 0, count)]);
        }
    }
    return 0;
}
