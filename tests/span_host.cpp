// span_bytes (csrc/span.h) on the host: "rows ld cols vec" per line of input, the bytes per line of output.
#include <cstdio>

#include "../paper_2608_13426_amd/csrc/span.h"

int main() {
    long long rows, ld, cols;
    int vec;
    while (scanf("%lld %lld %lld %d", &rows, &ld, &cols, &vec) == 4)
        printf("%lld\n", static_cast<long long>(rmm::span_bytes(rows, ld, cols, vec != 0)));
}
