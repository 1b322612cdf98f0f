// The shares of a workgroup's threads on the host (share.h).  Each argument is a case,
// "of:n:first:step", "entries:used:rows:first:step" or "blocks:n:block" (whose number is printed):
// walks one thread's places, compares each with 64-bit arithmetic, and prints how many there
// were.  Ends with 1 where one is wrong or the walk does not end.
#include <cstdio>
#include <cstdlib>

#include "share.h"

static bool of(const char* arg) {
    long long all, first, step;
    if (sscanf(arg, "of:%lld:%lld:%lld", &all, &first, &step) != 3) return false;
    int64_t place = first, n = 0;
    bool fine = true;
    each_of(all, (uint32_t)first, (uint32_t)step, [&](int64_t x) {
        if (x != place || x >= all) fine = false;
        if (!fine && n > all) {
            printf("%s does not end\n", arg);
            exit(1);
        }
        place += step;
        ++n;
    });
    if (!fine || place < all) {
        printf("%s is wrong after %lld\n", arg, (long long)n);
        return false;
    }
    printf("%s %lld\n", arg, (long long)n);
    return true;
}

static bool blocks(const char* arg) {
    int n, block;
    if (sscanf(arg, "blocks:%d:%d", &n, &block) != 2) return false;
    printf("%s %d\n", arg, blocks_of(n, block));
    return true;
}

static bool entries(const char* arg) {
    long long used, rows, first, step;
    if (sscanf(arg, "entries:%lld:%lld:%lld:%lld", &used, &rows, &first, &step) != 4) return false;
    const int64_t all = used * rows;
    int64_t place = first, n = 0;
    bool fine = true;
    each_entry((uint32_t)used, (uint32_t)rows, (uint32_t)first, (uint32_t)step, [&](uint32_t k, uint32_t e) {
        if (place >= all || k != place / used || e != place % used) fine = false;
        if (!fine && n > all) {
            printf("%s does not end\n", arg);
            exit(1);
        }
        place += step;
        ++n;
    });
    if (!fine || place < all) {
        printf("%s is wrong after %lld\n", arg, (long long)n);
        return false;
    }
    printf("%s %lld\n", arg, (long long)n);
    return true;
}

int main(int argc, char** argv) {
    for (int i = 1; i < argc; ++i)
        if (!(argv[i][0] == 'o' ? of(argv[i]) : argv[i][0] == 'b' ? blocks(argv[i]) : entries(argv[i]))) return 1;
    return 0;
}
