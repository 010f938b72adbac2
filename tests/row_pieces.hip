// Runs the pieces that the grouped dense layers read rows in on the host: every piece of every row, of arrays of all small sizes that end at an
// unreadable page.  Each load lies in the array and, where whole words are read, at a word's address; what comes of it are the row's elements, then
// zeros.  The last line printed names the case.
#include <hip/hip_runtime.h>
#undef __device__
#define __device__ __attribute__((host)) __attribute__((device))
#define __uint_as_float(x) __builtin_bit_cast(float, uint32_t(x))
#define __float_as_uint(x) __builtin_bit_cast(uint32_t, float(x))
#include "row_piece.hpp"

#include <sys/mman.h>
#include <unistd.h>

#include <cstdlib>
#include <cstring>

using namespace tma;

#define CHECK(cond)                                          \
    do {                                                     \
        if (!(cond)) {                                       \
            printf("%s: not so: %s\n", name, #cond);         \
            exit(1);                                         \
        }                                                    \
    } while (0)

// `page`: the end of a page that may not be passed
template <typename T, bool kWords>
static void pieces(char *page_end, int64_t n, int64_t ld, int F)
{
    typedef RowPiece<T, kWords> P;
    constexpr int E = P::E;
    char name[120];
    snprintf(name, sizeof(name), "%d bytes, words %d, n=%ld ld=%ld F=%d", int(sizeof(T)), int(kWords), long(n), long(ld), F);
    const int64_t extent = (n - 1) * ld + F;
    T *x = reinterpret_cast<T *>(page_end) - extent;
    if (kWords) {
        x = reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(x) / 4 * 4);
        if (P::last_place(n, ld, F) < 0) return;          // (such arrays are read element by element)
    }
    T *const h = static_cast<T *>(malloc(size_t(extent) * sizeof(T)));      // a mask: open throughout, or closed at the last element
    for (int64_t i = 0; i < extent; ++i) {
        x[i] = T(i % 251 + 1);
        h[i] = sizeof(T) == 4 ? T(1) : T(0x3F80);
    }
    const int64_t last = P::last_place(n, ld, F);
    if (kWords) CHECK(last + E <= extent && last * int64_t(sizeof(T)) % 4 == 0);
    CHECK(P::left_out(x, h, n, ld, F) == P::left_out(x, nullptr, n, ld, F));
    const uint32_t rest = P::left_out(x, h, n, ld, F);
    h[extent - 1] = T(0);
    CHECK(P::left_out(x, h, n, ld, F) == 0u);
    free(h);
    for (int64_t v = 0; v < n; ++v)
        for (int k = 0; k < F; k += E) {
            const int64_t at = v * ld + k;
            const int valid = F - k;
            if (kWords) {
                const int64_t from = at < last ? at : last;
                CHECK(from >= 0 && from + E <= extent && (reinterpret_cast<uintptr_t>(x + from) & 3) == 0);
            }
            uint4 p = P::load(x, at, valid, last);
            if (kWords && F % E != 0) {
                if (at > last) p = P::moved(p, int(at - last), rest);
                p = P::cut(p, valid);
            }
            T got[E];
            memcpy(got, &p, 16);
            for (int j = 0; j < E; ++j) CHECK(got[j] == (j < valid ? x[at + j] : T(0)));
        }
}

int main()
{
    const size_t page = size_t(sysconf(_SC_PAGESIZE)), room = 16 * page;
    char *base = static_cast<char *>(mmap(nullptr, room + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    if (base == MAP_FAILED) return 3;
    mprotect(base + room, page, PROT_NONE);
    int cases = 0;
    for (int64_t n = 1; n <= 11; ++n)
        for (int F = 1; F <= 41; ++F)
            for (int64_t ld = F; ld <= F + 9; ++ld, ++cases) {
                pieces<uint16_t, false>(base + room, n, ld, F);
                if (ld % 2 == 0) pieces<uint16_t, true>(base + room, n, ld, F);
                pieces<float, false>(base + room, n, ld, F);
                pieces<float, true>(base + room, n, ld, F);
            }
    printf("%d cases\n", cases);
    return 0;
}
