// Where the attention's tiles are loaded from (grawa_attend.h), on the host: the offsets of all pieces of all loads against the descriptor that
// bounds them, for every width and row length.
#include <cstdio>

#include "grawa_attend.h"

static int failures;

template <bool BF16, int DP, int ROWS, int NW> static void check()
{
    typedef TilePieces<BF16, DP, ROWS, NW> P;
    const uint32_t tokens[] = {(uint32_t)DP * P::ES, 4096, 1u << 20, (1u << 23) - 16, 1u << 23, (1u << 23) + 16, 8421376, 9000000 / 16 * 16, 9623040, 12000000 / 16 * 16, (1u << 24) - 16};
    for (int D = 8; D <= DP; D += 8)
        for (uint32_t token : tokens) {
            const uint64_t end = (uint64_t)(ROWS - 1) * token + D * P::ES; // of the largest descriptor
            int bad = end > 0xffffffffu;
            for (int id = 0; id < NW * 64; ++id)
                for (int i = 0; i < P::LOADS; ++i) {
                    const uint32_t at = P::later(P::first_of(id, i % P::TURNS, token, D), (uint32_t)(i / P::TURNS) * (P::RPL * P::TURNS * token));
                    const int row = id / P::PPR + i * P::RPL, c = (id % P::PPR) ^ P::key(row);
                    if (c * 16 < D * P::ES)
                        bad |= at != (uint64_t)row * token + c * 16 || at + 16ull > end;
                    else
                        bad |= at < end || at > 0xffffffffu - 15;
                }
            if (bad && ++failures <= 20) std::printf("%s, %d elements of %d, %d rows of %u bytes, %d waves\n", BF16 ? "bfloat16" : "float32", D, DP, ROWS, token, NW);
        }
}

int main()
{
    // keys, values and queries of the forward pass, of dq and of dk and dv, and the values that these keep
    check<true, 64, 64, 4>(), check<true, 128, 64, 4>(), check<false, 64, 64, 4>(), check<false, 128, 64, 4>();
    check<true, 64, 128, 4>(), check<true, 128, 128, 4>(), check<false, 64, 128, 4>(), check<false, 128, 64, 2>();
    check<true, 128, 64, 8>(), check<true, 128, 256, 8>(), check<false, 64, 128, 4>(), check<false, 128, 128, 4>();
    if (failures) {
        std::printf("%d failures\n", failures);
        return 1;
    }
    std::printf("ok\n");
    return 0;
}
