// CPU check of the matrix-product kernels' address arithmetic (dense_geom.hpp):
// every slot of a stage is filled once, a fragment read returns the elements
// that the matrix instruction's lane needs, the lanes that are served at once use
// different banks, and every tile and split belongs to one workgroup.
#define __host__
#define __device__
#include "dense_geom.hpp"

#include <stdio.h>
#include <stdlib.h>

#include <set>
#include <vector>

using namespace cliff;

#define REQUIRE(c, ...)                     \
    do {                                    \
        if (!(c)) {                         \
            printf("FAIL %d: ", __LINE__);  \
            printf(__VA_ARGS__);            \
            printf("\n");                   \
            exit(1);                        \
        }                                   \
    } while (0)

struct El {
    int row = -1, k = -1;
};

static void stage(const Stage& s)
{
    std::vector<El> lds(s.bytes() / 2);
    for (int e = 0; e < s.slots(); ++e) {
        const int r = s.slot_row(e), k = s.slot_k(e);
        REQUIRE(r >= 0 && k >= 0 && r < s.R && k < s.KT, "slot %d: row %d value %d", e, r, k);
        for (int i = 0; i < 8; ++i) {
            El& x = lds[8 * e + i];
            x.row = r + (s.KM ? 0 : i);
            x.k = k + (s.KM ? i : 0);
            REQUIRE(s.at(x.row, x.k) == 16 * e + 2 * i, "element (%d, %d)", x.row, x.k);
        }
    }
    std::set<std::pair<int, int>> seen;
    for (const El& x : lds) seen.insert({x.row, x.k});
    REQUIRE((int)seen.size() == s.R * s.KT, "stage not covered");
    for (int row0 = 0; row0 < s.R; row0 += 32)
        for (int k0 = 0; k0 < s.KT; k0 += 16)
            for (int lane = 0; lane < 64; ++lane)
                for (int i = 0; i < 8; ++i) {
                    El x;
                    if (s.KM) {
                        const int b = frag_byte(s, row0, k0, lane, 0);
                        REQUIRE(b % 16 == 0 && b + 16 <= s.bytes(), "fragment byte %d", b);
                        x = lds[b / 2 + i];
                    } else {
                        // the transposing read: lane t of 16 gets element t % 4 of what
                        // lane 4 i + t / 4 addresses, as its i-th value
                        const int t = lane & 15, from = (lane & 48) + 4 * (i & 3) + t / 4;
                        const int b = frag_byte(s, row0, k0, from, i / 4);
                        REQUIRE(b % 8 == 0 && b + 8 <= s.bytes(), "fragment byte %d", b);
                        x = lds[b / 2 + t % 4];
                    }
                    REQUIRE(x.row == row0 + (lane & 31) && x.k == k0 + 8 * (lane >> 5) + i,
                            "lane %d value %d: (%d, %d) at %d, %d", lane, i, x.row, x.k, row0, k0);
                }
    for (int row0 = 0; row0 < s.R; row0 += 16)
        for (int k0 = 0; k0 + 32 <= s.KT; k0 += 32)
            for (int lane = 0; lane < 64; ++lane)
                for (int i = 0; i < 8; ++i) {
                    El x;
                    if (s.KM) {
                        x = lds[frag16_byte(s, row0, k0, lane, 0) / 2 + i];
                    } else {
                        const int t = lane & 15, from = (lane & 48) + 4 * (i & 3) + t / 4;
                        const int b = frag16_byte(s, row0, k0, from, i / 4);
                        REQUIRE(b % 8 == 0 && b + 8 <= s.bytes(), "fragment byte %d", b);
                        x = lds[b / 2 + t % 4];
                    }
                    REQUIRE(x.row == row0 + (lane & 15) && x.k == k0 + 8 * (lane >> 4) + i,
                            "lane %d value %d: (%d, %d) at %d, %d", lane, i, x.row, x.k, row0, k0);
                }
    // banks: 32 lanes of a transposing read, 16 of a 16-byte read, at once
    const int at_once = s.KM ? 16 : 32;
    if (s.KM || s.line() >= 16)
        for (int lane = 0; lane < 64; lane += at_once) {
            std::set<int> banks;
            for (int l = lane; l < lane + at_once; ++l)
                for (int w = 0; w < 64 / at_once; ++w) banks.insert((frag_byte(s, 0, 0, l, 0) / 4 + w) % 64);
            REQUIRE(banks.size() == 64, "lanes from %d touch %d banks", lane, (int)banks.size());
        }
}

static void tiles(uint32_t tm, uint32_t tn, uint32_t splits)
{
    std::set<std::vector<int>> seen;
    for (uint32_t b = 0; b < tm * tn * splits; ++b) {
        const TileId t = tile_of(b, tm, tn, splits);
        REQUIRE(t.m >= 0 && t.n >= 0 && t.split >= 0 && (uint32_t)t.m < tm && (uint32_t)t.n < tn &&
                    (uint32_t)t.split < splits, "workgroup %u of %u x %u x %u", b, tm, tn, splits);
        seen.insert({t.m, t.n, t.split});
    }
    REQUIRE(seen.size() == (size_t)tm * tn * splits, "tiles %u x %u x %u", tm, tn, splits);
}

int main()
{
    for (int R : {32, 64, 128, 256})
        for (int KT : {16, 32, 64})
            for (bool km : {false, true}) stage(Stage{R, KT, km});
    for (uint32_t tm : {1, 2, 7, 8, 9, 17, 64})
        for (uint32_t tn : {1, 3, 8, 31})
            for (uint32_t s : {1, 2, 5}) tiles(tm, tn, s);
    puts("ok");
    return 0;
}
