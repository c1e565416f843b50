// Address arithmetic of the matrix-product kernels (dense.hip), shared with the
// CPU check of the tests: which tile a workgroup computes, how a stage of an
// operand lies in LDS, and which of its elements a fragment read returns.
#pragma once

#include <stdint.h>

namespace cliff {

// A stage of one operand: R rows (of the output's side) by KT contraction
// values of 16 bits, in LDS slots of 16 bytes (8 elements).  KM: memory is
// contiguous along the contraction, and a slot holds 8 of its values of one
// row; otherwise memory is contiguous along the rows, and a slot holds 8 rows
// of one contraction value.  Slots of a line (a row, or a contraction value)
// are permuted by an XOR so that the lanes that a fragment read serves at once
// (16 of 16 bytes, 32 of 8), which walk down the lines, touch all 64 banks once
// (two-way conflicts cost 30 % of the read rate); a direct load to LDS writes the
// slots in order and permutes the addresses that it reads instead.
struct Stage {
    int R, KT;
    bool KM;
    __host__ __device__ constexpr int line() const { return KM ? KT / 8 : R / 8; }  // slots per line
    __host__ __device__ constexpr int slots() const { return R * KT / 8; }
    __host__ __device__ constexpr int bytes() const { return R * KT * 2; }
    __host__ __device__ constexpr int swizzle(int l) const
    {
        return KM ? (l / (16 / line())) & (line() - 1)
                  : ((l & 3) << 2 | (l >> 2 & 2)) & (line() - 1);
    }
    // first row and contraction value of slot e
    __host__ __device__ constexpr int slot_row(int e) const
    {
        const int l = e / line(), s = (e % line()) ^ swizzle(l);
        return KM ? l : 8 * s;
    }
    __host__ __device__ constexpr int slot_k(int e) const
    {
        const int l = e / line(), s = (e % line()) ^ swizzle(l);
        return KM ? 8 * s : l;
    }
    // byte of element (row, k)
    __host__ __device__ constexpr int at(int row, int k) const
    {
        const int l = KM ? row : k, c = KM ? k : row;
        return (l * line() + ((c / 8) ^ swizzle(l))) * 16 + (c % 8) * 2;
    }
};

// A fragment of 32 rows by 16 contraction values (v_mfma_*_32x32x16): lane l
// holds row l & 31, values 8 (l >> 5) to + 7.  KM: one 16-byte read.
// Otherwise two transposing reads j of 8 bytes: within 16 lanes, lane t gets
// element t & 3 .. of the lanes 4 i + t / 4, that is row t of the four values
// that the lanes' lines are.
__host__ __device__ constexpr int frag_row(int lane) { return lane & 31; }
__host__ __device__ constexpr int frag_k(int lane) { return 8 * (lane >> 5); }
__host__ __device__ constexpr int frag_byte(const Stage& s, int row0, int k0, int lane, int j)
{
    if (s.KM) return s.at(row0 + frag_row(lane), k0 + frag_k(lane));
    const int t = lane & 15;
    return s.at(row0 + (lane & 16) + 4 * (t & 3), k0 + frag_k(lane) + 4 * j + (t >> 2));
}

// The same for fragments of 16 rows by 32 values (v_mfma_*_16x16x32): lane l
// holds row l & 15, values 8 (l >> 4) to + 7.
__host__ __device__ constexpr int frag16_byte(const Stage& s, int row0, int k0, int lane, int j)
{
    if (s.KM) return s.at(row0 + (lane & 15), k0 + 8 * (lane >> 4));
    const int t = lane & 15;
    return s.at(row0 + 4 * (t & 3), k0 + 8 * (lane >> 4) + 4 * j + (t >> 2));
}

// Workgroups go round the 8 XCDs; workgroup bid's place in an order in which
// each XCD has a run of neighbours, which share lines of its L2.
__host__ __device__ inline uint32_t xcd_run(uint32_t bid, uint32_t total)
{
    const uint32_t q = total / 8, r = total % 8, xcd = bid % 8;
    return xcd * q + (xcd < r ? xcd : r) + bid / 8;
}

// The tile and split of workgroup bid.  Each XCD gets a run of consecutive
// tiles; those go down 8 rows of tiles before the next column, so that what
// runs together shares operands in its L2.
struct TileId {
    int m, n, split;
};
__host__ __device__ inline TileId tile_of(uint32_t bid, uint32_t tm, uint32_t tn, uint32_t splits)
{
    const uint32_t t = xcd_run(bid, tm * tn * splits);
    const uint32_t split = t / (tm * tn), u = t % (tm * tn);
    const uint32_t g = u / (8 * tn), first = 8 * g, v = u % (8 * tn);
    const uint32_t rows = tm - first < 8 ? tm - first : 8;
    return TileId{(int)(first + v % rows), (int)(v / rows), (int)split};
}

}  // namespace cliff
