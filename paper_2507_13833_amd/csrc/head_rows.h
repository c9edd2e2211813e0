// Which rows of the head's operands take part, and operands laid out for the product: shared by the two directions.
#pragma once
#include "head_device.h"

namespace dc {

constexpr int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }
constexpr int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of * of; }

struct HeadShape {
    int64_t rows_pad;               // rows, to whole tiles of either kind
    int32_t k_pad;                  // columns, to whole steps
    bool    copy_hidden, copy_weight;   // not as the product reads it: laid out in the workspace first
};
// How a product of m by n rows with that many steps is cut: tiles of Q = 4 (small) or 8, the steps shared by `splits` workgroups a tile.
struct ProductCut { bool small; int32_t splits; };
ProductCut cut_product(int64_t m, int64_t n, int64_t steps, int32_t most_splits);
constexpr int64_t most_split_rows(int64_t rows, int64_t n, int32_t most_splits) {       // splits times rows (of whole tiles) of any cut of up to so many rows
    const int64_t tiles = whole(n, P_SIDE<4>) / P_SIDE<4>, all = rows * most_splits, some = (1 << 18) / tiles;
    return rows > (all < some ? all : some) ? rows : all < some ? all : some;
}

HeadShape head_shape(const dc_matrix& hidden, const dc_matrix& weight, bool listed);

// Rows `list` (or all) of src as planes of [rows][k_pad] 16-bit numbers, columns behind the last one 0; *count (or n) rows, the planes
// `plane` bytes apart.  16-bit numbers as they are, in one plane; others as two of f16 (or, apart == BF16S, three of bf16 that are the
// number itself), 2^(15 - exponent) times as much for the exponent of the row (row_exp) or of them all (all_exp).
enum Apart { F16S, BF16S };
hipError_t launch_lay_rows(const dc_matrix& src, int64_t first, int64_t n, const int32_t* list, const int32_t* count, int32_t k_pad,
                           char* dst, int64_t plane, Apart apart, const int32_t* row_exp, const int32_t* all_exp, hipStream_t st);
// out[i]: of the largest finite magnitude of row list[i] (or i) of 32 bits, the power of two above it.
hipError_t launch_row_exponents(const dc_matrix& src, int64_t n, const int32_t* list, const int32_t* count, int32_t* out, hipStream_t st);
// *top, raised to the same of rows first .. first + n - 1, f32 or bf16 (f16 wants none).
hipError_t launch_top_exponent(const dc_matrix& src, int64_t first, int64_t n, int32_t* top, hipStream_t st);
// What raised exponents begin with.  exact: all but the first are 15 instead, which leaves numbers as they are (f16 wants no other).
struct FirstExponents { int32_t* top; int32_t n; bool exact; };
hipError_t launch_first_exponents(const FirstExponents& x, hipStream_t st);

// The other way round: planes of [cols][rows_pad] f16, one for 16-bit numbers and two for others, rows behind the last one 0 to the next
// multiple of 64.  Values become 2^(15 - *top - term's exponent) times as much (a row's own exponent where there are terms).
struct RowTerm;
hipError_t launch_lay_columns(const dc_matrix& src, int64_t first, int64_t n, const int32_t* list, const int32_t* count, int64_t rows_pad,
                              const int32_t* top, const RowTerm* term, char* dst, int64_t plane, hipStream_t st);

// What the gradient of a live row's logits is made of: g_v = 2^exponent / T * (a (v == token) - p_v (a + b (log p_v + H))) with
// log2 p_v = (x_v - m) k - l2:  g_v = ga (v == token) + p_v (c0 + c1 log2 p_v).
// x_exp: of the row of hidden states, for numbers of 32 bits.
struct alignas(16) RowTerm { float m, l2, c0, c1, ga; int32_t token, exponent, x_exp; };

// The live rows of a batch, in order: list, their number, and where each row went (-1: nowhere).
struct LiveRows { int32_t* list; int32_t* pos; int32_t* count; };
// A row is live where its mask byte is not 0 (mask NULL: everywhere) and, where a is given, a or b is not 0.  Writes x on the way.
hipError_t launch_live_rows(const uint8_t* mask, const float* a, const float* b, int64_t n, const LiveRows& l, const FirstExponents& x,
                            hipStream_t st);

// Which of the planes of two operands are multiplied: of two f16 each, all pairs but the two small ones.
Parts parts_of(int32_t type, int64_t a_plane, int64_t b_plane);

}  // namespace dc
