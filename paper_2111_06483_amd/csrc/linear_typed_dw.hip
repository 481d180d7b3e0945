// Weight gradients by type: dW[t] (+)= X_t^T dZ_t over the rows of every type, X as fp32 or bf16 rows or in 8 bits (packed.h).
//
// The contraction runs along the rows, which both operands have as their slow dimension.  A workgroup of four wavefronts holds a tile of 128 x 256
// (256 x 128, 128 x 128, 128 x 64, 64 x 128) sums in registers, two or three of them a compute unit; its rows come in chunks of 16 (bf16: 32):
//   - A thread reads eight rows of two columns (four of packed rows) into registers, two chunks ahead (fp32 x fp32 in the wide tiles: one), turns them
//     into bf16 pieces along the rows (fp32: three, exact; bf16 rows and packed ones, whose values are bf16 values: one) and puts them to LDS as whole
//     fragments: 16 bytes are eight rows of a column, conflict-free to read.  (Not to write from 8 bits: of a thread's four columns two are
//     neighbours there, so lanes meet a bank twice; 25% of the LDS cycles at 867187 x 256 x 256.)  Two buffers, one barrier a chunk.
//   - fp32 x fp32 takes six products of pieces (linear_pieces.h), packed x fp32 three, packed or bf16 x bf16 one.
//   - Sums: fp32 products are summed from zero in the matrix unit over 16 rows, then added by vector instructions, every other chunk with the other
//     sign of X: the matrix unit cuts where it adds, and over a million rows that would lean to one side.  Bf16 products, as many times fewer, are
//     added to the sums there, X's sign turning every four chunks and with the workgroup.
// Rows are dealt evenly to the workgroups, whatever the types' sizes: a workgroup that meets the end of a type writes its sums and starts
// anew, so no workgroup has more rows than another.  Workgroup w writes its sums of type t to place w + t (every step along the rows goes to the
// next workgroup or the next type, so no two have the same place), and a second launch adds a type's places up in order: the result is the
// same in every run.  fp32 sums that are not finite (kUp: nor that large) are taken again there, from the operands.
// What bounds it: 237500 x 256 x 256, fp32, 210 us = 148 TFLOP/s (the six products' 890 TFLOP/s of bf16, of 1170 that a large library product reaches); bf16 from
// 8 bits, 867187 rows, 212 us: its 680 MB once would be 141, its products 97; every chunk's way from memory through registers to LDS is instructions between the
// products (the matrix cores are busy a quarter of the cycles).
#include "linear_typed_dw.h"

namespace sar {

size_t typed_dw_bytes(int64_t n, int K, int F, int T)
{
    auto most = [&](int chunk) { return std::max(most_groups(n, K, F, chunk, false), most_groups(n, K, F, chunk, true)); };
    return (size_t)(std::max(most(kChunk32), most(kChunk16)) + T) * K * F * sizeof(float);
}

int typed_dw(int dtype, const TypedDw& g, hipStream_t st)
{
    if (few_rows_dw(g.types.n, g.types.T, g.K, g.F)) return few_dw(dtype, g, st);
    const Shape s = shape_of(g.types.n, g.K, g.F, dtype == SAR_F32 ? kChunk32 : kChunk16, g.Xq != nullptr);
    const DwArgs a{g.X, g.Xq, g.Xe, g.dZ, g.partial, g.types, g.K, g.F, s.share};
    if (dtype == SAR_F32)
        return g.Xq ? run_all<PackedRows, F32Rows, kChunk32 / 16, 2>(a, s, g.accumulate, g.dW, st)
                    : run_all<F32Rows, F32Rows, kChunk32 / 16, 1>(a, s, g.accumulate, g.dW, st);
    return g.Xq ? run_all<PackedRows, Bf16Rows, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st)
                : run_all<Bf16Rows, Bf16Rows, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st);
}

}  // namespace sar
