// bf16 products on the tensor cores (tcgen05.mma kind::f16, one CTA): descriptors of operand tiles in shared memory and the
// instructions.  Every tile is an image of rows of 64 bf16 values (128 bytes) in the 128-byte swizzle, on a 1024-byte boundary: the 16-byte
// chunk c of row r lies at r * 128 + ((c ^ (r & 7)) << 4).  One image serves both ways round: its rows as rows of the operand (the
// 64 values are 64 steps of the contraction), or its rows as steps of the contraction (the 64 values are 64 rows of the operand).
#pragma once
#include "tma_util.cuh"
#include "tmem_util.cuh"

namespace hn {

__device__ __forceinline__ unsigned image_at(int row, int chunk) { return (unsigned)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

constexpr unsigned long long kUmmaBase = (1ull << 46) | (2ull << 61) | ((unsigned long long)(1024 >> 4) << 32);
// rows of the image = rows of the operand, from row r0 (a multiple of 8); contraction steps 16 ks .. 16 ks + 15
__device__ __forceinline__ unsigned long long umma_rows(unsigned image, int ks, int r0 = 0)
{
    return kUmmaBase | (1ull << 16) | (((image + (unsigned)(r0 * 128 + ks * 32)) & 0x3ffffu) >> 4);
}
// rows of the image = steps of the contraction, 16 ks .. 16 ks + 15; beyond 64 rows of the operand the next ones come from the image
// `next` bytes behind
__device__ __forceinline__ unsigned long long umma_cols(unsigned image, int ks, unsigned next = 1024)
{
    return kUmmaBase | ((unsigned long long)(next >> 4) << 16) | (((image + (unsigned)(ks * 2048)) & 0x3ffffu) >> 4);
}
// bf16 operands, fp32 accumulator of 128 rows and n columns; a_cols / b_cols: the operand is an image taken by its columns
__device__ __forceinline__ constexpr unsigned umma_kind(int n, bool a_cols, bool b_cols)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((unsigned)a_cols << 15) | ((unsigned)b_cols << 16) | ((unsigned)(n >> 3) << 17) | (8u << 24);
}
// The instructions are issued by one lane of a warp that comes here as a whole, in code that the compiler knows to be uniform: operands then
// stay in uniform registers and an instruction costs what the product takes (34 cycles for 64 columns, 13 for 16); from a branch of
// one thread each of them took 48 to 100.
__device__ __forceinline__ void umma_ss(unsigned d, unsigned long long a, unsigned long long b, unsigned kind, bool add)
{
    asm volatile("{\n .reg .pred p, one;\n elect.sync _|one, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n @one tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
// the A operand in tensor memory: row = lane, two values of the contraction to a column, 8 columns at `a`
__device__ __forceinline__ void umma_ts(unsigned d, unsigned a, unsigned long long b, unsigned kind, bool add)
{
    asm volatile("{\n .reg .pred p, one;\n elect.sync _|one, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n @one tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
// everything this warp has issued so far arrives on bar when it is through (elect.sync names the same lane every time)
__device__ __forceinline__ void umma_commit(uint64_t *bar)
{
    asm volatile("{\n .reg .pred one;\n elect.sync _|one, 0xffffffff;\n @one tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
                 ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace hn
