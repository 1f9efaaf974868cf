// bf16 products on the tensor cores (tcgen05.mma kind::f16, one CTA): descriptors of operand tiles in shared memory and the
// instructions.  Every tile is an image of rows of 64 bf16 values (128 bytes) in the 128-byte swizzle, on a 1024-byte boundary: the 16-byte
// chunk c of row r lies at r * 128 + ((c ^ (r & 7)) << 4).  One image serves both ways round: its rows as rows of the operand (the
// 64 values are 64 steps of the contraction), or its rows as steps of the contraction (the 64 values are 64 rows of the operand).
#pragma once
#include "tma_util.cuh"
#include "tmem_util.cuh"

namespace hn {

__device__ __forceinline__ unsigned image_at(int row, int chunk) { return (unsigned)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

// The low half of a descriptor (address, and for columns the distance to the next 64 rows of the operand); the high half is the same for
// all: 1024 bytes from eight rows of an image to the next, 128-byte swizzle.
// Rows of the image = rows of the operand, from row r0 (a multiple of 8); a 16-step of the contraction further on: kRowStep more
constexpr unsigned kUmmaHigh = (1024u >> 4) | (1u << 14) | (2u << 29), kRowStep = 32 >> 4, kColStep = 2048 >> 4;
__device__ __forceinline__ unsigned umma_rows(unsigned image, int r0 = 0) { return (1u << 16) | (((image + (unsigned)(r0 * 128)) & 0x3ffffu) >> 4); }
// rows of the image = steps of the contraction; beyond 64 rows of the operand the next ones come from the image `next` bytes behind; a 16-step
// further on: kColStep more
__device__ __forceinline__ unsigned umma_cols(unsigned image, unsigned next = 1024) { return ((next >> 4) << 16) | ((image & 0x3ffffu) >> 4); }
// bf16 operands, fp32 accumulator of 128 rows and n columns; a_cols / b_cols: the operand is an image taken by its columns
__device__ __forceinline__ constexpr unsigned umma_kind(int n, bool a_cols, bool b_cols)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((unsigned)a_cols << 15) | ((unsigned)b_cols << 16) | ((unsigned)(n >> 3) << 17) | (8u << 24);
}
// The instructions are issued by one lane of a warp that comes here as a whole, in code that the compiler knows to be uniform: operands then
// stay in uniform registers and an instruction costs what the product takes (34 cycles for 64 columns, 13 for 16); from a branch of
// one thread each of them took 48 to 100.
__device__ __forceinline__ void umma_ss(unsigned d, unsigned a, unsigned b, unsigned kind, bool add)
{
    asm volatile("{\n .reg .pred p, one;\n .reg .b64 a, b;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n elect.sync _|one, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
                 " @one tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "r"(b), "r"(kind), "r"((unsigned)add), "r"(kUmmaHigh) : "memory");
}
// the A operand in tensor memory: row = lane, two values of the contraction to a column, 8 columns at `a`
__device__ __forceinline__ void umma_ts(unsigned d, unsigned a, unsigned b, unsigned kind, bool add)
{
    asm volatile("{\n .reg .pred p, one;\n .reg .b64 b;\n mov.b64 b, {%2, %5};\n elect.sync _|one, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
                 " @one tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "r"(b), "r"(kind), "r"((unsigned)add), "r"(kUmmaHigh) : "memory");
}
// everything this warp has issued so far arrives on bar when it is through (elect.sync names the same lane every time)
__device__ __forceinline__ void umma_commit(uint64_t *bar)
{
    asm volatile("{\n .reg .pred one;\n elect.sync _|one, 0xffffffff;\n @one tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
                 ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace hn
