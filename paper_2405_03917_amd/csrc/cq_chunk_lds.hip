// Causal attention of a few query rows per KV head over a packed CQ cache (speculative
// verification, short prefill chunks), for gfx950: the codebooks of the KV head in LDS, every
// wavefront on tiles of its own.  The formats whose two codebooks fit there: CQ-8c8b and CQ-4c8b
// (2 x 64 KB of the CU's 160 KB).
//
// The kernel for many rows (cq_chunk.hip) expands each 64-token tile once per workgroup from
// codebooks in L2, which costs it 2 x 64 x Gh divergent lane-gathers of the texture path per
// tile (about 4100 clocks at CQ-4c8b) whatever the number of rows.  Here the expansion IS the
// operand load of the matrix product:
//   S^T = K Q^T      v_mfma_f32_16x16x32_f16, A = keys of 16 tokens: a lane's 8 channels are the
//                    centroid(s) of its token's code(s), read by ds_read_b128 / b64 at code
//                    times entry size; B = 16 query rows (registers)
//   softmax          each lane owns one query column; 2^12-scaled probabilities as two fp16
//                    numbers (22 bits) as in cq_chunk.hip
//   O^T += V^T P^T   A = values transposed: ds_read_b64_tr_b16 takes an address per lane and
//                    hands lane j of 16 the j-th of 16 channels of 4 tokens, so gather and
//                    transpose are one instruction; B = the probabilities just computed
// A tile costs a wavefront 48 (CQ-8c8b) or 64 (4c8b) LDS gathers, 48 matrix products (32 up to 8
// rows) and about 260 / 330 vector instructions, nothing is shared between wavefronts inside the
// loop and there is no barrier.  Bound: the LDS.  A gather of 64 random 16-byte entries takes
// 12.3 clocks (16 lanes at a time on 16 bank groups: the fullest holds 3.1), a transposing one
// 6.2, i.e. 394 clocks per tile and CU at CQ-8c8b; the kernel takes 488 (LDS active 79 %; up to eight rows).
// Measured: CQ-4c8b, batch 16, 32 heads, 5 tokens over 4096: 136 us token by token, 264 us in the
// many-row kernel, 43 to 49 us here; CQ-8c8b, batch 4 x 131072, 5 tokens: 441 -> 271 us in two pieces (given as
// tokens_per_split: the default's workspace holds one, and such a call goes token by token).  The first form
// waited for every gather by itself (5800 clocks per tile and wavefront, 61 us); values gathered
// ahead of the softmax in one batch of 64 registers spilled at CQ-4c8b and gained nothing.
//
// A workgroup of 8 wavefronts (one per CU) serves RB = 1, 2 or 4 blocks of 16 rows; the 8 / RB wavefronts of
// a block take every (8 / RB)-th tile and are merged through LDS at the end.  Workgroups walk
// several (sequence, split) items of one KV head, so the codebooks are staged once per workgroup.
// Parts, each taken out by itself (32 heads): all keys of a tile gathered at once and not two of four batches ahead, CQ-8c8b, 40 tokens, 64 x 1000
// 143.4 -> 140.3 us, 16 tokens 62.8 -> 61.5; CQ-4c8b, 5 tokens of 16 x 4096, 43.3 -> 42.9.  Priorities: CQ-8c8b, 40 tokens
// of 64 x 1000, 145.4 -> 140.3, CQ-4c8b, 5 tokens of 16 x 4096, 44.2 -> 42.9, of 64 x 300 44.8 -> 45.8; up to eight rows of CQ-8c8b do without
// (5 tokens of 64 x 1000 52.6, with them 55.7; 8 of 16 x 16384 119.0 and 123.8).  Codebooks ahead of the first codes and eight rows merged in one
// pass: the rest of CQ-8c8b, 5 tokens of 64 x 1000, 57.9 -> 52.6, 16 x 4096 39.2 -> 36.9.
#include "cq_key_gather.hpp"
#include "cq_lds_gather.hpp"

namespace cq {
namespace {

constexpr int kWaves = 8;
constexpr int kRows = 16;                               // query rows of a wavefront
constexpr unsigned kMergeBase = 2 * kBookBytes;         // (m, l) of every wavefront and row, or 64 channels of every wavefront's
constexpr unsigned kORow = 64 * 4;                      // output rows
constexpr unsigned kLdsBytes = kMergeBase + kWaves * kRows * kORow;
static_assert(kLdsBytes == 160 * 1024, "all of a CU's LDS");
__device__ __forceinline__ half8_t lds_half8(unsigned a) { return *(__attribute__((address_space(3))) half8_t*)(a); }
__device__ __forceinline__ half4_t lds_half4(unsigned a) { return *(__attribute__((address_space(3))) half4_t*)(a); }
// The exponent that probabilities are relative to where the largest score (base 2) is m: 12 below m, so that
// they fill fp16's range; m itself where 12 is lost in its rounding.
__device__ __forceinline__ float softmax_reference(float m) { return m - (fabsf(m) < 0x1p22f ? 12.f : 0.f); }
// maximum / sum over the four lanes l % 16 + 16 b
__device__ __forceinline__ float across_max(float v)
{
    return rows_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float across_sum(float v)
{
    return rows_reduce(v, [](float a, float b) { return a + b; });
}

// HALF: at most 8 rows in all.  Columns q and q + 8 of the score product hold the same query, and in the
// value product the high parts of its probabilities in one and the low parts in the other: half the
// matrix products there, one addition at the end.
#define CQ_VIEW_KERNEL 0
#include "cq_chunk_lds_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_chunk_lds_kernel.hpp"
#undef CQ_VIEW_KERNEL

// At most 4 rows: lane = token, as in the decode kernel for four query heads (cq_decode_quad.hip, which says how): a token's
// scores of the four rows in the registers of its lane, by v_mfma_f32_4x4x4_16B_f16 with the queries broadcast; every
// wavefront a tile of the item by itself; probabilities relative to a running reference that moves when a score
// exceeds it by 3, as three fp16 numbers each (33 bits; twelve columns) to a [token][column] array in LDS and back transposed.
// The kernel above computes sixteen columns of softmax whatever the rows, and is bound by the vector ALU as much as by the
// LDS then: CQ-4c8b 408 instructions per tile (here 290) next to 454 clocks of LDS, 656 clocks taken, 520 here.  Measured, above
// -> here: CQ-4c8b, 32 heads, 3 tokens of 16 x 4096 50.5 -> 43.1 us, of 64 x 1000 71.7 -> 58.5; CQ-8c8b, 4 tokens of 16 x 4096 37.8 ->
// 33.8, of 64 x 1000 55.3 -> 49.9; of 4 x 30000 130 / 130 and 77 / 78.  (The same for eight rows, two fp16 numbers each and
// twice the matrix instructions, 0.94 to 1.01 times as fast as above: there the columns are no waste.)
constexpr unsigned kFewWaveBytes = 2048;                // of a wavefront: 64 tokens x 16 columns; at the end of an item four output rows
constexpr unsigned kFewPairs = kMergeBase + kWaves * kFewWaveBytes;
constexpr unsigned kFewLds = kFewPairs + kWaves * 4 * 8;
static_assert(kTileTokens * 32 == kFewWaveBytes && 4 * 128 * 4 == kFewWaveBytes, "a wavefront's room");

#define CQ_VIEW_KERNEL 0
#include "cq_chunk_few_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_chunk_few_kernel.hpp"
#undef CQ_VIEW_KERNEL

template <class Kernel, class Args>
cq_status launch(Kernel kernel, LdsKernelSetup& setup, unsigned lds, const Args& a, hipStream_t stream, bool few)
{
    if (setup.ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
    const ChunkLdsPlan p = chunk_lds_plan(a.f, a.n_q_heads, a.m);
    const int items = a.batch * a.n_split;
    const int per_head = items < p.wgs_per_head ? items : p.wgs_per_head;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(per_head * a.f.n_kv_heads)), dim3(kWaves * 64), lds, stream, a, few ? per_head : p.rb_log2, items);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

template <int C>
cq_status launch_rows(const ChunkViewArgs& a, int rows, hipStream_t stream)
{
    static LdsKernelSetup setup[3];
    if (rows <= 4) return launch(chunk_few_window_kernel<C>, setup[0], kFewLds, a, stream, true);
    if (rows <= kRows / 2) return launch(chunk_lds_window_kernel<C, true>, setup[1], kLdsBytes, a, stream, false);
    return launch(chunk_lds_window_kernel<C, false>, setup[2], kLdsBytes, a, stream, false);
}
template <int C>
cq_status launch_rows(const ChunkArgs& a, int rows, hipStream_t stream)
{
    static LdsKernelSetup setup[3];
    if (rows <= 4) return launch(chunk_few_kernel<C>, setup[0], kFewLds, a, stream, true);
    if (rows <= kRows / 2) return launch(chunk_lds_kernel<C, true>, setup[1], kLdsBytes, a, stream, false);
    return launch(chunk_lds_kernel<C, false>, setup[2], kLdsBytes, a, stream, false);
}

template <class Args>
cq_status launch_format(const Args& a, hipStream_t stream)
{
    // (row / qper is formed in floating point: exact for far more rows than are served here)
    const int64_t rows = (int64_t)a.m * (a.n_q_heads / a.f.n_kv_heads);
    if (a.f.b != 8 || a.f.head_dim != 128 || rows > kChunkLdsRows) return CQ_ERR_UNSUPPORTED;
    if (a.f.c == 8) return launch_rows<8>(a, (int)rows, stream);
    if (a.f.c == 4) return launch_rows<4>(a, (int)rows, stream);
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace

ChunkLdsPlan chunk_lds_plan(const Derived& f, int n_q_heads, int m)
{
    ChunkLdsPlan p;
    const int blocks = (m * (n_q_heads / f.n_kv_heads) + kRows - 1) / kRows;
    p.rb_log2 = blocks <= 1 ? 0 : (blocks <= 2 ? 1 : 2);
    p.wgs_per_head = f.n_kv_heads < 256 ? 256 / f.n_kv_heads : 1;      // one workgroup per CU
    return p;
}

cq_status launch_chunk_lds(const ChunkArgs& a, hipStream_t stream) { return launch_format(a, stream); }
cq_status launch_chunk_lds_window(const ChunkViewArgs& a, hipStream_t stream) { return launch_format(a, stream); }

}  // namespace cq
