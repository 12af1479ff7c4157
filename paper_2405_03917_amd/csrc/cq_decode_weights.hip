// Attention weights added up per cached token (cq_decode_attention_weights), for gfx950: what follows the attention
// kernel, which left every score of the call (base 2) and, per context split, the softmax reference m and sum l.
//
//   weights[n][h][i] = decay weights[n][h][i] + sum over the query heads q of KV head h of 2^(s_q,i - M_q) / L_q,
//   M_q = max over splits of m, L_q = sum over splits of l 2^(m - M_q)
//
// A weight needs the sum over the whole context, which no workgroup of the attention kernel has while others still run,
// and with grouped queries a token's sum runs over workgroups; hence a second launch, which merges the output's
// splits too (the attention kernel does both itself where one query head's context is short: launch_decode_view).  Every sum is
// formed by one thread in a fixed order: no atomics, equal calls give equal bits.
// Bound by memory: 4 bytes a query head and token (the scores, mostly still in the caches) and 8 a KV head and token.  Of
// 4 x 131072 tokens, 32 heads: 37 us for 67 MB of scores and 134 of accumulators (5.4 TB/s).  Tokens per thread 4: 8 or 16 are slower.
#include "cq_decode_split.hpp"

namespace cq {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerThread = 4;
constexpr int kTokens = kThreads * kTokensPerThread;

__global__ __launch_bounds__(kThreads) void decode_weights_kernel(DecodeViewArgs a, int merge_wgs, int blocks)
{
    extern __shared__ float2 stats[];                       // (M, 1 / L) per query head of the KV head
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int D = a.f.head_dim, part = D + kPartialHeader;
    if ((int)blockIdx.x < merge_wgs) {                      // two rows of the output
        const int row = 2 * blockIdx.x + (tid >> 7);
        if (row < a.batch * a.n_q_heads)
            merge_splits<false>(a.partials + (size_t)row * a.n_split * part, a.n_split, D,
                                a.out + (size_t)(row / a.n_q_heads) * a.out_batch_stride + (size_t)(row % a.n_q_heads) * D, tid & 127, 128);
        return;
    }
    const int idx = blockIdx.x - merge_wgs;
    const int block = idx % blocks, stream = idx / blocks;
    const int n = stream / a.f.n_kv_heads, hkv = stream % a.f.n_kv_heads;
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    int t_n = a.t;
    if (a.seq_lens) t_n = min(max(a.seq_lens[n], 1), a.t);
    const int first = block * kTokens;
    if (first >= t_n) return;
    const size_t row0 = (size_t)n * a.n_q_heads + (size_t)hkv * qper;
    float* acc = a.weights + (size_t)stream * a.weights_stride;
    // The accumulators and the first head's scores are requested ahead of the statistics (of four heads all at once: no faster).
    float old[kTokensPerThread], w[kTokensPerThread], x[kTokensPerThread];
    auto request = [&](int h) {
#pragma unroll
        for (int k = 0; k < kTokensPerThread; ++k) x[k] = a.scores[(row0 + h) * a.score_stride + min(first + k * kThreads + tid, t_n - 1)];
    };
#pragma unroll
    for (int k = 0; k < kTokensPerThread; ++k) {
        old[k] = a.decay != 0.f ? acc[min(first + k * kThreads + tid, t_n - 1)] : 0.f;      // (without decay the accumulators are not read)
        w[k] = 0.f;
    }
    request(0);
    for (int h = wave; h < qper; h += kThreads / 64) {
        const float2 st = row_stats<false>(a, row0 + h, lane);
        if (lane == 0) stats[h] = st;
    }
    __syncthreads();
    for (int h = 0; h < qper; ++h) {
        const float2 st = stats[h];
#pragma unroll
        for (int k = 0; k < kTokensPerThread; ++k) w[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(x[k] - st.x), st.y, w[k]);
        if (h + 1 < qper) request(h + 1);
    }
#pragma unroll
    for (int k = 0; k < kTokensPerThread; ++k) {
        const int tok = first + k * kThreads + tid;
        if (tok < t_n) acc[tok] = __builtin_fmaf(a.decay, old[k], w[k]);
    }
}

}  // namespace

cq_status launch_decode_weights(const DecodeViewArgs& a, hipStream_t stream)
{
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int blocks = (a.t + kTokens - 1) / kTokens;
    const int merge_wgs = a.n_split > 1 ? (a.batch * a.n_q_heads + 1) / 2 : 0;
    const int64_t grid = (int64_t)merge_wgs + (int64_t)a.batch * a.f.n_kv_heads * blocks;
    if (grid > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL(decode_weights_kernel, dim3((unsigned)grid), dim3(kThreads), sizeof(float2) * (size_t)qper, stream, a, merge_wgs, blocks);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace cq
