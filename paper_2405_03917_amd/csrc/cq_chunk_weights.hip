// Attention weights of the last m tokens of every sequence, added up per cached token (cq_chunk_weights), for gfx950:
//   weights[n][h][i] = decay weights[n][h][i] + sum over rows r of KV head h of 2^(s_r,i - M_r) / L_r
// over the rows (query token, query head) of the KV head, s the causal scores in base 2.  Keys only.
//
// A row's M and L need all of its scores before the first weight is known, and the scores of a chunk are too many to be
// kept (four bytes each, where a token's codes are 16 to 64 for all rows together), so they are formed twice:
//   rows      every row's maximum and sum per piece of the context, one pass with a running maximum
//   columns   the scores again, 2^(s - M) times 1 / L, added over the rows in the registers of the lane that holds the
//             token, and one exchange between lanes per tile
// Both passes: a workgroup of 8 wavefronts serves one KV head, its key codebook (64 KB; CQ-8c10b: from L2) and up to
// 256 query rows in LDS; a wavefront takes 64-token tiles by itself, gathers their keys from the codebook straight into the
// operand of S^T = K Q^T (v_mfma_f32_32x32x16_f16: a lane's 8 channels are the centroids of its token's codes) and keeps
// them for all row blocks.  Every sum has a fixed order: equal calls give equal bits.
// Bound by the vector ALU, busy 0.72 to 0.80 of the time: of 1.07 M clocks of a pass over 4 x 32768 tokens of CQ-4c8b with 500 query tokens,
// 32 / 8 heads, the products take 0.52 M, an exponential per score at a quarter of the vector rate 0.51 M, a fused multiply-add before and
// one behind it 0.26 M, and they overlap in part: 1.17 ms for both passes, 913 TFLOP/s.  Short calls are two launches of 11 us each, the codebook's way to LDS among them.
#include <type_traits>

#include "cq_key_gather.hpp"
#include "cq_lds_gather.hpp"

namespace cq {
namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) u32x4 lds_q;
typedef __attribute__((address_space(3))) float2_t lds_f2;
typedef __attribute__((address_space(3))) int lds_i;

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBlockRows = 32;
constexpr int kGroupRows = 256;                         // query rows in LDS at a time
// LDS: key codebook, query rows, per row (M, 1 / L) and
// its position, the wavefronts' (maximum, sum) pairs, a word of each wavefront
constexpr unsigned kQueries = kBookBytes;
constexpr unsigned kQueryStride = 272;                  // (256 + 16: eight rows' pieces lie in different banks)
constexpr unsigned kRowStats = kQueries + kGroupRows * kQueryStride;
constexpr unsigned kRowPos = kRowStats + kGroupRows * 8;
constexpr unsigned kWavePairs = kRowPos + kGroupRows * 4;
constexpr unsigned kFlags = kWavePairs + kWaves * kGroupRows * 8;
constexpr unsigned kLds = kFlags + kWaves * 4;
static_assert(kLds <= 160 * 1024, "LDS of a CU");

__device__ __forceinline__ half8_t lds_half8(unsigned a) { return *(__attribute__((address_space(3))) half8_t*)(a); }

// The keys of a tile as A operands: lane (rc, kh) holds channels 16 s + 8 kh .. + 7 of tokens rc and 32 + rc.
template <int GH, int C, int B>
struct TileKeys {
    static constexpr int K = 1 << B;
    Tile<GH, B> rec[2];                                 // on their way: the records of both tokens
    half8_t kv[2][8];
    __device__ __forceinline__ void request(const uint8_t* tile, int rc)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const int u = 32 * tb + rc;
#pragma unroll
            for (int p = 0; p < GH / 16; ++p) rec[tb].lo[p] = *reinterpret_cast<const u32x4*>(tile + p * 1024 + u * 16);
            if constexpr (B == 10) rec[tb].hi = *reinterpret_cast<const unsigned*>(tile + kTileTokens * GH + u * 4);
            else rec[tb].hi = 0;
        }
    }
    __device__ __forceinline__ void gather(const uint16_t* ck_head, int rc, int kh)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const int u = 32 * tb + rc;
            Unrotate un;
            un.bytes = (unsigned)(GH - u) & 3u;
            un.dwords = ((unsigned)(GH - u) & (unsigned)(GH - 1)) >> 2;
            unsigned d[GH / 4];
            group_order<GH, B>(rec[tb], un, d);
            const unsigned base = (unsigned)kh * 4096;
            if constexpr (B == 10) {
                const unsigned hi = __builtin_amdgcn_alignbit(rec[tb].hi, rec[tb].hi, (32 - 2 * u) & 31);  // two bits per group
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const int g = 2 * s + kh;
                    const unsigned code = ((d[s >> 1] >> (16 * (s & 1) + 8 * kh)) & 0xffu) | ((hi >> (2 * g)) & 3u) << 8;
                    kv[tb][s] = *reinterpret_cast<const half8_t*>(ck_head + ((size_t)g * K + code) * C);
                }
            } else if constexpr (C == 8) {
#pragma unroll
                for (int i = 0; i < GH / 4; ++i) d[i] >>= 8 * kh;
#pragma unroll
                for (int s = 0; s < 8; ++s) kv[tb][s] = lds_half8(entry<C>(d[s >> 1], 2 * (s & 1), base) + (unsigned)s * 8192);
            } else if constexpr (C == 4) {
#pragma unroll
                for (int i = 0; i < GH / 4; ++i) d[i] >>= 16 * kh;
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const CenVec<4> a = lds_centroid<4>(entry<C>(d[s], 0, base) + (unsigned)s * 8192);
                    const CenVec<4> b = lds_centroid<4>(entry<C>(d[s], 1, base) + (unsigned)s * 8192 + 2048);
                    kv[tb][s] = __builtin_bit_cast(half8_t, u32x4{a.w[0], a.w[1], b.w[0], b.w[1]});
                }
            } else {
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const unsigned z = kh ? d[2 * s + 1] : d[2 * s];
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = lds_centroid<2>(entry<C>(z, e, base) + (unsigned)s * 8192 + (unsigned)e * 1024).w[0];
                    kv[tb][s] = __builtin_bit_cast(half8_t, w);
                }
            }
        }
    }
};

// A block of 32 query rows as B operands: lane (rc, kh) holds channels 16 s + 8 kh .. + 7 of row rc in q[s].
__device__ __forceinline__ half8_t read_query(int rb, int s, int rc, int kh)
{
    return lds_half8((unsigned)rc * kQueryStride + (unsigned)kh * 16 + (unsigned)rb * (kBlockRows * kQueryStride) + kQueries + (unsigned)s * 32);
}
// One of 16 products of a block's scores of the tile's 64 tokens: acc[tb][i] is token 32 tb + 8 (i / 4) + 4 kh + i % 4, query rc.
template <int GH, int C, int B>
__device__ __forceinline__ void product(const TileKeys<GH, C, B>& keys, const half8_t (&q)[8], float16_t (&acc)[2], int k)
{
    const int s = k >> 1, tb = k & 1;
    if (s == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[tb][i] = 0.f;
    }
    acc[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(keys.kv[tb][s], q[s], acc[tb], 0, 0, 0);
}

// Sum over the 32 lanes of a half-wavefront of 32 values each: lane rc receives the sum of value rc.
__device__ __forceinline__ float sum_over_rows(float (&v)[32], int rc)
{
    auto bits = [](float x) { return __float_as_uint(x); };
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(bits(v[i]), bits(v[i + 16]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    auto halve = [&](int n, bool upper, auto from) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float mine = upper ? v[i + n] : v[i], other = upper ? v[i] : v[i + n];
            v[i] = mine + __uint_as_float(from(bits(other)));
        }
    };
    halve(8, rc & 8, [](unsigned x) { return dpp_from<0x128>(x); });     // row_ror:8, lane ^ 8
    halve(4, rc & 4, [](unsigned x) { return dpp_from<0x141>(x); });     // row_half_mirror, lane ^ 7
    halve(2, rc & 2, [](unsigned x) { return dpp_from<0x4E>(x); });      // quad_perm, lane ^ 2
    halve(1, rc & 1, [](unsigned x) { return dpp_from<0xB1>(x); });      // lane ^ 1
    return v[0];
}

template <int GH, int C, int B, int NB, bool COLUMNS>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kThreads) void chunk_weights_kernel(ChunkWeightsArgs a, int items, int per_head)
{
    constexpr int D = 128, K = 1 << B, TILE = kTileTokens * GH * B / 8;
    extern __shared__ float smem[];
    (void)smem;
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rc = lane & 31, kh = lane >> 5;
    const int hkv = blockIdx.x % a.f.n_kv_heads;
    const int qper = a.n_q_heads / a.f.n_kv_heads, rows = a.m * qper;
    constexpr int kRows = NB * kBlockRows;
    const int groups = (rows + kRows - 1) / kRows;
    const uint16_t* ck_head = a.k_centroids + (size_t)hkv * GH * K * C;
    if constexpr (B == 8) {
        const u32x4* src = reinterpret_cast<const u32x4*>(ck_head);
        u32x4 book[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) book[i] = src[i * kThreads + tid];
#pragma unroll
        for (int i = 0; i < 8; ++i) *(lds_q*)((unsigned)(i * kThreads + tid) * 16) = book[i];
    }
    // (a negative scale turns the queries' signs; one of zero stands for one so small that every weight is 1: 0 times a masked
    // -infinity is no number)
    const float scale = a.scale_log2e == 0.f ? 1e-37f : fabsf(a.scale_log2e);
    const unsigned flip = a.scale_log2e < 0.f ? 0x80008000u : 0u;

#pragma unroll 1
    for (int item = blockIdx.x / a.f.n_kv_heads; item < items; item += per_head) {
        // rows: (sequence, group of rows, piece of the context); columns: (sequence, piece), and all groups in turn
        const int split = item % a.n_split;
        const int rest = item / a.n_split;
        const int n = COLUMNS ? rest : rest / groups;
        int t_n = a.t;
        if (a.seq_lens) t_n = min(max(a.seq_lens[n], a.m), a.t);
        const int pos0 = t_n - a.m;
        const int n_tiles = (t_n + kTileTokens - 1) / kTileTokens;
        const int tile0 = split * a.tiles_per_split, tile1 = min(tile0 + a.tiles_per_split, n_tiles);
        const size_t stream = (size_t)n * a.f.n_kv_heads + hkv;
        float2* const stats = a.stats + stream * rows * a.row_splits;
#pragma unroll 1
        for (int group = COLUMNS ? 0 : rest % groups; group < groups; group += COLUMNS ? 1 : groups) {
            const int row0 = group * kRows;
            const int blocks = min(NB, (rows - row0 + kBlockRows - 1) / kBlockRows);
            TileKeys<GH, C, B> keys;
            int tile = tile0 + wave;
            auto tile_at = [&](int i) { return a.k_codes + a.map.tile_index(n, hkv, min(i, n_tiles - 1)) * TILE; };
            keys.request(tile_at(tile), rc);
            lds_barrier();                                  // (what the last rows' readers used is free)
            // ---- the rows: queries, positions, and (columns) their statistics
            float q2 = 0.f;
            for (int i = tid; i < blocks * kBlockRows * 16; i += kThreads) {
                const int r = i >> 4, piece = i & 15;
                const int row = min(row0 + r, rows - 1), j = row / qper;
                u32x4 w = *reinterpret_cast<const u32x4*>(a.q + (((size_t)n * a.m + j) * a.n_q_heads + hkv * qper + (row - j * qper)) * D + piece * 8);
                w ^= flip;
                *(lds_q*)(kQueries + (unsigned)r * kQueryStride + (unsigned)piece * 16) = w;
                float mine = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const half2_t h = __builtin_bit_cast(half2_t, w[e]);
                    mine = __builtin_amdgcn_fdot2(h, h, mine, false);
                }
                q2 = fmaxf(q2, mine);                       // (of a piece: the row's square is 16 times the largest at most)
                if (piece == 0) *(lds_i*)(kRowPos + (unsigned)r * 4) = pos0 + j;
            }
            if constexpr (COLUMNS) {
                for (int r = tid; r < blocks * kBlockRows; r += kThreads) {
                    float2_t st = {3e38f, 0.f};             // (rows behind the last: weight 2^-inf times 0)
                    if (row0 + r < rows) {
                        const float2* p = stats + (size_t)(row0 + r) * a.row_splits;
                        float m = kNoScore, l = 0.f;
                        for (int s = 0; s < a.row_splits; ++s) {
                            const float2 x = p[s];
                            const float top = fmaxf(m, x.x);
                            l = __builtin_fmaf(l, __builtin_amdgcn_exp2f(m - top), x.y * __builtin_amdgcn_exp2f(x.x - top));
                            m = top;
                        }
                        st = float2_t{m, 1.f / l};
                    }
                    *(lds_f2*)(kRowStats + (unsigned)r * 8) = st;
                }
            }
            // Scores that could pass 2^24 are scaled before their maximum is taken, others inside the exponent, where a
            // rounding of the product costs nothing.
            const bool mine_large = scores_may_be_large(16.f * q2, scale, 0x1p24f);
            if (lane == 0) *(lds_i*)(kFlags + (unsigned)wave * 4) = mine_large;
            lds_barrier();
            const bool large = __builtin_amdgcn_ballot_w64(lane < kWaves && *(lds_i*)(kFlags + (unsigned)(lane & (kWaves - 1)) * 4) != 0) != 0;
            const float mult = large ? 1.f : scale, early = large ? scale : 1.f;

            if constexpr (!COLUMNS) {
                for (int r = lane; r < kRows; r += 64) *(lds_f2*)(kWavePairs + (unsigned)(wave * kGroupRows + r) * 8) = float2_t{kNoScore, 0.f};
                asm volatile("" ::: "memory");              // (a wavefront's LDS operations keep their order)
            }
#pragma unroll 1
            for (; tile < tile1; tile += kWaves) {
                half8_t q[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) q[k] = read_query(0, k, rc, kh);
                keys.gather(ck_head, rc, kh);
                keys.request(tile_at(tile + kWaves), rc);
                const bool hides = large || tile * kTileTokens + kTileTokens - 1 > pos0;
                auto mask = [&](int rb, float16_t (&acc)[2]) {
                    if (!hides) return;
                    const int rel = *(lds_i*)(kRowPos + (unsigned)(rb * kBlockRows + rc) * 4) - tile * kTileTokens - 4 * kh;
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[tb][i] = rel >= 32 * tb + 8 * (i >> 2) + (i & 3) ? acc[tb][i] * early : -INFINITY;
                };
                // The vector work on a block's scores goes slice by slice between the products of the next block, and behind each
                // product's operand the same one of the block after it is requested.
                auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
                auto between = [&](int rb, float16_t (&next)[2], auto last, auto&& slice) {
                    const int after = min(rb + 2, blocks - 1);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        if constexpr (!decltype(last)::value) {
                            product(keys, q, next, k);
                            if (k & 1) q[k >> 1] = read_query(after, k >> 1, rc, kh);
                        }
                        slice(k);
                        fence();
                    }
                };
                float16_t acc[2][2];
                fence();
#pragma unroll
                for (int k = 0; k < 16; ++k) product(keys, q, acc[0], k);
                fence();
                if constexpr (NB > 1) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) q[k] = read_query(min(1, blocks - 1), k, rc, kh);
                }
                fence();
                float col[32];
                if constexpr (COLUMNS) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) col[i] = 0.f;
                }
                auto here = [](float& v) { asm volatile("" : "+v"(v)); };   // (formed here, not where it is next used)
                auto value = [&](float16_t (&x)[2], int i) { return x[i >> 4][i & 15]; };
                auto block = [&](int rb, float16_t (&x)[2], float16_t (&next)[2], auto last) {
                    mask(rb, x);
                    if constexpr (!COLUMNS) {
                        // (a row's two half-wavefronts share reference and sum)
                        const unsigned at = kWavePairs + (unsigned)(wave * kGroupRows + rb * kBlockRows + rc) * 8;
                        const float2_t old = *(lds_f2*)at;
                        float top = -INFINITY, ref = 0.f, alpha = 0.f, sum[2] = {0.f, 0.f};
                        between(rb, next, last, [&](int k) {
                            if (k < 4) {
#pragma unroll
                                for (int i = 8 * k; i < 8 * k + 8; i += 2) top = fmaxf(top, fmaxf(value(x, i), value(x, i + 1)));
                                here(top);
                            } else if (k == 4) {
                                const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                                ref = fmaxf(old[0], fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * mult);
                                alpha = __builtin_amdgcn_exp2f(old[0] - ref);
                                here(alpha);
                            } else {
#pragma unroll
                                for (int i = 3 * (k - 5); i < 3 * (k - 5) + 3 && i < 32; ++i)
                                    sum[i & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(value(x, i), mult, -ref));
                                here(sum[0]);
                                here(sum[1]);
                            }
                        });
                        const float mine = sum[0] + sum[1];
                        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
                        if (kh == 0) *(lds_f2*)at = float2_t{ref, __builtin_fmaf(old[1], alpha, __uint_as_float(r[0]) + __uint_as_float(r[1]))};
                    } else {
                        const float2_t st = *(lds_f2*)(kRowStats + (unsigned)(rb * kBlockRows + rc) * 8);
                        between(rb, next, last, [&](int k) {
#pragma unroll
                            for (int i = 2 * k; i < 2 * k + 2; ++i)
                                col[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(value(x, i), mult, -st[0])), st[1], col[i]);
                            here(col[2 * k]);
                            here(col[2 * k + 1]);
                        });
                    }
                };
                if constexpr (NB == 1) {
                    block(0, acc[0], acc[1], std::true_type{});
                } else {
                    int rb = 0;
#pragma unroll 1
                    for (; rb + 2 < blocks; rb += 2) {
                        block(rb, acc[0], acc[1], std::false_type{});
                        block(rb + 1, acc[1], acc[0], std::false_type{});
                    }
                    if (rb + 1 < blocks) {
                        block(rb, acc[0], acc[1], std::false_type{});
                        block(rb + 1, acc[1], acc[0], std::true_type{});
                    } else {
                        block(rb, acc[0], acc[1], std::true_type{});
                    }
                }
                if constexpr (COLUMNS) {
                    const float sum = sum_over_rows(col, rc);
                    const int tok = tile * kTileTokens + (rc >> 4) * 32 + 8 * (rc >> 2 & 3) + 4 * kh + (rc & 3);
                    if (tok < t_n) {
                        float* const w = a.weights + stream * a.weights_stride + tok;
                        *w = group > 0 ? *w + sum : a.decay != 0.f ? __builtin_fmaf(a.decay, *w, sum) : sum;
                    }
                }
            }
            if constexpr (!COLUMNS) {
                // ---- the wavefronts' pairs of every row
                auto merged = [](float m0, float l0, float m1, float l1) {
                    const float m = fmaxf(m0, m1);
                    return float2_t{m, __builtin_fmaf(l0, __builtin_amdgcn_exp2f(m0 - m), l1 * __builtin_amdgcn_exp2f(m1 - m))};
                };
                lds_barrier();
                for (int r = tid; r < kRows && row0 + r < rows; r += kThreads) {
                    float2_t x = *(lds_f2*)(kWavePairs + (unsigned)r * 8);
#pragma unroll
                    for (int w = 1; w < kWaves; ++w) {
                        const float2_t y = *(lds_f2*)(kWavePairs + (unsigned)(w * kGroupRows + r) * 8);
                        x = merged(x[0], x[1], y[0], y[1]);
                    }
                    stats[(size_t)(row0 + r) * a.row_splits + split] = make_float2(x[0], x[1]);
                }
            }
        }
    }
}

template <int GH, int C, int B, int NB>
cq_status launch_passes(const ChunkWeightsArgs& a_in, hipStream_t stream)
{
    ChunkWeightsArgs a = a_in;
    const int qper = a.n_q_heads / a.f.n_kv_heads, rows = a.m * qper;
    const int groups = (rows + NB * kBlockRows - 1) / (NB * kBlockRows);
    const int n_tiles = (a.t + kTileTokens - 1) / kTileTokens;
    const int resident = chunk_weights_resident(a.f.n_kv_heads);
    for (int pass = 0; pass < 2; ++pass) {
        a.n_split = pass == 0 ? a.row_splits : chunk_weights_pieces(n_tiles, a.batch, resident);
        a.tiles_per_split = (n_tiles + a.n_split - 1) / a.n_split;
        const int64_t items = (int64_t)a.batch * a.n_split * (pass == 0 ? groups : 1);
        if (items > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
        const int per_head = items < resident ? (int)items : resident;
        static LdsKernelSetup setup[2];
        auto kernel = pass == 0 ? chunk_weights_kernel<GH, C, B, NB, false> : chunk_weights_kernel<GH, C, B, NB, true>;
        if (setup[pass].ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(per_head * a.f.n_kv_heads)), dim3(kThreads), kLds, stream, a, (int)items, per_head);
        if (hipGetLastError() != hipSuccess) return CQ_ERR_HIP;
    }
    return CQ_OK;
}

template <int GH, int C, int B>
cq_status launch_rows(const ChunkWeightsArgs& a, hipStream_t stream)
{
    const int blocks = (a.m * (a.n_q_heads / a.f.n_kv_heads) + kBlockRows - 1) / kBlockRows;
    // One block of rows needs no second operand of products and no second set of sums (158 registers of 250).  As one of up to eight, us:
    // CQ-8c8b 32 heads, 1 x 4096, 32 rows 13.9 instead of 13.4, 4 x 32768 128 instead of 121; CQ-2c8b 2 x 9000, 16 rows 36.2 instead of 32.8.
    if (blocks <= 1) return launch_passes<GH, C, B, 1>(a, stream);
    return launch_passes<GH, C, B, 8>(a, stream);
}

}  // namespace

int chunk_weights_resident(int n_kv_heads) { return n_kv_heads < 256 ? 256 / n_kv_heads : 1; }

// Pieces of a context of n_tiles tiles where `base` (sequences, or sequences and groups of rows) share a KV head's workgroups:
// as many as fill the CUs, of at least a tile for every wavefront.
int chunk_weights_pieces(int n_tiles, int64_t base, int resident)
{
    const int64_t want = (resident + base - 1) / base, most = (n_tiles + kWaves - 1) / kWaves;
    return (int)(want < most ? want : most);
}

int chunk_weights_row_splits(int n_tiles, int batch, int rows, int n_kv_heads)
{
    const int64_t groups = (rows + kGroupRows - 1) / kGroupRows;
    return chunk_weights_pieces(n_tiles, batch * groups, chunk_weights_resident(n_kv_heads));
}

cq_status launch_chunk_weights(const ChunkWeightsArgs& a, hipStream_t stream)
{
    if (a.f.head_dim != 128) return CQ_ERR_UNSUPPORTED;
    if (a.f.b == 10) return launch_rows<16, 8, 10>(a, stream);
    if (a.f.gh == 16) return launch_rows<16, 8, 8>(a, stream);
    if (a.f.gh == 32) return launch_rows<32, 4, 8>(a, stream);
    if (a.f.gh == 64) return launch_rows<64, 2, 8>(a, stream);
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace cq
