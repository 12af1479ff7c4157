// The 8-bit block cache, its codes: cq_append_q8 (rotation, block scales, codes, older tokens under a scale that grew) and
// cq_dequantize_q8, for gfx950.
//
//   key pair (i, i + 64) at position p:  k'_i = k_i cos(p th_i) - k_{i+64} sin(p th_i),  k'_{i+64} = k_{i+64} cos + k_i sin
//   block of 64 tokens and a head:  s = max(s before, if the block holds older tokens; need(largest |x| of the new ones))
//   need: integers fp32(largest / 127); e4m3 the smallest power of two >= largest / 448
//   code = nearest(x / s), ties to even; codes of older tokens, where s grew: nearest(c s_before / s)
//
// Which side of a border a number lies on is decided in 64 bits, on cosines and sines that are products of two table entries, off by
// 2^-50 + 2^-51 p th_i at most (th_i and its product with a position are rounded): codes do not depend on how a call is cut.
// fp64 costs what fp32 does here (no packed fp32), but for conversions; of values, which are fp16, fp32 decides where it can.
// e4m3 scales are powers of two so that a growing scale moves codes without rounding them again (but into
// subnormals); integers use the whole range instead: a power of two would cost up to a bit of seven.
// Bound by memory where there is much of it: 4 x 8192 tokens of 8 heads with 32 heads' queries, 738 MB, 149 us; 6 x 500 of 32 heads, 123 MB, 42 us, of
// few workgroups with a reduction each; single tokens by latency: length, page, scale, reduction, division, one after another.
#include <algorithm>

#include "cq_q8.hpp"

namespace cq {
namespace {

constexpr int kThreads = 256;

// A number in units of its block's scale (127 or 448 at most, but for the rounding of a scale) as its code byte, with other bits
// above it.  Integers: the sum with 1.5 x 2^52 has the nearest one in its last bits.  e4m3: x rounded to fp32 so that rounding once
// more is right: what lies below the 20 upper bits of the mantissa becomes one bit under them; zero, of either sign, has one code.
constexpr double kMagic64 = 6755399441055744.0;
constexpr float kMagic32 = 12582912.f;
__device__ __forceinline__ unsigned low_word(double x) { return (unsigned)__builtin_bit_cast(unsigned long long, x); }
__device__ __forceinline__ float to_odd(double x)
{
    const unsigned long long b = __builtin_bit_cast(unsigned long long, x + 0.0);
    return (float)__builtin_bit_cast(double, (b & 0xffffffff00000000ULL) | ((unsigned)b ? 0x20000000u : 0u));
}
// Four such bytes of integers' sums, and of e4m3 numbers in fp32, as a word of the cache.
__device__ __forceinline__ unsigned pack_integers(unsigned a, unsigned b, unsigned c, unsigned d)
{
    const unsigned lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return (lo | hi) ^ 0x80808080u;
}
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d)
{
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// x / s of an s whose reciprocal is `inv`, as IEEE division gives it (but for quotients no code depends on).
__device__ __forceinline__ double quotient(double x, double s, double inv)
{
    const double y = x * inv;
    return fma(fma(-y, s, x), inv, y);
}
// x / s, four of them.  (An e4m3 scale is a power of two.)
template <int KIND>
__device__ __forceinline__ unsigned codes4(const double* x, double s, double inv)
{
    if constexpr (KIND == CQ_Q8_INT8)
        return pack_integers(low_word(quotient(x[0], s, inv) + kMagic64), low_word(quotient(x[1], s, inv) + kMagic64), low_word(quotient(x[2], s, inv) + kMagic64),
                             low_word(quotient(x[3], s, inv) + kMagic64));
    else return pack_e4m3(to_odd(x[0] * inv), to_odd(x[1] * inv), to_odd(x[2] * inv), to_odd(x[3] * inv));
}
template <int KIND>
__device__ __forceinline__ float need_of(double largest)
{
    if constexpr (KIND == CQ_Q8_INT8) return (float)(largest / 127.0);
    const unsigned long long bits = __builtin_bit_cast(unsigned long long, largest / 448.0);
    return (float)__builtin_bit_cast(double, (bits + 0xfffffffffffffULL) & (0x7ffULL << 52));
}

template <class T>
__device__ __forceinline__ T wave_max(T x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T y = __shfl_xor(x, d);
        x = x > y ? x : y;
    }
    return x;
}

// the larger magnitude of two pairs of fp16 numbers, as bits
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned larger_halves(unsigned a, unsigned b)
{
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, a), __builtin_bit_cast(ushort2_t, b & 0x7fff7fffu)));
}
__device__ __forceinline__ float largest_half(unsigned w) { return (float)__builtin_bit_cast(_Float16, (unsigned short)max(w & 0xffffu, w >> 16)); }

// cos, sin of (64 tile + u) theta_i
__device__ __forceinline__ double2 angle_of(double2 tile, double2 lane)
{
    return make_double2(fma(tile.x, lane.x, -tile.y * lane.y), fma(tile.y, lane.x, tile.x * lane.y));
}

// Where the entry of pair i and token u lies in the second half of the table: [i % 16][u][i / 16], so that threads of the kernel
// that writes tiles, 16 pairs of a token each, read 1 KB of it together.
__device__ __forceinline__ int lane_entry(int u, int i) { return ((i & 15) * kTileTokens + u) * (kQ8Pairs / 16) + (i >> 4); }

// A block's scale from the largest new magnitude and the scale before (0 of a block that holds no older tokens); `grown`: the
// older tokens' codes change by `ratio`.
struct BlockScale {
    float scale;
    double s, inv, ratio;
    bool grown;
};
template <int KIND>
__device__ __forceinline__ BlockScale block_scale(double largest, bool has_old, float before)
{
    BlockScale b;
    b.scale = fmaxf(before, need_of<KIND>(largest));
    b.s = b.scale;
    b.inv = b.scale > 0.f ? 1.0 / b.s : 0.0;
    b.grown = has_old && b.scale > before;
    b.ratio = b.grown ? (double)before * b.inv : 1.0;
    return b;
}
// Four older codes of a block whose scale grew by 1 / ratio.  Of integers the ratio is rounded (twice: 2^-52 of it), and ties, every odd code
// where a scale doubles, must not fall to either side for that.  So c ratio is rounded to a multiple of 2^-36 first (the last place
// of 1.5 x 2^16 and a little): from within 2^-45 a tie comes back to itself, and what is no tie stays on its side, 2^-32 away or more.
// (c b / s - (k + 1/2) is (2 c b - (2 k + 1) s) / 2 s, of 24-bit b and s with s < 2^8 b where half a step is reached at all.)
constexpr double kSnap64 = 98304.0;
template <int KIND>
__device__ __forceinline__ unsigned regrown4(unsigned w, const BlockScale& b)
{
    double x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned byte = (w >> (8 * i)) & 0xffu;
        x[i] = KIND == CQ_Q8_INT8 ? (double)((int)byte - 128) : (double)__builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
        if (KIND == CQ_Q8_INT8) x[i] = fma(x[i], b.ratio, kSnap64) + (kMagic64 - kSnap64);
    }
    if constexpr (KIND == CQ_Q8_INT8) return pack_integers(low_word(x[0]), low_word(x[1]), low_word(x[2]), low_word(x[3]));
    else return codes4<KIND>(x, 1.0, b.ratio);
}
template <int KIND>
__device__ __forceinline__ q8_u4 regrown16(q8_u4 w, const BlockScale& b)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = regrown4<KIND>(w[i], b);
    return w;
}

// Queries: a thread rotates pairs 8 o .. 8 o + 7 of `q_heads` heads of a row, in fp32 (2^-24 of a product is nothing beside the 2^-11 of
// the fp16 they are rounded to).
__device__ __forceinline__ void rotate_queries(const Q8AppendArgs& a, unsigned idx, int tid)
{
    const int groups = a.n_q_heads / a.q_heads;
    const int64_t item = (int64_t)idx * (kThreads / 8) + (tid >> 3);
    const int o = tid & 7;
    const int64_t row = item / groups;
    const int group = (int)(item % groups);
    if (row >= (int64_t)a.batch * a.m) return;
    const int n = (int)(row / a.m), j = (int)(row % a.m);
    const int p = a.length(n) - a.m + j;
    if (p < 0) return;
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double2 r = angle_of(a.tile_tab[(size_t)(p >> 6) * kQ8Pairs + 8 * o + i], a.lane_tab[lane_entry(p & 63, 8 * o + i)]);
        c[i] = (float)r.x;
        s[i] = (float)r.y;
    }
    const uint16_t* src = a.q + n * a.q_batch_stride + j * a.q_row_stride + (size_t)group * a.q_heads * kQ8Head + 8 * o;
    uint16_t* dst = a.q_out + ((size_t)row * a.n_q_heads + (size_t)group * a.q_heads) * kQ8Head + 8 * o;
#pragma unroll 4
    for (int h = 0; h < a.q_heads; ++h) {
        const q8_half8 lo = *reinterpret_cast<const q8_half8*>(src + h * kQ8Head), hi = *reinterpret_cast<const q8_half8*>(src + h * kQ8Head + 64);
        q8_half8 y, z;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = (_Float16)fmaf((float)lo[i], c[i], -(float)hi[i] * s[i]);
            z[i] = (_Float16)fmaf((float)hi[i], c[i], (float)lo[i] * s[i]);
        }
        *reinterpret_cast<q8_half8*>(dst + h * kQ8Head) = y;
        *reinterpret_cast<q8_half8*>(dst + h * kQ8Head + 64) = z;
    }
}

// One token per sequence: a wavefront per sequence and head.  Lane i has channels i and i + 64 of the key and 2 i and 2 i + 1 of the
// value; older codes are read where their scale grew.
template <int KIND>
__global__ __launch_bounds__(kThreads) void append_token_q8_kernel(Q8AppendArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x >= a.kv_wgs) return rotate_queries(a, blockIdx.x - a.kv_wgs, tid);
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (item >= (int64_t)a.batch * a.n_kv_heads) return;
    const int n = (int)(item / a.n_kv_heads), h = (int)(item % a.n_kv_heads);
    const int p = a.length(n) - 1;
    if (p < 0) return;
    const int tile = p / kTileTokens, u = p % kTileTokens;
    const size_t at = a.cache.map.tile_index(n, h, tile);
    const float k_before = u ? a.cache.scales[0][at] : 0.f, v_before = u ? a.cache.scales[1][at] : 0.f;
    const uint16_t* x_k = a.x[0] + n * a.x_batch_stride + h * kQ8Head;
    const unsigned v = *reinterpret_cast<const unsigned*>(a.x[1] + n * a.x_batch_stride + h * kQ8Head + 2 * lane);
    const double x0 = (double)(float)__builtin_bit_cast(_Float16, x_k[lane]), x1 = (double)(float)__builtin_bit_cast(_Float16, x_k[64 + lane]);
    double y[4] = {x0, x1, (double)(float)__builtin_bit_cast(_Float16, (unsigned short)v), (double)(float)__builtin_bit_cast(_Float16, (unsigned short)(v >> 16))};
    if (a.tile_tab) {
        const double2 r = angle_of(a.tile_tab[(size_t)tile * kQ8Pairs + lane], a.lane_tab[lane_entry(u, lane)]);
        y[0] = fma(x0, r.x, -x1 * r.y);
        y[1] = fma(x1, r.x, x0 * r.y);
    }
    const BlockScale k_scale = block_scale<KIND>(wave_max(fmax(fabs(y[0]), fabs(y[1]))), u > 0, k_before);
    const BlockScale v_scale = block_scale<KIND>((double)wave_max(largest_half(v & 0x7fff7fffu)), u > 0, v_before);
    if (lane == 0) {
        a.cache.scales[0][at] = k_scale.scale;
        a.cache.scales[1][at] = v_scale.scale;
    }
    y[0] = KIND == CQ_Q8_INT8 ? quotient(y[0], k_scale.s, k_scale.inv) : y[0] * k_scale.inv;
    y[1] = KIND == CQ_Q8_INT8 ? quotient(y[1], k_scale.s, k_scale.inv) : y[1] * k_scale.inv;
    y[2] = KIND == CQ_Q8_INT8 ? quotient(y[2], v_scale.s, v_scale.inv) : y[2] * v_scale.inv;
    y[3] = KIND == CQ_Q8_INT8 ? quotient(y[3], v_scale.s, v_scale.inv) : y[3] * v_scale.inv;
    const unsigned codes = codes4<KIND>(y, 1.0, 1.0);
    uint8_t* k_dst = a.cache.codes[0] + at * kQ8TileBytes;
    uint8_t* v_dst = a.cache.codes[1] + at * kQ8TileBytes;
    k_dst[u * kQ8Head + lane] = (uint8_t)codes;
    k_dst[u * kQ8Head + 64 + lane] = (uint8_t)(codes >> 8);
    if (k_scale.grown)
        for (int i = lane; i < u * (kQ8Head / 16); i += 64) {
            q8_u4* w = reinterpret_cast<q8_u4*>(k_dst) + i;
            *w = regrown16<KIND>(*w, k_scale);
        }
    if (!v_scale.grown) {
        v_dst[2 * lane * kTileTokens + u] = (uint8_t)(codes >> 16);
        v_dst[(2 * lane + 1) * kTileTokens + u] = (uint8_t)(codes >> 24);
        return;
    }
    // ... of values each 16 bytes hold one channel's: its new one goes into them
    const int part = lane & 3, from = 16 * part;
#pragma unroll 2
    for (int i = 0; i < 8; ++i) {
        const int channel = 16 * i + (lane >> 2);
        const unsigned fresh = (unsigned)__shfl((int)codes, channel >> 1) >> (16 + 8 * (channel & 1)) & 0xffu;
        if (from > u) continue;
        q8_u4* at_w = reinterpret_cast<q8_u4*>(v_dst + channel * kTileTokens + from);
        const q8_u4 old = *at_w, now = regrown16<KIND>(old, v_scale);
        q8_u4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int before = min(max(u - from - 4 * k, 0), 4);        // bytes of older tokens
            const unsigned older = (unsigned)((1ULL << (8 * before)) - 1);
            w[k] = (now[k] & older) | (old[k] & ~older);
            if (before < 4 && u >= from + 4 * k) w[k] = (w[k] & ~(0xffu << (8 * before))) | fresh << (8 * before);
        }
        *at_w = w;
    }
}

// A workgroup: one tile of one sequence, `heads` heads in a row, keys or values; behind those, queries.
template <int KIND>
__global__ __launch_bounds__(kThreads, 4) void append_q8_kernel(Q8AppendArgs a)
{
    __shared__ double lds[2][kThreads / 64];                // largest magnitudes of the wavefronts, of this head and the next
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned idx = blockIdx.x;
    if (idx >= 2 * a.kv_wgs) return rotate_queries(a, idx - 2 * a.kv_wgs, tid);
    const int which = idx >= a.kv_wgs;
    idx -= which ? a.kv_wgs : 0;
    const int groups = a.n_kv_heads / a.heads;
    const int group = idx % groups;
    const int slot = (idx / groups) % a.slots, n = idx / groups / a.slots;
    const int t_n = a.length(n);
    const int start = max(t_n - a.m, 0);                    // the first new position
    const int tile = start / kTileTokens + slot;
    if (tile * kTileTokens >= t_n) return;
    const int lo = max(start - tile * kTileTokens, 0), hi = min(t_n - tile * kTileTokens, kTileTokens);    // new: lo .. hi - 1
    // (row 0 of the tile, which need not be a row of x: only rows of new tokens are read)
    const uint16_t* x0 = a.x[which] + n * a.x_batch_stride + (int64_t)(tile * kTileTokens - (t_n - a.m)) * a.x_row_stride;
    if (which == 0) {
        // ---- keys: thread (u, o) holds pairs 16 o .. 16 o + 15 of token u
        const int u = tid >> 2, o = tid & 3;
        const bool fresh = u >= lo && u < hi;
        double2 ang[16];
        if (a.tile_tab && fresh) {
#pragma unroll
            for (int i = 0; i < 16; ++i) ang[i] = angle_of(a.tile_tab[(size_t)tile * kQ8Pairs + 16 * o + i], a.lane_tab[lane_entry(u, 16 * o + i)]);
        }
        for (int i = 0; i < a.heads; ++i) {
            const int h = group * a.heads + i;
            const size_t at = a.cache.map.tile_index(n, h, tile);
            const float before = lo > 0 ? a.cache.scales[0][at] : 0.f;
            // (keys are rotated twice, for their scale and for their codes: held in between, they
            // would be 64 registers, and 3 wavefronts a SIMD instead of 4: 6 x 500 tokens of 32 heads 62.1 -> 60.4 us, 4 x 8192 of 8 196 -> 192.6,
            // with the rows read back)
            q8_u4 raw[4];
            double mine = 0.0;
            auto rotated4 = [&](int k, double* y, double* z) {
                const q8_half8 l = __builtin_bit_cast(q8_half8, raw[k >> 1]), r = __builtin_bit_cast(q8_half8, raw[2 + (k >> 1)]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double p = (double)(float)l[4 * (k & 1) + e], q = (double)(float)r[4 * (k & 1) + e];
                    if (a.tile_tab) {
                        y[e] = fma(p, ang[4 * k + e].x, -q * ang[4 * k + e].y);
                        z[e] = fma(q, ang[4 * k + e].x, p * ang[4 * k + e].y);
                    } else {
                        y[e] = p;
                        z[e] = q;
                    }
                }
            };
            if (fresh) {
                const uint16_t* src = x0 + u * a.x_row_stride + h * kQ8Head + 16 * o;
#pragma unroll
                for (int k = 0; k < 4; ++k) raw[k] = *reinterpret_cast<const q8_u4*>(src + 64 * (k >> 1) + 8 * (k & 1));
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    double y[4], z[4];
                    rotated4(k, y, z);
#pragma unroll
                    for (int e = 0; e < 4; ++e) mine = fmax(mine, fmax(fabs(y[e]), fabs(z[e])));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(raw[k]));
            }
            mine = wave_max(mine);
            double* all = lds[i & 1];
            if (lane == 0) all[wave] = mine;
            __syncthreads();
            const BlockScale b = block_scale<KIND>(fmax(fmax(all[0], all[1]), fmax(all[2], all[3])), lo > 0, before);
            if (tid == 0) a.cache.scales[0][at] = b.scale;
            uint8_t* dst = a.cache.codes[0] + at * kQ8TileBytes + u * kQ8Head + 16 * o;
            if (fresh) {
                q8_u4 w[2];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    double y[4], z[4];
                    rotated4(k, y, z);
                    w[0][k] = codes4<KIND>(y, b.s, b.inv);
                    w[1][k] = codes4<KIND>(z, b.s, b.inv);
                }
                *reinterpret_cast<q8_u4*>(dst) = w[0];
                *reinterpret_cast<q8_u4*>(dst + 64) = w[1];
            } else if (u < lo && b.grown) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    q8_u4* w = reinterpret_cast<q8_u4*>(dst + 64 * k);
                    *w = regrown16<KIND>(*w, b);
                }
            }
        }
        return;
    }
    // ---- values: thread (a4, o) holds tokens 4 a4 .. 4 a4 + 3 of channels 8 o .. 8 o + 7, a word of the cache per channel
    const int u = 4 * (lane & 15), o = (lane >> 4) + 4 * wave;
    const bool some_new = u + 4 > lo && u < hi, all_new = u >= lo && u + 4 <= hi;
    for (int r = 0; r < a.heads; ++r) {
        const int h = group * a.heads + r;
        const size_t at = a.cache.map.tile_index(n, h, tile);
        const float before = lo > 0 ? a.cache.scales[1][at] : 0.f;
        unsigned top = 0;
        q8_u4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = q8_u4{0, 0, 0, 0};
            if (u + k >= lo && u + k < hi) x[k] = *reinterpret_cast<const q8_u4*>(x0 + (u + k) * a.x_row_stride + h * kQ8Head + 8 * o);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = larger_halves(top, x[k][i]);
        const float mine = wave_max(largest_half(top));
        double* all = lds[r & 1];
        if (lane == 0) all[wave] = mine;
        __syncthreads();
        const BlockScale b = block_scale<KIND>(fmax(fmax(all[0], all[1]), fmax(all[2], all[3])), lo > 0, before);
        if (tid == 0) a.cache.scales[1][at] = b.scale;
        if (!some_new && !(b.grown && u < lo)) continue;
        uint8_t* dst = a.cache.codes[1] + at * kQ8TileBytes + (size_t)(8 * o) * kTileTokens + u;
        // an fp16 number over a power of two is exact in fp32; of integers' quotients there the code is right unless it lies within
        // 2^-15 of a border (2^-24 of 127 twice): then all of the thread's are computed as the keys' are
        unsigned codes[8];
        const float inv = (float)b.inv;
        float off = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[k] = fmaf((float)__builtin_bit_cast(q8_half8, x[k])[i], inv, 0.f);
                if (KIND == CQ_Q8_INT8) {
                    const float sum = f[k] + kMagic32;
                    off = fmaxf(off, fabsf(f[k] - (sum - kMagic32)));
                    f[k] = sum;
                }
            }
            if (KIND == CQ_Q8_INT8)
                codes[i] = pack_integers(__builtin_bit_cast(unsigned, f[0]), __builtin_bit_cast(unsigned, f[1]), __builtin_bit_cast(unsigned, f[2]), __builtin_bit_cast(unsigned, f[3]));
            else codes[i] = pack_e4m3(f[0], f[1], f[2], f[3]);
        }
        if (KIND == CQ_Q8_INT8 && !(off < 0.5f - 0x1p-15f)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                double f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = (double)(float)__builtin_bit_cast(q8_half8, x[k])[i];
                codes[i] = codes4<KIND>(f, b.s, b.inv);
            }
        }
        if (all_new) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<unsigned*>(dst + i * kTileTokens) = codes[i];
            continue;
        }
        const int olds = min(max(lo - u, 0), 4), news = min(max(hi - u, 0), 4);         // bytes: older tokens', then new ones', then none
        const unsigned older = (unsigned)((1ULL << (8 * olds)) - 1), fresh = (unsigned)((1ULL << (8 * news)) - 1) & ~older;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            unsigned* w = reinterpret_cast<unsigned*>(dst + i * kTileTokens);
            const unsigned old = *w, now = b.grown ? regrown4<KIND>(old, b) : old;
            *w = (now & older) | (codes[i] & fresh) | (old & ~(older | fresh));
        }
    }
}

// A workgroup: one tile of one sequence and head, keys or values.
template <int KIND>
__global__ __launch_bounds__(kThreads) void dequantize_q8_kernel(Q8DequantArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned idx = blockIdx.x;
    const int which = a.out[0] ? idx >= a.kv_wgs : 1;
    idx -= idx >= a.kv_wgs ? a.kv_wgs : 0;
    const int h = idx % a.n_kv_heads;
    const int slot = (idx / a.n_kv_heads) % a.slots, n = idx / a.n_kv_heads / a.slots;
    const int t_n = a.length(n);
    const int start = max(t_n - a.m, 0);
    const int tile = start / kTileTokens + slot;
    if (tile * kTileTokens >= t_n) return;
    const int lo = max(start - tile * kTileTokens, 0), hi = min(t_n - tile * kTileTokens, kTileTokens);
    const size_t at = a.cache.map.tile_index(n, h, tile);
    const float s = a.cache.scales[which][at];
    const uint8_t* src = a.cache.codes[which] + at * kQ8TileBytes;
    uint16_t* out = a.out[which] + n * a.out_batch_stride + (int64_t)(tile * kTileTokens - (t_n - a.m)) * a.out_row_stride + h * kQ8Head;
    if (which == 0) {
        const int u = tid >> 2, o = tid & 3;
        if (u < lo || u >= hi) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const q8_u4 w = *reinterpret_cast<const q8_u4*>(src + u * kQ8Head + 16 * o + 64 * k);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const q8_half8 c = q8_half8_of<KIND>(w[2 * e], w[2 * e + 1]);
                q8_half8 y;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = (_Float16)((float)c[i] * s);
                *reinterpret_cast<q8_half8*>(out + u * a.out_row_stride + 16 * o + 64 * k + 8 * e) = y;
            }
        }
        return;
    }
    const int u = 4 * (lane & 15), o = (lane >> 4) + 4 * wave;
    if (u + 4 <= lo || u >= hi) return;
    q8_half8 y[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned w = *reinterpret_cast<const unsigned*>(src + (8 * o + i) * kTileTokens + u);
        half2_t c[2];
        q8_halves<KIND>(w, &c[0], &c[1]);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k][i] = (_Float16)((float)c[k >> 1][k & 1] * s);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (u + k >= lo && u + k < hi) *reinterpret_cast<q8_half8*>(out + (u + k) * a.out_row_stride + 8 * o) = y[k];
}

// [tile][pair], then entries in the order of lane_entry
__global__ void q8_rope_table_kernel(double base, int n_tiles, double2* table)
{
    const int idx = blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= (n_tiles + kTileTokens) * kQ8Pairs) return;
    const int i = idx % kQ8Pairs, row = idx / kQ8Pairs;
    const double pos = row < n_tiles ? 64.0 * row : (double)(row - n_tiles);
    const double ang = pos * pow(base, -2.0 * (double)i / kQ8Head);
    table[row < n_tiles ? idx : n_tiles * kQ8Pairs + lane_entry(row - n_tiles, i)] = make_double2(cos(ang), sin(ang));
}

// Tiles of a sequence that its last m tokens can lie in.
int tile_slots(int m, int t, bool ragged)
{
    if (!ragged) return (t - 1) / kTileTokens - (t - m) / kTileTokens + 1;
    return (int)std::min<int64_t>(((int64_t)m + kTileTokens - 2) / kTileTokens + 1, (t + kTileTokens - 1) / kTileTokens);
}

}  // namespace

size_t q8_rope_table_bytes(int positions) { return sizeof(double2) * kQ8Pairs * ((size_t)positions / kTileTokens + kTileTokens); }

cq_status launch_q8_rope_table(double base, int positions, void* table, hipStream_t stream)
{
    const int n_tiles = positions / kTileTokens;
    const int64_t total = ((int64_t)n_tiles + kTileTokens) * kQ8Pairs;
    if (total > 0x7fffff00LL) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL(q8_rope_table_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, stream, base, n_tiles, static_cast<double2*>(table));
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_append_q8(const Q8AppendArgs& args, int kind, hipStream_t stream)
{
    Q8AppendArgs a = args;
    a.slots = tile_slots(a.m, a.t, a.seq_lens != nullptr);
    // Heads in a row share their angles (64 KB of the table to a tile), as far as 512 workgroups remain: of 256, 512 and 1024, 6 x 500
    // tokens of 32 heads take 62, 62 and 67 us, 4 x 8192 of 8 heads, 194, 194 and 201 (with the rows read back).
    const int64_t tiles = (int64_t)a.batch * a.slots;
    a.heads = 1;
    while (a.heads < 8 && a.n_kv_heads % (2 * a.heads) == 0 && tiles * a.n_kv_heads / (2 * a.heads) >= 512) a.heads *= 2;
    const bool token = a.m == 1;
    const int64_t kv = token ? ((int64_t)a.batch * a.n_kv_heads + kThreads / 64 - 1) / (kThreads / 64) : tiles * (a.n_kv_heads / a.heads);
    int64_t q_wgs = 0;
    if (a.q) {
        const int64_t rows = (int64_t)a.batch * a.m;
        a.q_heads = 1;
        while (a.q_heads < 8 && a.n_q_heads % (2 * a.q_heads) == 0 && rows * a.n_q_heads / (2 * a.q_heads) >= 32768) a.q_heads *= 2;
        q_wgs = (rows * (a.n_q_heads / a.q_heads) + kThreads / 8 - 1) / (kThreads / 8);
    }
    if (2 * kv + q_wgs > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    a.kv_wgs = (unsigned)kv;
    const dim3 grid((unsigned)((token ? 1 : 2) * kv + q_wgs));
    const bool integers = kind == CQ_Q8_INT8;
    if (token && integers) hipLaunchKernelGGL(append_token_q8_kernel<CQ_Q8_INT8>, grid, dim3(kThreads), 0, stream, a);
    else if (token) hipLaunchKernelGGL(append_token_q8_kernel<CQ_Q8_E4M3>, grid, dim3(kThreads), 0, stream, a);
    else if (integers) hipLaunchKernelGGL(append_q8_kernel<CQ_Q8_INT8>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(append_q8_kernel<CQ_Q8_E4M3>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_dequantize_q8(const Q8DequantArgs& args, int kind, hipStream_t stream)
{
    Q8DequantArgs a = args;
    a.slots = tile_slots(a.m, a.t, a.seq_lens != nullptr);
    const int64_t kv = (int64_t)a.batch * a.slots * a.n_kv_heads;
    const int64_t grid = kv * ((a.out[0] != nullptr) + (a.out[1] != nullptr));
    if (grid > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    a.kv_wgs = (unsigned)kv;
    if (kind == CQ_Q8_INT8) hipLaunchKernelGGL(dequantize_q8_kernel<CQ_Q8_INT8>, dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(dequantize_q8_kernel<CQ_Q8_E4M3>, dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace cq
