// The 8-bit block cache, its codes: cq_append_q8 (rotation, block scales, codes, older tokens under a scale that grew) and
// cq_dequantize_q8, for gfx950.
//
//   key pair (i, i + 64) at position p:  k'_i = k_i cos(p th_i) - k_{i+64} sin(p th_i),  k'_{i+64} = k_{i+64} cos + k_i sin
//   block of 64 tokens and a head:  s = max(s before, if the block holds older tokens; need(largest |x| of the new ones))
//   need: integers fp32(largest / 127); e4m3 the smallest power of two >= largest / 448
//   code = nearest(x / s), ties to even; codes of older tokens, where s grew: nearest(c s_before / s)
//
// Which side of a border a number lies on is decided in 64 bits (angles are products of two table entries in 64 bits): codes are
// those of exact arithmetic but for borders met to 2^-50, whatever the position, and do not depend on how a call is cut.
// fp64 costs what fp32 does here (no packed fp32), and the kernel is bound by memory.
// e4m3 scales are powers of two so that a growing scale moves codes without rounding them again (but into
// subnormals); integers use the whole range instead: a power of two would cost up to a bit of seven.
#include <algorithm>

#include "cq_q8.hpp"

namespace cq {
namespace {

constexpr int kThreads = 256;

// x rounded to fp32 so that rounding once more, to fewer bits, is right: towards zero, and the last bit set if something was cut off.
__device__ __forceinline__ float to_odd(double x)
{
    float f = (float)x;
    const double back = (double)f;
    if (back != x) {
        unsigned b = __builtin_bit_cast(unsigned, f);
        if (fabs(back) > fabs(x)) b -= 1;
        f = __builtin_bit_cast(float, b | 1u);
    }
    return f;
}

// The code byte of a number in units of its block's scale.
template <int KIND>
__device__ __forceinline__ unsigned code_of(double x)
{
    if constexpr (KIND == CQ_Q8_INT8) {
        const int c = (int)fmin(fmax(rint(x), -127.0), 127.0);
        return (unsigned)(c + 128);
    } else {
        const float f = fminf(fmaxf(to_odd(x), -448.f), 448.f) + 0.f;         // (zero, of either sign, has one code)
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f, f, 0, false) & 0xffu;
    }
}
// ... of code byte w's number under a scale that grew by 1 / ratio.
template <int KIND>
__device__ __forceinline__ unsigned regrown(unsigned w, double ratio)
{
    if constexpr (KIND == CQ_Q8_INT8) return code_of<KIND>((double)((int)w - 128) * ratio);
    else return code_of<KIND>((double)__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio);
}
template <int KIND>
__device__ __forceinline__ unsigned regrown4(unsigned w, double ratio)
{
    unsigned r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= regrown<KIND>((w >> (8 * i)) & 0xffu, ratio) << (8 * i);
    return r;
}

template <int KIND>
__device__ __forceinline__ float need_of(double largest)
{
    if constexpr (KIND == CQ_Q8_INT8) return (float)(largest / 127.0);
    const unsigned long long bits = __builtin_bit_cast(unsigned long long, largest / 448.0);
    return (float)__builtin_bit_cast(double, (bits + 0xfffffffffffffULL) & (0x7ffULL << 52));
}

// x / s of an s whose reciprocal is `inv`, as IEEE division gives it (but for quotients no code depends on).
__device__ __forceinline__ double quotient(double x, double s, double inv)
{
    const double y = x * inv;
    return fma(fma(-y, s, x), inv, y);
}

__device__ __forceinline__ double wave_max_f64(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmax(x, __shfl_xor(x, d));
    return x;
}

__device__ __forceinline__ void halves_of(q8_u4 w, double* x)
{
    const q8_half8 h = __builtin_bit_cast(q8_half8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (double)(float)h[i];
}

// cos, sin of (64 tile + u) theta_i
__device__ __forceinline__ double2 angle_of(double2 tile, double2 lane)
{
    return make_double2(fma(tile.x, lane.x, -tile.y * lane.y), fma(tile.y, lane.x, tile.x * lane.y));
}

// The block's scale from the largest new magnitude of every thread; `grown`: the older tokens' codes change by `ratio`.
struct BlockScale {
    double s, inv, ratio;
    bool grown;
};
template <int KIND>
__device__ __forceinline__ BlockScale block_scale(double mine, bool has_old, float* at, double* lds, int tid)
{
    const double w = wave_max_f64(mine);
    __syncthreads();                                        // (the reads of the head before are done)
    if ((tid & 63) == 0) lds[tid >> 6] = w;
    if (tid == 0) lds[4] = has_old ? (double)*at : 0.0;     // (the thread that writes it is the only one that reads it)
    __syncthreads();
    const double largest = fmax(fmax(lds[0], lds[1]), fmax(lds[2], lds[3]));
    const float before = (float)lds[4];
    const float s = fmaxf(before, need_of<KIND>(largest));
    if (tid == 0) *at = s;
    BlockScale b;
    b.s = s;
    b.inv = s > 0.f ? 1.0 / (double)s : 0.0;
    b.grown = has_old && s > before;
    b.ratio = b.grown ? (double)before / (double)s : 1.0;
    return b;
}

// A workgroup: one tile of one sequence, `heads` heads in a row, keys or values; behind those, queries.
template <int KIND>
__global__ __launch_bounds__(kThreads) void append_q8_kernel(Q8AppendArgs a)
{
    __shared__ double lds[kThreads / 64 + 1];               // largest magnitudes of the wavefronts, the scale before
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned idx = blockIdx.x;
    if (idx >= 2 * a.kv_wgs) {
        // ---- queries: a thread rotates pairs 8 o .. 8 o + 7 of `q_heads` heads of a row
        idx -= 2 * a.kv_wgs;
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
            const double2 r = angle_of(a.tile_tab[(size_t)(p >> 6) * kQ8Pairs + 8 * o + i], a.lane_tab[(p & 63) * kQ8Pairs + 8 * o + i]);
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
        return;
    }
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
            for (int i = 0; i < 16; ++i) ang[i] = angle_of(a.tile_tab[(size_t)tile * kQ8Pairs + 16 * o + i], a.lane_tab[u * kQ8Pairs + 16 * o + i]);
        }
        for (int h = group * a.heads; h < (group + 1) * a.heads; ++h) {
            const size_t at = a.cache.map.tile_index(n, h, tile);
            double x[32], mine = 0.0;
            if (fresh) {
                const uint16_t* src = x0 + u * a.x_row_stride + h * kQ8Head + 16 * o;
                halves_of(*reinterpret_cast<const q8_u4*>(src), x);
                halves_of(*reinterpret_cast<const q8_u4*>(src + 8), x + 8);
                halves_of(*reinterpret_cast<const q8_u4*>(src + 64), x + 16);
                halves_of(*reinterpret_cast<const q8_u4*>(src + 72), x + 24);
                if (a.tile_tab) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const double y = fma(x[i], ang[i].x, -x[16 + i] * ang[i].y), z = fma(x[16 + i], ang[i].x, x[i] * ang[i].y);
                        x[i] = y;
                        x[16 + i] = z;
                    }
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) mine = fmax(mine, fabs(x[i]));
            }
            const BlockScale b = block_scale<KIND>(mine, lo > 0, a.cache.scales[0] + at, lds, tid);
            uint8_t* dst = a.cache.codes[0] + at * kQ8TileBytes + u * kQ8Head + 16 * o;
            if (fresh) {
                unsigned w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[i] |= code_of<KIND>(quotient(x[4 * i + k], b.s, b.inv)) << (8 * k);
                }
                *reinterpret_cast<q8_u4*>(dst) = q8_u4{w[0], w[1], w[2], w[3]};
                *reinterpret_cast<q8_u4*>(dst + 64) = q8_u4{w[4], w[5], w[6], w[7]};
            } else if (u < lo && b.grown) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    q8_u4 w = *reinterpret_cast<const q8_u4*>(dst + 64 * k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = regrown4<KIND>(w[i], b.ratio);
                    *reinterpret_cast<q8_u4*>(dst + 64 * k) = w;
                }
            }
        }
        return;
    }
    // ---- values: thread (a4, o) holds tokens 4 a4 .. 4 a4 + 3 of channels 8 o .. 8 o + 7, a word of the cache per channel
    const int u = 4 * (lane & 15), o = (lane >> 4) + 4 * wave;
    const bool some_new = u + 4 > lo && u < hi, all_new = u >= lo && u + 4 <= hi;
    for (int h = group * a.heads; h < (group + 1) * a.heads; ++h) {
        const size_t at = a.cache.map.tile_index(n, h, tile);
        double mine = 0.0;
        q8_half8 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (u + k < lo || u + k >= hi) continue;
            x[k] = *reinterpret_cast<const q8_half8*>(x0 + (u + k) * a.x_row_stride + h * kQ8Head + 8 * o);
#pragma unroll
            for (int i = 0; i < 8; ++i) mine = fmax(mine, fabs((double)(float)x[k][i]));
        }
        const BlockScale b = block_scale<KIND>(mine, lo > 0, a.cache.scales[1] + at, lds, tid);
        if (!some_new && !(b.grown && u < lo)) continue;
        uint8_t* dst = a.cache.codes[1] + at * kQ8TileBytes + (size_t)(8 * o) * kTileTokens + u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            unsigned w = 0;
            if (!all_new) {
                const unsigned old = *reinterpret_cast<const unsigned*>(dst + i * kTileTokens);
                const unsigned now = b.grown ? regrown4<KIND>(old, b.ratio) : old;
#pragma unroll
                for (int k = 0; k < 4; ++k) w |= (u + k < lo ? now : old) & (0xffu << (8 * k));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (u + k >= lo && u + k < hi) w = (w & ~(0xffu << (8 * k))) | code_of<KIND>(quotient((double)(float)x[k][i], b.s, b.inv)) << (8 * k);
            *reinterpret_cast<unsigned*>(dst + i * kTileTokens) = w;
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

// [tile][pair], then [u][pair]
__global__ void q8_rope_table_kernel(double base, int n_tiles, double2* table)
{
    const int idx = blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= (n_tiles + kTileTokens) * kQ8Pairs) return;
    const int i = idx % kQ8Pairs, row = idx / kQ8Pairs;
    const double pos = row < n_tiles ? 64.0 * row : (double)(row - n_tiles);
    const double ang = pos * pow(base, -2.0 * (double)i / kQ8Head);
    table[idx] = make_double2(cos(ang), sin(ang));
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
    const int64_t tiles = (int64_t)a.batch * a.slots;
    // heads in a row share their angles, as far as enough workgroups remain
    a.heads = 1;
    while (a.heads < 8 && a.n_kv_heads % (2 * a.heads) == 0 && tiles * a.n_kv_heads / (2 * a.heads) >= 1024) a.heads *= 2;
    const int64_t kv = tiles * (a.n_kv_heads / a.heads);
    int64_t q_wgs = 0;
    if (a.q) {
        const int64_t rows = (int64_t)a.batch * a.m;
        a.q_heads = 1;
        while (a.q_heads < 8 && a.n_q_heads % (2 * a.q_heads) == 0 && rows * a.n_q_heads / (2 * a.q_heads) >= 32768) a.q_heads *= 2;
        q_wgs = (rows * (a.n_q_heads / a.q_heads) + kThreads / 8 - 1) / (kThreads / 8);
    }
    if (2 * kv + q_wgs > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    a.kv_wgs = (unsigned)kv;
    const dim3 grid((unsigned)(2 * kv + q_wgs));
    if (kind == CQ_Q8_INT8) hipLaunchKernelGGL(append_q8_kernel<CQ_Q8_INT8>, grid, dim3(kThreads), 0, stream, a);
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
