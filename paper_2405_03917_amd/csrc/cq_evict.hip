// Eviction from a coded cache, for gfx950: which tokens of every (sequence, KV head) stay, and the caches and
// accumulators moved together.
//
// cq_select_tokens.  A stream's `keep` tokens are its first n_sink, its last n_recent and, between them, the heaviest,
// ties to the lowest index.  The weight of the last one that stays is found by its digits (a radix selection on the
// weights' order-preserving integers); what is above it stays, and of what equals it the first few.  Ranks come from
// counts in index order, so the list is ascending and a function of the weights alone.
//
// cq_compact_cache.  The token of rank r moves to position r.  A record's bytes are rotated by its token's position in
// the tile (slot s of token u holds group (s + u) mod Gh), so a move from u to u' rotates the record by u' - u bytes
// (10-bit codes: the word of high bits by twice as many bits).  A lane moves a token's record.
// Bound by the chain of requests and barriers of each launch where little moves, else by the bytes moved.  32 streams of 131072 tokens to
// 2047: counts 7.3 us, lists 9.4, positions 12.4, the move 5.4 (17 MB of weights, 4 MB moved).  512 streams of 4160 to 4096 in place:
// selection 12 to 14; the move of CQ-4c8b 10 to 12 where a sixth of the tokens change their place, 60 where nearly all do (281 MB read and
// written, 4.7 TB/s; a copy reaches 5.18), of CQ-8c8b then 34, of CQ-2c8b 112.
#include "cq_decode_common.hpp"

namespace cq {
namespace {

// ---------------------------------------------------------------------------------- selection
constexpr int kSelectThreads = 512;                     // of a run of a long stream
constexpr int kDigitBits = 11;                          // three digits: 11, 11, 10 bits
constexpr int kBins = 1 << kDigitBits;
constexpr int kPerThread = 16;                          // tokens of a run per thread, in registers
constexpr int kPart = kSelectThreads * kPerThread;
constexpr int kCopies = 4;                            // of the first digits' counts in LDS, by lane
constexpr int kListRoom = 8192;                         // listed keys of a stream that are held in LDS (32 KB)
static_assert(kPart == kSelectRun, "as the workspace is sized");

// order-preserving: larger weights have larger keys, both zeros the same; what is no number ranks below every number
__device__ __forceinline__ unsigned weight_key(float w)
{
    const unsigned u = __float_as_uint(w + 0.f);
    if (w != w) return 0;
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// exclusive prefix sum over the workgroup's NT threads; *total: the sum
template <int NT>
__device__ __forceinline__ unsigned block_prefix(unsigned v, unsigned* sums, int tid, unsigned* total)
{
    constexpr int kSelectWaves = NT / 64;
    const int lane = tid & 63, wave = tid >> 6;
    unsigned x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned y = __shfl_up(x, d);
        x += lane >= d ? y : 0u;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        const unsigned s = sums[w];
        before += w < wave ? s : 0u;
        all += s;
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

// The middle of a stream: what is left to choose from once its first and last tokens are kept.
struct Middle {
    int t_n, len;                       // tokens of the sequence, between the kept ends (0: nothing to choose)
    unsigned need;                      // of them, to be chosen
    const float* w;
    int32_t* kept;
};
__device__ __forceinline__ Middle middle_of(const SelectArgs& a, int stream)
{
    const int n = stream / a.n_kv_heads;
    Middle m;
    m.t_n = a.t;
    if (a.seq_lens) m.t_n = min(max(a.seq_lens[n], 0), a.t);
    m.kept = a.kept + (size_t)stream * a.keep;
    m.w = a.weights + (size_t)stream * a.weights_stride + a.n_sink;
    m.need = (unsigned)(a.keep - a.n_sink - a.n_recent);
    m.len = m.t_n > a.keep && m.need > 0 ? m.t_n - a.n_sink - a.n_recent : 0;
    return m;
}
// What needs no choice: the new length, the ends, short sequences.  (Workgroup `part` of `parts`.)
template <int NT>
__device__ __forceinline__ void keep_ends(const SelectArgs& a, const Middle& m, int stream, int part, int parts, int tid)
{
    const int first = part * NT + tid, step = parts * NT;
    if (stream % a.n_kv_heads == 0 && first == 0) a.kept_lens[stream / a.n_kv_heads] = min(m.t_n, a.keep);
    if (m.t_n <= a.keep) {
        for (int r = first; r < a.keep; r += step) m.kept[r] = r < m.t_n ? r : -1;
        return;
    }
    for (int r = first; r < a.n_sink; r += step) m.kept[r] = r;
    for (int r = first; r < a.n_recent; r += step) m.kept[a.keep - a.n_recent + r] = m.t_n - a.n_recent + r;
}

// Keys k of tokens first + NT k + thread, of a run of up to 16 NT tokens, in registers.
template <int NT>
struct Keys {
    unsigned key[kPerThread];
    int first, count;                   // tokens of the run
    __device__ __forceinline__ void load(const Middle& m, int part, int tid)
    {
        first = part * (NT * kPerThread);
        count = min(NT * kPerThread, m.len - first);
        float w[kPerThread];
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) w[k] = has(k, tid) ? m.w[first + k * NT + tid] : 0.f;
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) key[k] = weight_key(w[k]);
    }
    __device__ __forceinline__ bool has(int k, int tid) const { return k * NT + tid < count; }
    __device__ __forceinline__ bool any(int k) const { return k * NT < count; }      // (uniform)
};

// The bin, from the top, in which `need` is reached, and what is still needed of it: thread i holds bins hi, hi - 1, ... (N of
// them), hi = bins - 1 - N i.
template <int NT, int N>
__device__ __forceinline__ void find_among(const unsigned (&c)[N], int hi, unsigned& need, unsigned& bin, unsigned* sums, unsigned* found, int tid)
{
    unsigned sum = 0, total;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += c[i];
    unsigned above = block_prefix<NT>(sum, sums, tid, &total);
    if (above < need && above + sum >= need) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (above < need && above + c[i] >= need) {
                found[0] = (unsigned)(hi - i);
                found[1] = need - above;
            }
            above += c[i];
        }
    }
    __syncthreads();
    bin = found[0];
    need = found[1];
}
template <int NT>
__device__ __forceinline__ void find_bin(const unsigned* hist, int bins, unsigned& need, unsigned& bin, unsigned* sums, unsigned* found, int tid)
{
    constexpr int N = kBins / NT;
    const int hi = bins - 1 - N * tid;
    unsigned c[N];
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = hi - i >= 0 ? hist[hi - i] : 0u;
    find_among<NT, N>(c, hi, need, bin, sums, found, tid);
}
template <int NT>
__device__ __forceinline__ void clear(unsigned* hist, int tid)
{
    for (int i = tid; i < kBins / 4; i += NT) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
}
// The first digits of a run counted in LDS, in kCopies counts of each: sign, exponent and two bits of weights that are alike
// name a few digits, and additions to one word wait for each other.  Zeros, of which there may be many (tokens that never drew
// weight), are counted a wavefront at a time.
template <int NT>
__device__ __forceinline__ void count_first_digits(const Keys<NT>& keys, unsigned* hist, int tid)
{
    constexpr unsigned kZero = 0x80000000u;
    unsigned zeros = 0;
    for (int i = tid; i < kBins * kCopies / 4; i += NT) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (!keys.any(k)) break;
        const bool in = keys.has(k, tid), zero = in && keys.key[k] == kZero;
        zeros += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(zero));
        if (in && !zero) atomicAdd(&hist[(keys.key[k] >> 21) * kCopies + (tid & (kCopies - 1))], 1u);
    }
    if ((tid & 63) == 0 && zeros) atomicAdd(&hist[(kZero >> 21) * kCopies], zeros);
    __syncthreads();
}

__device__ __forceinline__ unsigned first_digits(const unsigned* hist, int digit)
{
    static_assert(kCopies == 4, "read as 16 bytes");
    const uint4 x = reinterpret_cast<const uint4*>(hist)[digit];
    return x.x + x.y + x.z + x.w;
}

// `from` and the lanes in front of this one that are in the mask
__device__ __forceinline__ unsigned lanes_below(unsigned long long mask, unsigned from)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, from));
}

// Positions of the run's tokens whose key is above `key`, or equals it where fewer than `need` equals lie in front, behind
// gt_base, eq_base such tokens of earlier runs.
template <int NT>
__device__ __forceinline__ void write_kept(const SelectArgs& a, const Middle& m, const Keys<NT>& keys, unsigned key, unsigned need, unsigned gt_base,
                                           unsigned eq_base, unsigned* counts, int tid)
{
    constexpr int kWaves = NT / 64, N = kPerThread * kWaves / 64;      // counts per lane of a wavefront
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const bool in = keys.has(k, tid);
        const unsigned gt = (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in && keys.key[k] > key));
        const unsigned eq = (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in && keys.key[k] == key));
        if (lane == 0) counts[k * kWaves + wave] = gt | eq << 16;
    }
    __syncthreads();
    if (wave == 0) {                    // exclusive prefix sums; (equals of a run reach 2^13: 16 bits hold both)
        unsigned c[N], sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            c[i] = sum;
            sum += counts[N * lane + i];
        }
        unsigned x = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const unsigned y = __shfl_up(x, d);
            x += lane >= d ? y : 0u;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) counts[N * lane + i] = c[i] + x - sum;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (!keys.any(k)) break;
        const bool in = keys.has(k, tid), gt = in && keys.key[k] > key, eq = in && keys.key[k] == key;
        const unsigned long long gts = __builtin_amdgcn_ballot_w64(gt), eqs = __builtin_amdgcn_ballot_w64(eq);
        const unsigned at = counts[k * kWaves + wave];
        const unsigned g = lanes_below(gts, gt_base + (at & 0xffffu)), e = lanes_below(eqs, eq_base + (at >> 16));
        if (gt || (eq && e < need)) m.kept[a.n_sink + g + min(e, need)] = a.n_sink + keys.first + k * NT + tid;
    }
}

// Streams of one run: a workgroup each, the keys read once.
template <int NT>
__global__ __launch_bounds__(NT) void select_short_kernel(SelectArgs a)
{
    __shared__ __align__(16) unsigned hist[kBins * kCopies];
    __shared__ unsigned sums[NT / 64];
    __shared__ unsigned found[2];
    const int tid = threadIdx.x, stream = blockIdx.x;
    const Middle m = middle_of(a, stream);
    Keys<NT> keys;
    keys.load(m, 0, tid);
    keep_ends<NT>(a, m, stream, 0, 1, tid);
    if (m.len == 0) return;
    unsigned need = m.need, bin;
    count_first_digits(keys, hist, tid);
    {
        constexpr int N = kBins / NT;
        unsigned c[N];
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = first_digits(hist, kBins - 1 - N * tid - i);
        find_among<NT, N>(c, kBins - 1 - N * tid, need, bin, sums, found, tid);
    }
    unsigned prefix = bin << 21, mask = (kBins - 1u) << 21;
#pragma unroll 1
    for (int shift = 10; shift >= 0; shift -= 10) {
        const int bins = shift == 0 ? kBins / 2 : kBins;
        clear<NT>(hist, tid);
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            if (!keys.any(k)) break;
            if (keys.has(k, tid) && (keys.key[k] & mask) == prefix) atomicAdd(&hist[(keys.key[k] >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        find_bin<NT>(hist, bins, need, bin, sums, found, tid);
        prefix |= bin << shift;
        mask |= (unsigned)(bins - 1) << shift;
    }
    __syncthreads();
    write_kept<NT>(a, m, keys, prefix, need, 0, 0, hist, tid);
}

// Longer streams: a workgroup per run.  Each run's first digits are counted; the digit in which the key lies follows from the
// counts of all, and every run lists its keys that have it, in any order: what follows is a function of the set; the key is found
// among the stream's listed ones, and with it what each run has in front of its own tokens, which it then writes.  Digit and key
// are found by every run again (three launches), or, where a stream has many, by a workgroup per stream (five).
// (The listed keys are those of one of 2048 digits, usually less than a hundredth of the stream, and are held in LDS.  If there is
// only one among them, such as zero for tokens that never drew weight, there is nothing to find.)
__global__ __launch_bounds__(kSelectThreads) void select_count_kernel(SelectArgs a)
{
    __shared__ __align__(16) unsigned hist[kBins * kCopies];
    const int tid = threadIdx.x, part = blockIdx.x % a.parts, stream = blockIdx.x / a.parts;
    const Middle m = middle_of(a, stream);
    Keys<kSelectThreads> keys;
    keys.load(m, part, tid);
    keep_ends<kSelectThreads>(a, m, stream, part, a.parts, tid);
    if (m.len == 0) return;
    count_first_digits(keys, hist, tid);
    static_assert(kBins == 2 * kSelectCounts && kSelectRun < 65536, "two counts a word");
    unsigned* out = a.counts + (size_t)blockIdx.x * kSelectCounts;
    for (int i = tid; i < kSelectCounts; i += kSelectThreads) out[i] = first_digits(hist, 2 * i) | first_digits(hist, 2 * i + 1) << 16;
}

// A thread's four bins of a stream from the top (hi, hi - 1, ...), added over its runs.
__device__ __forceinline__ void add_counts(const SelectArgs& a, int stream, int hi, unsigned (&c)[4])
{
    static_assert(kBins == 4 * kSelectThreads, "four bins a thread");
    const unsigned* all = a.counts + (size_t)stream * a.parts * kSelectCounts + (hi - 3) / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = 0;
#pragma unroll 1
    for (int p0 = 0; p0 < a.parts; p0 += 8) {               // (eight runs' counts requested at once)
        uint2 x[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) x[p] = *reinterpret_cast<const uint2*>(all + (size_t)min(p0 + p, a.parts - 1) * kSelectCounts);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const unsigned down[4] = {x[p].y >> 16, x[p].y & 0xffffu, x[p].x >> 16, x[p].x & 0xffffu};
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] += p0 + p < a.parts ? down[i] : 0u;
        }
    }
}

// Streams of many runs: the digit, by a workgroup per stream.
__global__ __launch_bounds__(kSelectThreads) void select_digit_kernel(SelectArgs a)
{
    __shared__ unsigned sums[kSelectThreads / 64];
    __shared__ unsigned found[2];
    const int tid = threadIdx.x, stream = blockIdx.x;
    const Middle m = middle_of(a, stream);
    if (m.len == 0) return;
    unsigned c[4], need = m.need, bin;
    add_counts(a, stream, kBins - 1 - 4 * tid, c);
    find_among<kSelectThreads, 4>(c, kBins - 1 - 4 * tid, need, bin, sums, found, tid);
    if (tid == 0) a.found[stream] = make_uint2(bin, need);
}

__global__ __launch_bounds__(kSelectThreads) void select_list_kernel(SelectArgs a)
{
    __shared__ unsigned sums[kSelectThreads / 64];
    __shared__ unsigned found[2];
    __shared__ unsigned listed, lowest, highest, above;
    const int tid = threadIdx.x, part = blockIdx.x % a.parts, stream = blockIdx.x / a.parts;
    const int lane = tid & 63;
    const Middle m = middle_of(a, stream);
    if (m.len == 0) return;
    Keys<kSelectThreads> keys;
    keys.load(m, part, tid);
    unsigned need = m.need, bin;
    if (tid == 0) {
        listed = highest = above = 0;
        lowest = 0xffffffffu;
    }
    if (a.many) {                                           // (uniform)
        bin = a.found[stream].x;
        __syncthreads();
    } else {
        unsigned c[4];
        add_counts(a, stream, kBins - 1 - 4 * tid, c);
        find_among<kSelectThreads, 4>(c, kBins - 1 - 4 * tid, need, bin, sums, found, tid);
        if (part == 0 && tid == 0) a.found[stream] = make_uint2(bin, need);
    }
    unsigned* const list = a.lists + (size_t)blockIdx.x * kPart;
    unsigned larger = 0, some = 0;                          // (of a wavefront: one of its listed keys)
    bool any = false, mixed = false;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (!keys.any(k)) break;
        const bool has = keys.has(k, tid), in = has && keys.key[k] >> 21 == bin;
        larger += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(has && keys.key[k] >> 21 > bin));
        const unsigned long long b = __builtin_amdgcn_ballot_w64(in);
        if (b == 0) continue;
        unsigned base = 0;
        if (lane == 0) base = atomicAdd(&listed, (unsigned)__builtin_popcountll(b));
        base = (unsigned)__builtin_amdgcn_readfirstlane((int)base);
        if (in) list[lanes_below(b, base)] = keys.key[k];
        if (!any) some = (unsigned)__builtin_amdgcn_readlane((int)keys.key[k], __builtin_ctzll(b));
        any = true;
        mixed = mixed || __builtin_amdgcn_ballot_w64(in && keys.key[k] != some) != 0;
    }
    if (lane == 0) {
        atomicAdd(&above, larger);
        if (any) {                                          // (of different ones any bounds will do that are not equal)
            atomicMin(&lowest, mixed ? 0u : some);
            atomicMax(&highest, mixed ? 0xffffffffu : some);
        }
    }
    __syncthreads();
    if (tid == 0) a.runs[blockIdx.x] = make_uint4(listed, above, lowest, highest);
}

// A stream's key among the listed ones, by a workgroup.
struct KeySearch {
    static constexpr int kStarts = 1024, kWaves = kSelectThreads / 64;
    struct Lds {
        unsigned hist[kBins];
        unsigned held[kListRoom];
        unsigned starts[kStarts + 1];                       // where each run's keys begin among the stream's
        unsigned sums[kWaves], found[2];
        unsigned listed, lowest, highest;
    };
    Lds& s;
    const int parts;
    const uint4* const runs;                                // (listed, above, lowest, highest)
    const unsigned* const lists;
    bool in_lds, one;                                       // the listed keys are held; are all the same
    unsigned key, need;

    __device__ __forceinline__ KeySearch(Lds& lds, const SelectArgs& a, int stream)
        : s(lds), parts(a.parts), runs(a.runs + (size_t)stream * a.parts), lists(a.lists + (size_t)stream * a.parts * kPart)
    {
    }
    __device__ __forceinline__ unsigned count_of(int p) const { return parts <= kStarts ? s.starts[p + 1] - s.starts[p] : runs[p].x; }
    // the keys of run p, by a wavefront: from memory, eight requests at a time, or held
    template <class F>
    __device__ __forceinline__ void of_run(int p, bool from_lds, F&& f) const
    {
        const int lane = threadIdx.x & 63;
        const unsigned n = count_of(p);
        if (from_lds) {
            for (unsigned i = 0; i < n; i += 64) f(i + lane < n, i + lane, s.held[s.starts[p] + min(i + lane, n - 1)]);
            return;
        }
        const unsigned* const l = lists + (size_t)p * kPart;
#pragma unroll 1
        for (unsigned i0 = 0; i0 < n; i0 += 8 * 64) {
            unsigned x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = i0 + k * 64 < n ? l[min(i0 + k * 64 + lane, n - 1)] : 0u;
#pragma unroll
            for (int k = 0; k < 8; ++k) f(i0 + k * 64 + lane < n, i0 + k * 64 + lane, x[k]);
        }
    }
    __device__ __forceinline__ void find(uint2 digit)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        if (wave == 0) {
            unsigned base = 0, low = 0xffffffffu, high = 0;
            for (int p0 = 0; p0 < parts; p0 += 64) {
                const uint4 r = p0 + lane < parts ? runs[p0 + lane] : make_uint4(0, 0, 0xffffffffu, 0);
                low = min(low, r.z);
                high = max(high, r.w);
                unsigned x = r.x;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const unsigned y = __shfl_up(x, d);
                    x += lane >= d ? y : 0u;
                }
                if (parts <= kStarts && p0 + lane < parts) s.starts[p0 + lane + 1] = base + x;
                base += (unsigned)__builtin_amdgcn_readlane((int)x, 63);
            }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                low = min(low, (unsigned)__shfl_xor((int)low, d));
                high = max(high, (unsigned)__shfl_xor((int)high, d));
            }
            if (lane == 0) {
                s.starts[0] = 0;
                s.listed = base;
                s.lowest = low;
                s.highest = high;
            }
        }
        __syncthreads();
        in_lds = parts <= kStarts && s.listed <= kListRoom;
        one = s.lowest == s.highest;                        // (zero mostly: nothing to find)
        key = s.lowest;
        need = digit.y;
        if (one) return;
        if (in_lds && parts <= 64) {
            for (unsigned i = tid; i < s.listed; i += kSelectThreads) {
                int p = 0;
#pragma unroll
                for (int step = 32; step > 0; step >>= 1)
                    if (p + step < parts && s.starts[p + step] <= i) p += step;
                s.held[i] = lists[(size_t)p * kPart + (i - s.starts[p])];
            }
        } else if (in_lds) {
            for (int p = wave; p < parts; p += kWaves)
                of_run(p, false, [&](bool is, unsigned i, unsigned x) {
                    if (is) s.held[s.starts[p] + i] = x;
                });
        }
        unsigned prefix = digit.x << 21, mask = (kBins - 1u) << 21, bin;
#pragma unroll 1
        for (int shift = 10; shift >= 0; shift -= 10) {
            const int bins = shift == 0 ? kBins / 2 : kBins;
            clear<kSelectThreads>(s.hist, tid);
            auto count = [&](bool is, unsigned, unsigned x) {
                if (is && (x & mask) == prefix) atomicAdd(&s.hist[(x >> shift) & (bins - 1)], 1u);
            };
            if (in_lds) {
                for (unsigned i = tid; i < s.listed; i += kSelectThreads) count(true, i, s.held[i]);
            } else {
                for (int p = wave; p < parts; p += kWaves) of_run(p, false, count);
            }
            __syncthreads();
            find_bin<kSelectThreads>(s.hist, bins, need, bin, s.sums, s.found, tid);
            prefix |= bin << shift;
            mask |= (unsigned)(bins - 1) << shift;
        }
        key = prefix;
    }
    // of a run's tokens, those above the key and those that equal it, by a wavefront
    __device__ __forceinline__ uint2 kept_of(int p) const
    {
        uint2 c = make_uint2(runs[p].y, one ? count_of(p) : 0u);
        if (!one)
            of_run(p, in_lds, [&](bool is, unsigned, unsigned x) {
                c.x += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(is && x > key));
                c.y += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(is && x == key));
            });
        return c;
    }
};

// Streams of many runs: the key, and what every run's tokens have in front of them, by a workgroup per stream.
__global__ __launch_bounds__(kSelectThreads) void select_key_kernel(SelectArgs a)
{
    __shared__ __align__(16) KeySearch::Lds lds;
    const int stream = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Middle m = middle_of(a, stream);
    if (m.len == 0) return;
    KeySearch search(lds, a, stream);
    search.find(a.found[stream]);
    uint4* const runs = a.runs + (size_t)stream * a.parts;
    for (int p = wave; p < a.parts; p += KeySearch::kWaves) {
        const uint2 c = search.kept_of(p);
        if (lane == 0) runs[p] = make_uint4(c.x, c.y, 0, 0);
    }
    __syncthreads();
    if (wave != 0) return;
    unsigned gt_base = 0, eq_base = 0;
    for (int p0 = 0; p0 < a.parts; p0 += 64) {
        const bool is = p0 + lane < a.parts;
        const uint4 r = is ? runs[p0 + lane] : make_uint4(0, 0, 0, 0);
        unsigned x = r.x, y = r.y;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const unsigned gx = __shfl_up(x, d), ey = __shfl_up(y, d);
            x += lane >= d ? gx : 0u;
            y += lane >= d ? ey : 0u;
        }
        if (is) runs[p0 + lane] = make_uint4(gt_base + x - r.x, eq_base + y - r.y, search.key, search.need);
        gt_base += (unsigned)__builtin_amdgcn_readlane((int)x, 63);
        eq_base += (unsigned)__builtin_amdgcn_readlane((int)y, 63);
    }
}

static_assert(kSelectManyRuns <= 64 && kSelectManyRuns <= kSelectThreads, "a thread per run in front");

// The positions: MANY: behind select_key_kernel; else every run finds the key itself.
template <bool MANY>
__global__ __launch_bounds__(kSelectThreads) void select_write_kernel(SelectArgs a)
{
    __shared__ unsigned counts[kPerThread * kSelectThreads / 64];
    const int tid = threadIdx.x, part = blockIdx.x % a.parts, stream = blockIdx.x / a.parts;
    const Middle m = middle_of(a, stream);
    if (m.len <= part * kPart) return;
    Keys<kSelectThreads> keys;
    keys.load(m, part, tid);
    if constexpr (MANY) {
        const uint4 run = a.runs[blockIdx.x];
        write_kept<kSelectThreads>(a, m, keys, run.z, run.w, run.x, run.y, counts, tid);
    } else {
        __shared__ __align__(16) KeySearch::Lds lds;
        KeySearch search(lds, a, stream);
        search.find(a.found[stream]);
        // what the runs in front keep
        unsigned gt = tid < part ? search.runs[tid].y : 0u, eq = 0, gt_base, eq_base;
        if (search.one) {
            eq = tid == 0 ? lds.starts[part] : 0u;
        } else if (search.in_lds) {
            for (unsigned i = tid; i < lds.starts[part]; i += kSelectThreads) {
                gt += lds.held[i] > search.key;
                eq += lds.held[i] == search.key;
            }
        } else {
            for (int p = tid >> 6; p < part; p += KeySearch::kWaves)
                search.of_run(p, false, [&](bool is, unsigned, unsigned x) {
                    gt += is && x > search.key;
                    eq += is && x == search.key;
                });
        }
        block_prefix<kSelectThreads>(gt, lds.sums, tid, &gt_base);
        block_prefix<kSelectThreads>(eq, lds.sums, tid, &eq_base);
        write_kept<kSelectThreads>(a, m, keys, search.key, search.need, gt_base, eq_base, counts, tid);
    }
}

// ---------------------------------------------------------------------------------- moving
constexpr int kMoveThreads = 256;

// out byte i = in byte (i + by) mod 4 W
// (A vector, and a mask the compiler cannot see through: it makes of a choice between two words one word at a chosen index, and
// of an array that is indexed so memory.)
template <int W>
using Words = unsigned __attribute__((ext_vector_type(W)));
template <int W>
__device__ __forceinline__ void rotate_bytes(Words<W>& w, unsigned by)
{
#pragma unroll
    for (int d = 1; d < W; d *= 2) {
        unsigned on = 0u - ((by >> 2 & (unsigned)d) / d);
        asm("" : "+v"(on));
        Words<W> x;
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = (w[(i + d) % W] & on) | (w[i] & ~on);
        w = x;
    }
    const unsigned first = w[0];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = __builtin_amdgcn_alignbyte(i + 1 < W ? w[i + 1] : first, w[i], by & 3u);
}

// a token's record: Gh low bytes in 16-byte pieces, and (b = 10) the word of high bits
template <int GH, int B>
struct Record {
    Words<GH / 4> w;
    unsigned hi;
    __device__ __forceinline__ void load(const uint8_t* tile, int u)
    {
#pragma unroll
        for (int p = 0; p < GH / 16; ++p) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(tile + p * 1024 + u * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * p + i] = x[i];
        }
        if constexpr (B == 10) hi = *reinterpret_cast<const unsigned*>(tile + kTileTokens * GH + u * 4);
    }
    __device__ __forceinline__ void store(uint8_t* tile, int u) const
    {
#pragma unroll
        for (int p = 0; p < GH / 16; ++p)
            *reinterpret_cast<u32x4*>(tile + p * 1024 + u * 16) = u32x4{w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]};
        if constexpr (B == 10) *reinterpret_cast<unsigned*>(tile + kTileTokens * GH + u * 4) = hi;
    }
    __device__ __forceinline__ void move(int from, int to)
    {
        const unsigned by = (unsigned)(to - from) & (unsigned)(GH - 1);
        rotate_bytes<GH / 4>(w, by);
        if constexpr (B == 10) hi = __builtin_amdgcn_alignbit(hi, hi, 2 * by);
    }
};

// A wavefront moves a tile of one stream of one cache, or (tiles behind the last that is kept) clears its accumulators.
// GATHER: from a token's old position to its new one (in the caches, or in the workspace where the caches' own places are
// still to be read); else from the workspace to the caches.
// Bound by the length of its chain of requests (arguments, list and lengths, codes), so each link asks for all it can: left to the
// compiler the arguments' loads stand behind the branches that use them, a round each (2047 of 131072 tokens of 32 streams 17 us).
template <int GH, int B, bool GATHER>
__global__ __launch_bounds__(kMoveThreads) void move_tokens_kernel(CompactArgs a, int tiles, int work_tiles)
{
    constexpr int TILE = kTileTokens * GH * B / 8;
    const int lane = threadIdx.x & 63;
    const int tile = (int)blockIdx.x * (kMoveThreads / 64) + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int stream = blockIdx.y, which = blockIdx.z;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    const int r = tile * kTileTokens + lane;
    const uint8_t* const in = which ? a.in[1] : a.in[0];
    uint8_t* const out = which ? a.out[1] : a.out[0];
    const CacheMap map_in = a.map_in, map_out = a.map_out;
    asm volatile("" ::"s"(in), "s"(out), "s"(map_in.block_table), "s"(map_in.bt_stride), "s"(map_in.n_pages), "s"(map_in.tiles_cap),
                 "s"(map_in.n_kv_heads), "s"(map_out.block_table), "s"(map_out.bt_stride), "s"(map_out.n_pages), "s"(map_out.tiles_cap),
                 "s"(map_out.n_kv_heads), "s"(a.weights), "s"(a.weights_stride), "s"(a.weights_out), "s"(a.weights_out_stride), "s"(a.kept),
                 "s"(a.kept_lens), "s"(a.t), "s"(a.keep), "s"(a.clear_end), "s"(a.work), "s"(a.work_weights));
    int from = a.kept[(size_t)stream * a.keep + min(r, a.keep - 1)], len = a.kept_lens[n];
    size_t out_tile = map_out.tile_index(n, h, tile);
    asm volatile("" : "+v"(from), "+v"(len), "+v"(out_tile));
    const int count = min(max(len, 0), a.keep);
    const size_t work_tile = ((size_t)stream * work_tiles + tile) * 2 + which;
    float* const weights_out = a.weights_out + (size_t)stream * a.weights_out_stride + r;
    float* const work_weights = a.work_weights + (size_t)stream * a.keep + r;
    const bool weigh = which == 0 && a.weights;
    if (r < count) {
        Record<GH, B> rec;
        float w = 0.f;
        if constexpr (GATHER) {
            from = min(max(from, 0), a.t - 1);
            rec.load(in + map_in.tile_index(n, h, from / kTileTokens) * TILE, from % kTileTokens);
            if (weigh) w = a.weights[(size_t)stream * a.weights_stride + from];
            rec.move(from % kTileTokens, lane);
            rec.store(a.work ? a.work + work_tile * TILE : out + out_tile * TILE, lane);
            if (weigh) *(a.work ? work_weights : weights_out) = w;
        } else {
            rec.load(a.work + work_tile * TILE, lane);
            if (weigh) w = *work_weights;
            rec.store(out + out_tile * TILE, lane);
            if (weigh) *weights_out = w;
        }
    } else if (weigh && r < a.clear_end && (!a.work || !GATHER)) {
        *weights_out = 0.f;
    }
}

// In place, a workgroup per stream of one cache: a token moves towards the front and the list ascends, so a block of tokens
// that is read before it is written overwrites nothing that a later one reads.  The next block is on its way meanwhile.
constexpr int kSlideThreads = 512;
template <int GH, int B>
__global__ __launch_bounds__(kSlideThreads) void slide_tokens_kernel(CompactArgs a)
{
    constexpr int TILE = kTileTokens * GH * B / 8;
    const int tid = threadIdx.x, which = blockIdx.x & 1, stream = blockIdx.x >> 1;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    uint8_t* const codes = which ? a.out[1] : a.out[0];
    const CacheMap map = a.map_out;
    asm volatile("" ::"s"(codes), "s"(map.block_table), "s"(map.bt_stride), "s"(map.n_pages), "s"(map.tiles_cap), "s"(map.n_kv_heads),
                 "s"(a.weights), "s"(a.weights_out), "s"(a.weights_out_stride), "s"(a.kept), "s"(a.kept_lens), "s"(a.t), "s"(a.keep), "s"(a.clear_end));
    const int count = min(max(a.kept_lens[n], 0), a.keep);
    const int32_t* kept = a.kept + (size_t)stream * a.keep;
    const bool weigh = which == 0 && a.weights;
    float* const weights = a.weights_out + (size_t)stream * a.weights_out_stride;
    auto source = [&](int r) { return r < count ? min(max(kept[r], 0), a.t - 1) : r; };
    struct Token {
        Record<GH, B> rec;
        float w;
        int from;
    };
    auto load = [&](Token& x, int r, int from) {
        x.from = from;
        if (from != r) {                                    // (tokens in front of the first that goes stay where they are)
            x.rec.load(codes + map.tile_index(n, h, from / kTileTokens) * TILE, from % kTileTokens);
            if (weigh) x.w = weights[from];
        }
    };
    Token now, next;
    load(now, tid, source(tid));
    int from_next = source(kSlideThreads + tid);
#pragma unroll 1
    for (int base = 0; base < count; base += kSlideThreads) {
        const int r = base + tid;
        load(next, r + kSlideThreads, from_next);
        from_next = source(r + 2 * kSlideThreads);
        const bool moves = now.from != r;
        if (moves) {
            now.rec.move(now.from % kTileTokens, r % kTileTokens);
            asm volatile("" :: "v"(now.rec.w[0]), "v"(now.rec.w[GH / 4 - 1]), "v"(now.rec.hi), "v"(now.w) : "memory");   // (all of it is here)
        }
        lds_barrier();                                      // the block is read
        if (moves) {
            now.rec.store(codes + map.tile_index(n, h, r / kTileTokens) * TILE, r % kTileTokens);
            if (weigh) weights[r] = now.w;
        }
        now = next;
    }
    if (weigh)
        for (int r = count + tid; r < a.clear_end; r += kSlideThreads) weights[r] = 0.f;
}

template <int GH, int B>
cq_status launch_move(const CompactArgs& a, hipStream_t stream)
{
    const int streams = a.batch * a.n_kv_heads;
    if (a.slide) {
        hipLaunchKernelGGL((slide_tokens_kernel<GH, B>), dim3(2u * (unsigned)streams), dim3(kSlideThreads), 0, stream, a);
        return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
    }
    const int work_tiles = (a.keep + kTileTokens - 1) / kTileTokens, end_tiles = (a.clear_end + kTileTokens - 1) / kTileTokens;
    for (int pass = 0; pass < (a.work ? 2 : 1); ++pass) {
        const bool last = !a.work || pass == 1;
        const int tiles = last && a.weights && end_tiles > work_tiles ? end_tiles : work_tiles;
        const dim3 grid((unsigned)((tiles + kMoveThreads / 64 - 1) / (kMoveThreads / 64)), (unsigned)streams, 2);
        if (pass == 0) hipLaunchKernelGGL((move_tokens_kernel<GH, B, true>), grid, dim3(kMoveThreads), 0, stream, a, tiles, work_tiles);
        else hipLaunchKernelGGL((move_tokens_kernel<GH, B, false>), grid, dim3(kMoveThreads), 0, stream, a, tiles, work_tiles);
        if (hipGetLastError() != hipSuccess) return CQ_ERR_HIP;
    }
    return CQ_OK;
}

}  // namespace

cq_status launch_select_tokens(const SelectArgs& a, hipStream_t stream)
{
    const unsigned grid = (unsigned)(a.batch * a.n_kv_heads) * (unsigned)a.parts;
    if (a.parts == 1) {
        hipLaunchKernelGGL(select_short_kernel<kSelectThreads>, dim3(grid), dim3(kSelectThreads), 0, stream, a);
    } else {
        hipLaunchKernelGGL(select_count_kernel, dim3(grid), dim3(kSelectThreads), 0, stream, a);
        const unsigned streams = (unsigned)(a.batch * a.n_kv_heads);
        if (a.many) hipLaunchKernelGGL(select_digit_kernel, dim3(streams), dim3(kSelectThreads), 0, stream, a);
        hipLaunchKernelGGL(select_list_kernel, dim3(grid), dim3(kSelectThreads), 0, stream, a);
        if (a.many) {
            hipLaunchKernelGGL(select_key_kernel, dim3(streams), dim3(kSelectThreads), 0, stream, a);
            hipLaunchKernelGGL(select_write_kernel<true>, dim3(grid), dim3(kSelectThreads), 0, stream, a);
        } else {
            hipLaunchKernelGGL(select_write_kernel<false>, dim3(grid), dim3(kSelectThreads), 0, stream, a);
        }
    }
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_compact(const CompactArgs& a, const Derived& f, hipStream_t stream)
{
    if (f.b == 10) return launch_move<16, 10>(a, stream);
    if (f.gh == 16) return launch_move<16, 8>(a, stream);
    if (f.gh == 32) return launch_move<32, 8>(a, stream);
    if (f.gh == 64) return launch_move<64, 8>(a, stream);
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace cq
