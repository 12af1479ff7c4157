// A kernel of cq_chunk_lds.hip: included twice there, for whole contexts and (CQ_VIEW_KERNEL) for windows of them.  (One text and two
// kernels: as a function that both inline, the first was scheduled otherwise.)
#if CQ_VIEW_KERNEL
#define CQ_TILE(i) it.seen.tile(i)
#define CQ_REQUESTED(i) it.seen.requested(i, it.tile0, it.tile1)
#define CQ_HIDES(tile) (CQ_TILE(tile) * kTileTokens + kTileTokens - 1 > it.pos_first || before_window(a, CQ_TILE(tile), it.pos_last))
#define CQ_SEES(tok) in_window(a, tok, it.pos)
template <int C, bool HALF>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kWaves * 64) void chunk_lds_window_kernel(ChunkViewArgs a, int rb_log2, int items)
{
#else
#define CQ_TILE(i) (i)
#define CQ_REQUESTED(i) max(min(i, it.tile1 - 1), it.tile0)
#define CQ_HIDES(tile) tile * kTileTokens + kTileTokens - 1 > it.pos_first
#define CQ_SEES(tok) tok <= it.pos
template <int C, bool HALF>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kWaves * 64) void chunk_lds_kernel(ChunkArgs a, int rb_log2, int items)
{
#endif
    constexpr int D = 128;
    constexpr int GH = D / C;
    constexpr int PL = GH / 16;
    constexpr int TILE_BYTES = kTileTokens * GH;
    extern __shared__ float smem[];
    (void)smem;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, blk = lane >> 4;

    const int cs = kWaves >> rb_log2;                       // context slices of each of the 2^rb_log2 row blocks
    const int rb = wave >> (3 - rb_log2), slice = wave & (cs - 1);
    const int hkv = blockIdx.x % a.f.n_kv_heads;
    const int stride = gridDim.x / a.f.n_kv_heads;
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int rows_total = a.m * qper;

    // ---- this lane's places: keys, token col of a block of 16, groups blk, blk + 4, ...; values, token
    // 4 blk + col / 4 of a block, channels 4 (col % 4) .. of 16 (C = 8: half of group (col % 4) / 2, then
    // every second group; C = 4: group col % 4, then every fourth)
    const int vtok = 4 * blk + (col >> 2);
    const CodePick<GH, 4> kpick(blk, col);
    const CodePick<GH, C == 8 ? 2 : 4> vpick(C == 8 ? (col & 3) >> 1 : (col & 3), vtok);
    const unsigned kbase = (unsigned)blk * (256 * 2 * C);
    const unsigned vbase = kBookBytes + (C == 8 ? ((unsigned)(col & 3) >> 1) * 4096 + (unsigned)(col & 1) * 8 : (unsigned)(col & 3) * 2048);


    // ---- the items of this workgroup: (sequence, split), advanced without divisions
    const float inv_qper = 1.f / (float)qper;
    const auto row_token = [&](int row) { return (int)(((float)row + 0.5f) * inv_qper); };     // row / qper (few rows: exact)
    int item = blockIdx.x / a.f.n_kv_heads;
    int split = item % a.n_split, n = item / a.n_split;
    const int d_split = stride % a.n_split, d_n = stride / a.n_split;
    int row0 = rb * kRows;                                  // (a block beyond the last row repeats it and stores nothing)
    struct Item {
        int n, split, pos, pos_first, tile0, tile1;
#if CQ_VIEW_KERNEL
        int pos_last;
        ChunkSeen seen;
#endif
    };
    // (a scale of zero stands for one so small that every weight is 1: 0 times a masked -infinity is no number)
    const float scale = a.scale_log2e == 0.f ? 1e-37f : fabsf(a.scale_log2e);
    half8_t qreg[4];
    // the records of a tile on their way from memory, and the codes of one that this lane needs
    u32x4 rk[4][PL], rv[4][PL];                             // token 16 i + col, token 16 i + vtok
    unsigned zk[4][GH / 16], zv[4][2];
    auto request = [&](const Item& it, int tile) {
        const size_t at = a.map.tile_index(it.n, hkv, CQ_REQUESTED(tile)) * TILE_BYTES;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int p = 0; p < PL; ++p) {
                rk[i][p] = *reinterpret_cast<const u32x4*>(a.k_codes + at + p * 1024 + (16 * i + col) * 16);
                rv[i][p] = *reinterpret_cast<const u32x4*>(a.v_codes + at + p * 1024 + (16 * i + vtok) * 16);
            }
    };
    auto unpack = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kpick(rk[i], i & 1, zk[i]);
            vpick(rv[i], i & 1, zv[i]);
        }
    };
    // an item's places, its queries and its first tile's records (requested ahead of the codebooks or of
    // the previous item's merge)
    auto open_item = [&]() {
        // (opaque per item: what follows from it would be kept in registers through the tiles, which spill then)
        asm volatile("" : "+s"(row0));
        Item it;
        it.n = n;
        it.split = split;
        int t_n = a.t;
        if (a.seq_lens) t_n = min(max(a.seq_lens[n], a.m), a.t);
        const int pos0 = t_n - a.m;                         // position of query token 0
        const int row = min(row0 + (HALF ? col & 7 : col), rows_total - 1);
        const int j = row_token(row);
        it.pos = pos0 + j;
        it.pos_first = __builtin_amdgcn_readfirstlane(pos0 + row_token(min(row0, rows_total - 1)));
        const int last_row = min(row0 + kRows, rows_total) - 1;
#if CQ_VIEW_KERNEL
        it.pos_last = __builtin_amdgcn_readfirstlane(pos0 + row_token(max(last_row, 0)));
        it.seen = ChunkSeen(a, it.pos_first, it.pos_last);
        const int last_tile = it.seen.n_tiles - 1;
#else
        const int last_tile = __builtin_amdgcn_readfirstlane((pos0 + row_token(last_row)) / kTileTokens);
#endif
        it.tile0 = split * a.tiles_per_split;
        it.tile1 = row0 < rows_total ? min(it.tile0 + a.tiles_per_split, last_tile + 1) : it.tile0;
        const uint16_t* qrow = a.q + (((size_t)n * a.m + j) * a.n_q_heads + hkv * qper + (row - j * qper)) * D;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if constexpr (C == 8) {
                qreg[s] = *reinterpret_cast<const half8_t*>(qrow + 32 * s + 8 * blk);
            } else {
                const half4_t lo = *reinterpret_cast<const half4_t*>(qrow + 32 * s + 4 * blk);
                const half4_t hi = *reinterpret_cast<const half4_t*>(qrow + 32 * s + 16 + 4 * blk);
                qreg[s] = half8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            }
        }
        request(it, it.tile0 + slice);
        return it;
    };
    // ---- both codebooks of the head to LDS as they are ([group][code] entries); requested ahead of the first codes, which
    // come from further away (loads return in order)
    typedef __attribute__((address_space(3))) u32x4 lds_q;
    u32x4 book[2][8];
    {
        const u32x4* src[2] = {reinterpret_cast<const u32x4*>(a.k_centroids + (size_t)hkv * GH * 256 * C),
                               reinterpret_cast<const u32x4*>(a.v_centroids + (size_t)hkv * GH * 256 * C)};
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) book[w][i] = src[w][i * (kWaves * 64) + tid];
    }
    __builtin_amdgcn_sched_barrier(0);
    Item it = open_item();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 8; ++i) *(lds_q*)(w * kBookBytes + (unsigned)(i * (kWaves * 64) + tid) * 16) = book[w][i];

    lds_barrier();

#pragma unroll 1
    for (;;) {
        float4_t o[8];
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) o[cb] = float4_t{0.f, 0.f, 0.f, 0.f};
        float ref = -INFINITY, l_run = 0.f;             // probabilities and their sum are relative to 2^ref

        // (a negative scale goes into the queries, so that the largest product is the largest score)
        if (a.scale_log2e < 0.f) {
#pragma unroll
            for (int s = 0; s < 4; ++s) qreg[s] = -qreg[s];
        }
        // (no element of Q Q^T is larger than the largest of its diagonal, the squares of the queries' norms)
        float4_t g = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) g = __builtin_amdgcn_mfma_f32_16x16x32_f16(qreg[s], qreg[s], g, 0, 0, 0);
        const bool large = scores_may_be_large(fmaxf(fmaxf(g[0], g[1]), fmaxf(g[2], g[3])), scale, 0x1p24f);
        int tile = it.tile0 + slice;
        unpack();
        request(it, tile + cs);
        const float mult = large ? 1.f : scale, early = large ? scale : 1.f;
        bool turn = wave < kWaves / 2;                  // (priorities as in cq_decode_quad.hip)
        constexpr bool kPriorities = !(HALF && C == 8);
#pragma unroll 1
        for (; tile < it.tile1; tile += cs) {
            // All keys of the tile are gathered at once, the values in batches that the products behind them work off, one batch
            // ahead (the scheduling fences pin that order: left alone, the compiler waits for every gather by itself,
            // 130 clocks each).
            // ---- scores: acc[i][e] is token 16 i + 4 blk + e, query col
            if constexpr (kPriorities) {
                turn = !turn;
                if (turn) __builtin_amdgcn_s_setprio(1);
                else __builtin_amdgcn_s_setprio(0);
            }
            float4_t acc[4];
            half8_t kv[4][4];
            auto gather_keys = [&](int i) {
                unsigned at[GH / 4];
#pragma unroll
                for (int k = 0; k < GH / 4; ++k) at[k] = entry<C>(zk[i][k >> 2], k & 3, kbase);
                __builtin_amdgcn_sched_barrier(0);          // (addresses first: a gather right behind its own would wait for it)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if constexpr (C == 8) {
                        kv[i][s] = lds_half8(at[s] + (unsigned)s * 16384);
                    } else {
                        const half4_t lo = lds_half4(at[2 * s] + (unsigned)(2 * s) * 8192);
                        const half4_t hi = lds_half4(at[2 * s + 1] + (unsigned)(2 * s + 1) * 8192);
                        kv[i][s] = half8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    }
                }
            };
            half8_t av[2][8];
            auto gather_values = [&](int t) {
                unsigned at[2][8];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int cb = 0; cb < 8; ++cb) at[h][cb] = entry<C>(zv[2 * t + h][cb >> 2], cb & 3, vbase);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) {
                    const half4_t v0 = lds_transposed(at[0][cb] + (unsigned)cb * 8192), v1 = lds_transposed(at[1][cb] + (unsigned)cb * 8192);
                    av[t][cb] = half8_t{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                }
            };
            gather_keys(0);
            gather_keys(1);
            gather_keys(2);
            gather_keys(3);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv[i][s], qreg[s], acc[i], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            gather_values(0);
            __builtin_amdgcn_sched_barrier(0);
            // ---- online softmax of the lane's query column
            if constexpr (kPriorities) {
                if (turn) __builtin_amdgcn_s_setprio(3);
                else __builtin_amdgcn_s_setprio(2);
            }
            if (large || CQ_HIDES(tile)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int tok = CQ_TILE(tile) * kTileTokens + 16 * i + 4 * blk + e;
                        acc[i][e] = CQ_SEES(tok) ? acc[i][e] * early : -INFINITY;
                    }
            }
            float bmax = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) bmax = fmaxf(bmax, acc[i][e]);
            const float ref_new = fmaxf(ref, softmax_reference(across_max(bmax) * mult));
            const float shift = ref_new == -INFINITY ? 0.f : ref_new;       // nothing visible yet: all weights 0
            const float alpha = __builtin_amdgcn_exp2f(ref - shift);
            ref = ref_new;
            float psum = 0.f;
            half8_t ph[2], pl[2];                           // p = ph + pl to 22 bits (HALF: ph of columns q, q + 8)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float2_t ps = {__builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][e], mult, -shift)),
                                         __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][e + 1], mult, -shift))};
                    psum += ps[0];
                    psum += ps[1];
                    const half2_t hi = __builtin_convertvector(ps, half2_t);
                    const float2_t rest = {__builtin_fmaf((float)hi[0], -1.f, ps[0]), __builtin_fmaf((float)hi[1], -1.f, ps[1])};
                    const half2_t lo = __builtin_convertvector(rest, half2_t);
                    const int at = 4 * (i & 1) + e;
                    if constexpr (HALF) {
                        const half2_t v = __builtin_bit_cast(half2_t, col < 8 ? __builtin_bit_cast(unsigned, hi) : __builtin_bit_cast(unsigned, lo));
                        ph[i >> 1][at] = v[0];
                        ph[i >> 1][at + 1] = v[1];
                    } else {
                        ph[i >> 1][at] = hi[0];
                        ph[i >> 1][at + 1] = hi[1];
                        pl[i >> 1][at] = lo[0];
                        pl[i >> 1][at + 1] = lo[1];
                    }
                }
            l_run = __builtin_fmaf(l_run, alpha, psum);
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) o[cb] *= alpha;
            }
            // ---- O^T += V^T P^T: contraction index (blk, 4 h + e) is token 32 t + 16 h + 4 blk + e
            __builtin_amdgcn_sched_barrier(0);
            gather_values(1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) {
                    o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[t][cb], ph[t], o[cb], 0, 0, 0);
                    if constexpr (!HALF) o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[t][cb], pl[t], o[cb], 0, 0, 0);
                }
            // the next tile's codes, and the request for the tile after it
            unpack();
            request(it, tile + 2 * cs);
        }

        // ---- the next item's requests go out, then the context slices of every row block are merged: (ref, l),
        // then the rows, scaled to the common maximum, 64 channels at a time
        const Item done = it;
        item += stride;
        const bool more = item < items;
        if (more) {
            split += d_split;
            const int c1 = split >= a.n_split;
            split -= c1 ? a.n_split : 0;
            n += d_n + c1;
            it = open_item();
        }
        typedef __attribute__((address_space(3))) float lds_f;
        typedef __attribute__((address_space(3))) float2_t lds_f2;
        typedef __attribute__((address_space(3))) float4_t lds_f4;
        const float l = across_sum(l_run);
        if (blk == 0) *(lds_f2*)(kMergeBase + (unsigned)(wave * kRows + col) * 8) = float2_t{ref, l};
        lds_barrier();
        float2_t ml[kWaves];                                // of the wavefronts that share this one's row block, this lane's row
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ml[w] = *(lds_f2*)(kMergeBase + (unsigned)((rb * cs + (w & (cs - 1))) * kRows + col) * 8);
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, ml[w][0]);
        const float mz = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ll += w < cs ? ml[w][1] * __builtin_amdgcn_exp2f(ml[w][0] - mz) : 0.f;
        float weight = __builtin_amdgcn_exp2f(ref - mz);
        if (a.n_split == 1) weight *= 1.f / ll;
        if (a.n_split > 1 && slice == 0 && blk == 0 && row0 + col < rows_total) {
            const int j = row_token(row0 + col);
            const size_t out_row = ((size_t)done.n * a.m + j) * a.n_q_heads + hkv * qper + (row0 + col - j * qper);
            float* dst = a.partials + (out_row * a.n_split + done.split) * (D + kPartialHeader);
            dst[0] = mm;
            dst[1] = ll;
        }
        lds_barrier();                                      // the pairs are read: their room is the rows'
        if constexpr (HALF) {
            // (8 rows, one row block: all 128 channels of every wavefront at once; the parts of a row's probabilities, columns
            // q and q + 8, are added here)
            const int q = tid >> 6;
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) {
                float4_t v = o[cb];
#pragma unroll
                for (int e = 0; e < 4; ++e)             // (lane l + 8 mod 16 of the row)
                    v[e] += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v[e]), 0x128, 0xf, 0xf, false));
                // (the pieces of row q change places by 4 q: the 32 lanes that write fill 512 bytes)
                if (col < 8) *(lds_f4*)(kMergeBase + (unsigned)(wave * 8 + col) * 512 + (unsigned)((4 * cb + blk) ^ (4 * col)) * 16) = v * weight;
            }
            lds_barrier();
            float2_t sum = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                sum += *(lds_f2*)(kMergeBase + (unsigned)(w * 8 + q) * 512 + (unsigned)((lane >> 1) ^ (4 * q)) * 16 + (lane & 1) * 8);
            if (q < rows_total) {
                const int j = row_token(q);
                const size_t out_row = ((size_t)done.n * a.m + j) * a.n_q_heads + hkv * qper + (q - j * qper);
                if (a.n_split == 1)
                    *reinterpret_cast<half2_t*>(a.out + out_row * D + 2 * lane) = __builtin_convertvector(sum, half2_t);
                else
                    *reinterpret_cast<float2_t*>(a.partials + (out_row * a.n_split + done.split) * (D + kPartialHeader) + kPartialHeader + 2 * lane) = sum;
            }
            if (!more) break;
            lds_barrier();
            continue;
        }
        int tid_o = tid, lane_o = lane;                     // (opaque, as above; all of it only where registers are short)
        if constexpr (C == 4) asm volatile("" : "+v"(tid_o), "+v"(lane_o));
        int q = tid_o >> 5;                                 // this thread's row and pair of channels
        if constexpr (C != 4) asm volatile("" : "+v"(q));
        const unsigned osrc = kMergeBase + (unsigned)q * kORow + (((unsigned)(tid_o & 31) >> 1) ^ (unsigned)q) * 16 + (tid_o & 1) * 8;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float4_t v = o[4 * part + h];
                // (16-byte pieces of a row change places by the row's number: 16 rows, 16 different banks)
                *(lds_f4*)(kMergeBase + (unsigned)(wave * kRows + (lane_o & 15)) * kORow + (unsigned)((4 * h + (lane_o >> 4)) ^ (lane_o & 15)) * 16) = v * weight;
            }
            lds_barrier();
            float2_t sum = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                sum += *(lds_f2*)(osrc + (unsigned)(w * kRows) * kORow);
                if (((w + 1) & (cs - 1)) != 0) continue;    // (the row block's last slice)
                const int r2 = (w >> (3 - rb_log2)) * kRows + q;
                if (r2 < rows_total) {
                    const int j = row_token(r2);
                    const size_t out_row = ((size_t)done.n * a.m + j) * a.n_q_heads + hkv * qper + (r2 - j * qper);
                    const int ch = part * 64 + 2 * (tid_o & 31);
                    if (a.n_split == 1)
                        *reinterpret_cast<half2_t*>(a.out + out_row * D + ch) = __builtin_convertvector(sum, half2_t);
                    else
                        *reinterpret_cast<float2_t*>(a.partials + (out_row * a.n_split + done.split) * (D + kPartialHeader) + kPartialHeader + ch) = sum;
                }
                sum = float2_t{0.f, 0.f};
            }
            lds_barrier();
        }
        if (!more) break;
    }
}
#undef CQ_TILE
#undef CQ_REQUESTED
#undef CQ_HIDES
#undef CQ_SEES
