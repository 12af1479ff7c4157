// A kernel of cq_chunk_lds.hip: included twice there, for whole contexts and (CQ_VIEW_KERNEL) for windows of them.  (One text and two
// kernels: as a function that both inline, the first was scheduled otherwise.)
#if CQ_VIEW_KERNEL
#define CQ_TILE(i) it.seen.tile(i)
#define CQ_HIDES(tile) CQ_TILE(tile) * kTileTokens + kTileTokens - 1 > pos0 || before_window(a, CQ_TILE(tile), it.t_n - 1)
#define CQ_SEES(tok, pos) in_window(a, tok, pos)
template <int C>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kWaves * 64) void chunk_few_window_kernel(ChunkViewArgs a, int per_head, int items)
{
#else
#define CQ_TILE(i) (i)
#define CQ_HIDES(tile) tile * kTileTokens + kTileTokens - 1 > pos0
#define CQ_SEES(tok, pos) tok <= pos
template <int C>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kWaves * 64) void chunk_few_kernel(ChunkArgs a, int per_head, int items)
{
#endif
    constexpr int D = 128, GH = D / C, K = 256, PL = GH / 16, NT = kWaves * 64, ROWS = 4, PARTS = 3;
    constexpr int TILE_BYTES = kTileTokens * GH;
    typedef __attribute__((address_space(3))) u32x4 lds_q;
    typedef __attribute__((address_space(3))) float lds_f;
    typedef __attribute__((address_space(3))) float2_t lds_f2;
    typedef __attribute__((address_space(3))) float4_t lds_f4;
    extern __shared__ float smem[];
    (void)smem;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, blk = lane >> 4;
    const int hkv = blockIdx.x % a.f.n_kv_heads;
    int item = blockIdx.x / a.f.n_kv_heads;
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int rows_total = a.m * qper;
    const float inv_qper = 1.f / (float)qper;
    const auto row_token = [&](int row) { return (int)(((float)row + 0.5f) * inv_qper); };     // row / qper (few rows: exact)

    // ---- both codebooks of the head on their way to LDS, ahead of the first codes, which come from further away
    u32x4 book[2][8];
    {
        const u32x4* src[2] = {reinterpret_cast<const u32x4*>(a.k_centroids + (size_t)hkv * GH * K * C),
                               reinterpret_cast<const u32x4*>(a.v_centroids + (size_t)hkv * GH * K * C)};
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) book[w][i] = src[w][i * NT + tid];
    }

    // ---- this lane's places: keys, token `lane`; values, tokens 32 t + 8 blk + 4 r + col / 4, channels 4 (col % 4) .. of 16
    // (C = 8: half of group (col % 4) / 2, then every second group; C = 4: group col % 4, then every fourth)
    Unrotate unrot;
    unrot.bytes = (unsigned)(GH - lane) & 3u;
    unrot.dwords = ((unsigned)(GH - lane) & (unsigned)(GH - 1)) >> 2;
    const int vg0 = C == 8 ? (col & 3) >> 1 : (col & 3);
    const int u0 = 8 * blk + (col >> 2);
    const CodePick<GH, C == 8 ? 2 : 4> pick0(vg0, u0), pick1(vg0, u0 + 4);
    const unsigned vbase = kBookBytes + (C == 8 ? (unsigned)vg0 * 4096 + (unsigned)(col & 1) * 8 : (unsigned)vg0 * 2048);
    // (a token's 32 bytes of probabilities: halves exchanged for every second run of eight tokens, for the banks)
    const unsigned work = kMergeBase + (unsigned)wave * kFewWaveBytes;
    const unsigned prob_in = work + (unsigned)lane * 32, prob_swap = (unsigned)((lane >> 3) & 1) * 16;
    const unsigned prob_out = work + (unsigned)u0 * 32 + (((unsigned)(col & 3) * 8) ^ (unsigned)(blk & 1) * 16);

    struct Item {
        int n, split, t_n, tile0, tile1, n_tiles;
#if CQ_VIEW_KERNEL
        ChunkSeen seen;
#endif
    };
    half4_t qreg[2];                                    // channels 4 (16 r + lane / 4) .. of row lane % 4
    Tile<GH, 8> krec;
    u32x4 vrec[2][2][PL];
    auto request = [&](const Item& it, int tile) {
        const size_t at = a.map.tile_index(it.n, hkv, CQ_TILE(min(tile, it.n_tiles - 1))) * TILE_BYTES;
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) krec.lo[pl] = *reinterpret_cast<const u32x4*>(a.k_codes + at + pl * 1024 + lane * 16);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int rr = 0; rr < 2; ++rr)
#pragma unroll
                for (int pl = 0; pl < PL; ++pl)
                    vrec[t][rr][pl] = *reinterpret_cast<const u32x4*>(a.v_codes + at + pl * 1024 + (32 * t + 4 * rr + u0) * 16);
    };
    auto open_item = [&](int at) {
        Item it;
        it.split = at % a.n_split;
        it.n = at / a.n_split;
        it.t_n = a.t;
        if (a.seq_lens) it.t_n = min(max(a.seq_lens[it.n], a.m), a.t);
#if CQ_VIEW_KERNEL
        it.seen = ChunkSeen(a, it.t_n - a.m, it.t_n - 1);
        it.n_tiles = it.seen.n_tiles;
#else
        it.n_tiles = (it.t_n + kTileTokens - 1) / kTileTokens;
#endif
        it.tile0 = it.split * a.tiles_per_split;
        it.tile1 = min(it.tile0 + a.tiles_per_split, it.n_tiles);
        const int row = min(lane & 3, rows_total - 1), j = row_token(row);
        const uint16_t* qrow = a.q + (((size_t)it.n * a.m + j) * a.n_q_heads + hkv * qper + (row - j * qper)) * D;
#pragma unroll
        for (int i = 0; i < 2; ++i) qreg[i] = *reinterpret_cast<const half4_t*>(qrow + 64 * i + 4 * (lane >> 2));
        request(it, it.tile0 + wave);
        return it;
    };
    Item it = open_item(item);
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 8; ++i) *(lds_q*)(w * kBookBytes + (unsigned)(i * NT + tid) * 16) = book[w][i];
    lds_barrier();

#pragma unroll 1
    for (;;) {
        float4_t o[8];
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) o[cb] = float4_t{0.f, 0.f, 0.f, 0.f};
        float ref[ROWS], l[ROWS];                           // (l: this lane's tokens)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            ref[r] = kNoScore;
            l[r] = 0.f;
        }
        unsigned d[GH / 4], z[2][2][2];                     // codes of the tile to come: keys in group order, values as picked
        auto unpack = [&]() {
            group_order<GH, 8>(krec, unrot, d);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                pick0(vrec[t][0], 0, z[t][0]);
                pick1(vrec[t][1], 0, z[t][1]);
            }
        };
        const int pos0 = it.t_n - a.m;                      // position of query token 0
        int tile = it.tile0 + wave;
        bool turn = wave < kWaves / 2;                      // (priorities as in cq_decode_quad.hip)
        unpack();
        request(it, tile + kWaves);
#pragma unroll 1
        for (; tile < it.tile1; tile += kWaves) {
            turn = !turn;
            if (turn) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
            // ---- scores of the lane's token
            float4_t acc[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = float4_t{0.f, 0.f, 0.f, 0.f};
            {
                unsigned at[GH];
#pragma unroll
                for (int g = 0; g < GH; ++g) at[g] = entry<C>(d[g >> 2], g & 3, 0u);
                __builtin_amdgcn_sched_barrier(0);          // (addresses first: a gather right behind its own would wait for it)
                CenVec<C> kv[GH];
#pragma unroll
                for (int g = 0; g < GH; ++g) kv[g] = lds_centroid<C>(at[g] + (unsigned)g * (K * C * 2));
                __builtin_amdgcn_sched_barrier(0);
                typedef unsigned u2 __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int g = 0; g < GH; ++g)
#pragma unroll
                    for (int p = 0; p < C / 4; ++p) {
                        const int i = g * (C / 4) + p;
                        acc[i & 3] = mfma_quad(qreg, __builtin_bit_cast(half4_t, u2{kv[g].w[2 * p], kv[g].w[2 * p + 1]}), acc[i & 3], i);
                    }
            }
            // ---- the values of tokens 0-31 on their way
            half8_t av[2][8];
            auto gather = [&](int t) {
                unsigned at[2][8];
#pragma unroll
                for (int rr = 0; rr < 2; ++rr)
#pragma unroll
                    for (int cb = 0; cb < 8; ++cb) at[rr][cb] = entry<C>(z[t][rr][cb >> 2], cb & 3, vbase);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) {
                    const half4_t v0 = lds_transposed(at[0][cb] + (unsigned)cb * 8192), v1 = lds_transposed(at[1][cb] + (unsigned)cb * 8192);
                    av[t][cb] = half8_t{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            if (turn) __builtin_amdgcn_s_setprio(3);
            else __builtin_amdgcn_s_setprio(2);
            gather(0);
            // ---- softmax
            float s[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s[r] = ((acc[0][r] + acc[1][r]) + (acc[2][r] + acc[3][r])) * a.scale_log2e;
            if (CQ_HIDES(tile)) {      // (some row does not see all of this tile)
                const int tok = CQ_TILE(tile) * kTileTokens + lane;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) s[r] = CQ_SEES(tok, pos0 + row_token(min(r, rows_total - 1))) ? s[r] : -INFINITY;
            }
            float over = s[0] - ref[0];
#pragma unroll
            for (int r = 1; r < ROWS; ++r) over = fmaxf(over, s[r] - ref[r]);
            if (__builtin_amdgcn_ballot_w64(over > 3.f) != 0) {
                float mine = 1.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fmaxf(ref[r], wave_max(s[r])))));
                    const float alpha = __builtin_amdgcn_exp2f(ref[r] - top);
                    l[r] *= alpha;
                    ref[r] = top;
                    mine = (lane & (ROWS - 1)) == r ? alpha : mine;
                }
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) o[cb] *= mine;
            }
            // p 2^12 as the sum of three fp16 numbers (what is left over each time is exact)
            unsigned part[PARTS][ROWS / 2];
#pragma unroll
            for (int r = 0; r < ROWS; r += 2) {
                float2_t p;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(s[r + e] - ref[r + e]) * 4096.f;     // (12 in the exponent would be lost in a large reference)
                    l[r + e] += p[e];
                }
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    const half2_t v = __builtin_convertvector(p, half2_t);
                    part[k][r >> 1] = __builtin_bit_cast(unsigned, v);
                    if (k + 1 < PARTS) p = float2_t{__builtin_fmaf((float)v.x, -1.f, p[0]), __builtin_fmaf((float)v.y, -1.f, p[1])};
                }
            }
            // (a wavefront's LDS operations keep their order; the statements keep the compiler from moving the reads, which
            // are of what other lanes wrote)
            *(lds_q*)(prob_in + prob_swap) = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
            *(lds_q*)(prob_in + (prob_swap ^ 16u)) = u32x4{part[2][0], part[2][1], 0u, 0u};
            asm volatile("" ::: "memory");
            half8_t pb[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const half4_t v0 = lds_transposed(prob_out + (unsigned)t * 1024), v1 = lds_transposed(prob_out + (unsigned)t * 1024 + 128);
                pb[t] = half8_t{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            }
            asm volatile("" ::: "memory");
            gather(1);
            // ---- O^T += V^T P
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int cb = 0; cb < 8; ++cb) o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[t][cb], pb[t], o[cb], 0, 0, 0);
            // the next tile's codes, and the request for the tile after it
            unpack();
            request(it, tile + 2 * kWaves);
        }

        // ---- the next item's requests go out, then the wavefronts are merged
        const Item done = it;
        item += per_head;
        const bool more = item < items;
        if (more) it = open_item(item);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float sum = wave_sum(l[r]);
            if (lane == 0) *(lds_f2*)(kFewPairs + (unsigned)(wave * ROWS + r) * 8) = float2_t{ref[r], sum};
        }
        // (the parts of a row are columns r, r + 4, r + 8)
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) {
            float4_t v = o[cb];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v[e]), 0x128, 0xf, 0xf, false));    // row_ror:8
                v[e] += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v[e]), 0x124, 0xf, 0xf, false));    // row_ror:4
            }
            if (col < ROWS) *(lds_f4*)(work + (unsigned)(col * D + 16 * cb + 4 * blk) * 4) = v;
        }
        lds_barrier();
        static_assert(NT == ROWS * D, "one output per thread");
        const int r = tid / D, ch = tid % D;
        float2_t ml[kWaves];
        float m = kNoScore;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            ml[w] = *(lds_f2*)(kFewPairs + (unsigned)(w * ROWS + r) * 8);
            m = fmaxf(m, ml[w][0]);
        }
        float sum = 0.f, ll = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float weight = __builtin_amdgcn_exp2f(ml[w][0] - m);
            sum = __builtin_fmaf(*(lds_f*)(kMergeBase + (unsigned)(w * ROWS * D + tid) * 4), weight, sum);
            ll = __builtin_fmaf(ml[w][1], weight, ll);
        }
        if (r < rows_total) {
            const int j = row_token(r);
            const size_t out_row = ((size_t)done.n * a.m + j) * a.n_q_heads + hkv * qper + (r - j * qper);
            if (a.n_split == 1) {
                a.out[out_row * D + ch] = __builtin_bit_cast(uint16_t, (_Float16)(sum / ll));
            } else {                                    // (a row that sees no token of the split: no weight)
                float* dst = a.partials + (out_row * a.n_split + done.split) * (D + kPartialHeader);
                if (ch == 0) {
                    dst[0] = m;
                    dst[1] = ll * 0x1p-12f;
                }
                dst[kPartialHeader + ch] = sum * 0x1p-12f;
            }
        }
        if (!more) break;
        lds_barrier();                                  // the rows and pairs are read: their room is the next item's
    }
}
#undef CQ_TILE
#undef CQ_HIDES
#undef CQ_SEES
