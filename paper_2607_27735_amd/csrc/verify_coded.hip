// verify_coded.hip -- verify attention with fused importance scores over the
// 8-bit paged cache.
//
//   out[row]    = sum_i P_i (vc_i vs_i),  P = softmax_i(sm_scale (q . kc_i) ks_i)
//   scores[i]   = sum over the window rows of P_i                       (Eq. 3)
//
// A score needs its row's normalizer over the whole context, which a pass that
// is split over the keys has only at its end.  So the call is two kernels:
//
//   coded_sweep_kernel   reads K and V once: per item (sequence, KV head, key
//                        chunk) and row the running maximum and sum of 2^y and
//                        the partial output over the item's keys;
//   coded_finish_kernel  its first workgroups read K again and write the
//                        scores 2^(y - lse); the others add the items' partial
//                        outputs, one row each.
//
// Bound by the codes' stream: 256 bytes per key and KV head in the first
// kernel, K's 128 again in the second, which finds part of them in the caches.
// Four sequences of 65536 keys, 48 rows, e4m3: 145 us per call back to back, for
// 541 MB that the sweep fetches (two workgroups per CU, so that one decodes while
// the other's loads are under way) and 288 for the scores, so that little of K is
// still in a cache: 5.7 TB/s over the call.  A ragged batch of 8 (298632 keys, 12 to
// 40 rows, int8): 170 us, 621 and 322 MB, 5.5 TB/s.  (Traced, each launch on its own,
// sweep and scores take about 104 and 62 us in the median of 60 launches, 91 and 50
// at the least; ragged about 123 and 65, 112 and 58.)  The matrix cores are busy for
// 13 to 22 % of that, the vector units for 41 to 53 %.  Where a call's chunks run in
// one round the streaming kernel of verify_stream.hip takes it, which reads K once
// and needs no second launch.
// More than 48 rows take four row tiles in one workgroup per CU, all sequences of
// the call alike (4 x 65536 keys, 56 rows: 180 to 187 us); more than 64 run in row
// blocks, each with both passes (128 rows: 376).
#include <stddef.h>

#include "coded_common.h"

namespace ssl {
namespace {

using namespace vc;
using namespace cc;

constexpr float kEmpty = kNoRef;

// decode_item() without its chain of loads: sixteen starts are compared at a
// time (those past the last sequence are larger than any item).
__device__ __forceinline__ int seq_of(const int32_t* start, int n_seq, int x) {
    int b = 0;
    for (int b0 = 0; b0 + 1 < n_seq; b0 += 16) {
#pragma unroll
        for (int i = 1; i <= 16; ++i) b += x >= start[b0 + i] ? 1 : 0;
    }
    return b;
}
__device__ __forceinline__ Item coded_item(const VerifyArgs& a, int item) {
    const int bt = seq_of(a.seq.item_start, a.seq.n_seq, item);
    Item it;
    it.bt = bt;
    it.b = a.sid[bt];
    it.T = a.seq.ctx[bt];
    it.nq = a.seq.qlen[bt];
    it.qoff = a.qoff[bt];
    it.qfull = a.qfull[bt];
    it.nchunk = (it.T + a.chunk - 1) / a.chunk;
    const int start = a.seq.item_start[bt], local = item - start;
    it.c = __builtin_amdgcn_readfirstlane(local / it.nchunk);
    it.s = local - it.c * it.nchunk;
    it.key_begin = it.s * a.chunk;
    it.key_end = min(it.key_begin + a.chunk, it.T);
    it.unit = it.b * a.n_kv_heads + it.c;
    it.item0 = start + it.c * it.nchunk;
    return it;
}

// What a sweep of NRT row tiles needs in LDS.
template <int NRT>
struct SweepLds {
    float2 wml[kWaves][NRT * 16];
    int last_key[NRT * 16];   // that each row sees
    union {
        __attribute__((aligned(16))) char q[NRT * 16 * kQStride];   // during the sweep
        f32x4 o[2][NRT * 16][kHeadDim / 4];                         // then
    };
};

template <int NRT, bool kInt8>
__device__ __forceinline__ void sweep_item(const CodedVerifyArgs& ca, const Item& it, SweepLds<NRT>& lds) {
    const VerifyArgs& a = ca.v;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // scalar, so buffer descriptors are
    const int m16 = lane & 15, G = lane >> 4;
    const int ntile = (it.key_end - it.key_begin + kTile - 1) / kTile;
    const int32_t* table = a.block_table + (size_t)it.b * a.max_blocks;
    const int all_see = it.T - it.qfull + it.qoff;   // keys up to here are visible to every row

    u32x4 q[NRT];
    q_load<NRT>(a, it.b, it.c, it.nq, it.qoff, q);
    float M[NRT], D[NRT], L[NRT];
    f32x4 oacc[8][NRT];
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
        M[rt] = kEmpty;
        D[rt] = L[rt] = 0.f;
#pragma unroll
        for (int jd = 0; jd < 8; ++jd) oacc[jd][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Logits: y[t][i] is key 16t + G + 4i for the lane's row (not yet scaled).
    auto logits = [&](const u32x4 (&k)[2][2], int key0, f32x4 (&y)[NRT][2]) __attribute__((always_inline)) {
        const int place = q_place(m16, G);
        u32x4 kd[2][4];
        decode_k<kInt8>(k[0], kd[0]);
        decode_k<kInt8>(k[1], kd[1]);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) {
            u32x4 qv[4];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) qv[kb] = q_operand(lds.q, place, rt, kb);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) s = mfma_bf16(kd[t][kb], qv[kb], s);
                y[rt][t] = s;
            }
        }
        if (key0 + kTile - 1 > all_see) {   // wave-uniform: some row does not see some key
#pragma unroll
            for (int rt = 0; rt < NRT; ++rt) {
                const int n = lds.last_key[place / kQStride + rt * 16] - key0 - G;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (16 * (e >> 2) + 4 * (e & 3) > n) y[rt][e >> 2][e & 3] = -INFINITY;
            }
        }
    };
    // The keys' weights in fp16.
    auto probs = [&](const f32x4 (&y)[NRT][2], float ks, float ve, float vr, u32x4 (&pb)[NRT]) __attribute__((always_inline)) {
        const float scale = logit_scale(a.scale_log2, ks);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) {
            f32x4 p[2], w[2];
            key_weights(
                y[rt], scale, ve, vr, M[rt], D[rt], L[rt], p, w, [](float, bool) {},
                [&](float alpha) __attribute__((always_inline)) {
#pragma unroll
                    for (int jd = 0; jd < 8; ++jd) oacc[jd][rt] *= alpha;
                });
            pb[rt] = u32x4{pack_f16(w[0][0], w[0][1]), pack_f16(w[0][2], w[0][3]), pack_f16(w[1][0], w[1][1]),
                           pack_f16(w[1][2], w[1][3])};
        }
    };
    auto values = [&](const u32x2 (&v)[8], const u32x4 (&pb)[NRT]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 av[4];
            decode_v<kInt8, true>(v, h, av);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int rt = 0; rt < NRT; ++rt) oacc[4 * h + d][rt] = mfma_f16(av[d], pb[rt], oacc[4 * h + d][rt]);
        }
    };
    auto start = [&] {
        q_store<NRT>(q, lds.q);
        if (threadIdx.x < NRT * 16) lds.last_key[threadIdx.x] = all_see + (int)threadIdx.x / a.group;
        __syncthreads();
    };
    const TileRun run = tile_run(ca.c, table, a.n_kv_heads, it.c, a.page_size, it.key_begin, ntile, wave, lane);
    // (K stays in the L2 for the score pass, V is not read again)
    auto load_k = [&](u32x4 (&k)[2][2], int t) __attribute__((always_inline)) {
        load_k_codes<false>(ca.c.k + tile_off(run, t), it.T - (it.key_begin + t * kTile), G, a_row_key(m16), k);
    };
    auto load_v = [&](u32x2 (&v)[8], int t) __attribute__((always_inline)) {
        load_v_codes<true>(ca.c.v + tile_off(run, t), it.T - (it.key_begin + t * kTile), m16, G, v);
    };
    auto scales = [&](int t, float& ks, float& ve, float& vr) __attribute__((always_inline)) {
        const int l = (t - wave) / kWaves;
        ks = lane_f(run.ks, l);
        ve = lane_f(run.ve, l);
        vr = lane_f(run.vr, l);
    };
    if constexpr (NRT <= 2) {
        tile_pipeline<(NRT == 1 ? 3 : 2), KVCodes>(
            wave, ntile, kWaves,
            [&](KVCodes& b, int t) __attribute__((always_inline)) {
                load_k(b.k, t);
                load_v(b.v, t);
            },
            [&](const KVCodes& b, int t) __attribute__((always_inline)) {
                f32x4 y[NRT][2];
                u32x4 pb[NRT];
                float ks, ve, vr;
                scales(t, ks, ve, vr);
                logits(b.k, it.key_begin + t * kTile, y);
                probs(y, ks, ve, vr, pb);
                values(b.v, pb);
            },
            start);
    } else {
        // One tile's codes in registers, so that a SIMD holds two waves: K of
        // the next tile is requested when the logits are formed, V when P V is.
        u32x4 k[2][2];
        u32x2 v[8];
        if (wave < ntile) {
            load_k(k, wave);
            __builtin_amdgcn_sched_barrier(0);
            load_v(v, wave);
            __builtin_amdgcn_sched_barrier(0);
        }
        start();
        auto step = [&](int t, bool last) __attribute__((always_inline)) {
            f32x4 y[NRT][2];
            u32x4 pb[NRT];
            float ks, ve, vr;
            scales(t, ks, ve, vr);
            logits(k, it.key_begin + t * kTile, y);
            if (!last) load_k(k, t + kWaves);
            probs(y, ks, ve, vr, pb);
            values(v, pb);
            if (!last) load_v(v, t + kWaves);
        };
        // (the last tile is peeled off: a load that may be skipped would make
        // every wait for K also wait for V)
        int t = wave;
        for (; t + kWaves < ntile; t += kWaves) step(t, false);
        if (t < ntile) step(t, true);
    }

    // The waves' statistics, then their shares of the workgroup's partial
    // output (see kPartialExp): waves 0 and 1 put theirs into LDS, 2 and 3 add
    // theirs, and the two sums are added on the way out.
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
        L[rt] += shfl_xor_f(L[rt], 16);
        L[rt] += shfl_xor_f(L[rt], 32);
        if (G == 0) lds.wml[wave][rt * 16 + m16] = make_float2(M[rt], L[rt]);
    }
    __syncthreads();
    const int R = it.nq * a.group;
    if (threadIdx.x < R) {
        float Mx = kEmpty, Lx = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) Mx = fmaxf(Mx, lds.wml[w][threadIdx.x].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) Lx += lds.wml[w][threadIdx.x].y * fast_exp2(lds.wml[w][threadIdx.x].x - Mx);
        a.part_ml[(size_t)blockIdx.x * kRowCap + threadIdx.x] = make_float2(Mx, Lx);
    }
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        if (wave >> 1 == turn) {
#pragma unroll
            for (int rt = 0; rt < NRT; ++rt) {
                const int row = rt * 16 + m16;
                float Mx = kEmpty;
#pragma unroll
                for (int u = 0; u < kWaves; ++u) Mx = fmaxf(Mx, lds.wml[u][row].x);
                const int shift = partial_shift(M[rt], D[rt], Mx);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4* at = &lds.o[wave & 1][row][8 * G + 2 * i];
                    f32x4 w0 = times_2(f32x4{oacc[0][rt][i], oacc[1][rt][i], oacc[2][rt][i], oacc[3][rt][i]}, shift);
                    f32x4 w1 = times_2(f32x4{oacc[4][rt][i], oacc[5][rt][i], oacc[6][rt][i], oacc[7][rt][i]}, shift);
                    if (turn) {
                        w0 += at[0];
                        w1 += at[1];
                    }
                    at[0] = w0;
                    at[1] = w1;
                }
            }
        }
        __syncthreads();
    }
    f32x4* po = reinterpret_cast<f32x4*>(a.part_o + (size_t)blockIdx.x * kRowCap * kHeadDim);
    for (int x = threadIdx.x; x < R * (kHeadDim / 4); x += kThreads)
        po[x] = lds.o[0][x >> 5][x & 31] + lds.o[1][x >> 5][x & 31];
}

// kMost: row tiles of the call's largest item.  Up to three (a SIMD holds two
// waves), each workgroup runs the body for its own sequence's row tiles.
template <int kMost, bool kInt8>
__global__ __launch_bounds__(kThreads, kMost <= 3 ? 2 : 1) void coded_sweep_kernel(CodedVerifyArgs ca) {
    __shared__ SweepLds<kMost> lds;
    const Item it = coded_item(ca.v, blockIdx.x);
    const int R = it.nq * ca.v.group;
    if constexpr (kMost == 4) {
        sweep_item<4, kInt8>(ca, it, lds);
    } else if (kMost == 1 || R <= 16) {
        sweep_item<1, kInt8>(ca, it, reinterpret_cast<SweepLds<1>&>(lds));
    } else if (kMost == 2 || R <= 32) {
        if constexpr (kMost >= 2) sweep_item<2, kInt8>(ca, it, reinterpret_cast<SweepLds<2>&>(lds));
    } else {
        if constexpr (kMost >= 3) sweep_item<3, kInt8>(ca, it, reinterpret_cast<SweepLds<3>&>(lds));
    }
}

// Merge of (M, L, o) states whose empty form is M = kEmpty, L = 0, o = 0.
__device__ __forceinline__ void mlo_merge(float& M, float& L, f32x4& o, float m, float l, f32x4 v) {
    const float Mn = fmaxf(M, m);
    const float fa = fast_exp2(M - Mn), fb = fast_exp2(m - Mn);
    L = L * fa + l * fb;
    o = o * fa + v * fb;
    M = Mn;
}

// One output row: its items' partial sums, eight groups of 32 lanes taking
// every eighth item, eight loads in flight each; merged in a fixed order.
constexpr int kRowGroups = kThreads / 32;
__device__ __forceinline__ void finish_row(const VerifyArgs& a, int gr, f32x4 (*red)[32], float2* gml) {
    const SeqTable& st = a.seq;
    const int bt = seq_of(st.row_start, st.n_seq, gr);
    const int b = a.sid[bt];
    const int R = st.qlen[bt] * a.group;
    const int local = gr - st.row_start[bt];
    const int c = local / R;
    const int row = local - c * R;
    const int nchunk = (st.ctx[bt] + a.chunk - 1) / a.chunk;
    const int item0 = st.item_start[bt] + c * nchunk;
    const int d4 = threadIdx.x & 31, sg = threadIdx.x >> 5;
    const f32x4* po = reinterpret_cast<const f32x4*>(a.part_o);
    float M = kEmpty, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = sg; s0 < nchunk; s0 += 8 * kRowGroups) {
        f32x4 v[8];
        float2 ml[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int s = s0 + u * kRowGroups;
            const size_t slot = (size_t)(item0 + min(s, nchunk - 1)) * kRowCap + row;
            v[u] = po[slot * (kHeadDim / 4) + d4];
            ml[u] = a.part_ml[slot];
            if (s >= nchunk) {
                v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                ml[u] = make_float2(kEmpty, 0.f);
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) mlo_merge(M, L, acc, ml[u].x, ml[u].y, v[u]);
    }
    red[sg][d4] = acc;
    if (d4 == 0) gml[sg] = make_float2(M, L);
    __syncthreads();
    if (sg != 0) return;
#pragma unroll
    for (int gq = 1; gq < kRowGroups; ++gq) mlo_merge(M, L, acc, gml[gq].x, gml[gq].y, red[gq][d4]);
    const f32x4 o = acc * (1.f / L) * kWhole;
    const int jl = row / a.group;
    const int h = c * a.group + (row - jl * a.group);
    const size_t base = (((size_t)b * a.max_q + a.qoff[bt] + jl) * a.n_q_heads + h) * kHeadDim + 4 * d4;
    if (a.out_fp32) {
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + base) = o;
    } else {
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + base) =
            make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
    }
}

// The scores' tile: the verify rows are the MFMA's A rows and the keys its
// columns, so lane (m16, G) gets key m16 (+16 for t = 1) of rows 16 rt + 4 G + i:
// the sum over rows is one of registers, then over the four lane groups.
struct ScoreLds {
    float2 ml[kWaves][kRowCap];
    __attribute__((aligned(16))) float lse[kRowCap];
    __attribute__((aligned(16))) int last_key[kRowCap];
    __attribute__((aligned(16))) char q[kRowCap * kQStride];
};

template <int NRT, bool kInt8, bool kPerHead>
__device__ __forceinline__ void score_item(const CodedVerifyArgs& ca, const Item& it, char* lds) {
    const VerifyArgs& a = ca.v;
    float2(*gml)[kRowCap] = reinterpret_cast<ScoreLds*>(lds)->ml;
    float* lse_row = reinterpret_cast<ScoreLds*>(lds)->lse;
    int* last_key = reinterpret_cast<ScoreLds*>(lds)->last_key;
    char* q_lds = reinterpret_cast<ScoreLds*>(lds)->q;   // (NRT * 16 rows of it)
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, G = lane >> 4;
    const int ntile = (it.key_end - it.key_begin + kTile - 1) / kTile;
    const int32_t* table = a.block_table + (size_t)it.b * a.max_blocks;
    const int all_see = it.T - it.qfull + it.qoff;
    // (per-head scores: the row of the group's first query head)
    float* srow = a.scores + (a.per_head ? ((size_t)it.b * a.n_q_heads + it.c * a.group) * a.max_ctx
                                         : (size_t)it.unit * a.max_ctx);
    f32x4 lse[NRT];
    // The rows' log-sum-exps from every item of this (sequence, KV head):
    // thread t merges row t % 64 over items t / 64, t / 64 + 4, ..., eight
    // loads in flight, the first of them before K's.  Infinity for rows whose
    // probabilities do not count.
    const int rr = threadIdx.x & (kRowCap - 1);
    const bool row_real = rr < it.nq * a.group;
    float2 ml[8];
    auto load_ml = [&](int s0) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int s2 = s0 + u * kWaves;
            ml[u] = make_float2(kEmpty, 0.f);
            if (row_real && s2 < it.nchunk) ml[u] = a.part_ml[(size_t)(it.item0 + s2) * kRowCap + rr];
        }
    };
    load_ml(wave);
    auto row_lse = [&] {
        float M = kEmpty, L = 0.f;
        for (int s0 = wave;;) {
            float Mn = M;
#pragma unroll
            for (int u = 0; u < 8; ++u) Mn = fmaxf(Mn, ml[u].x);
            L *= fast_exp2(M - Mn);
#pragma unroll
            for (int u = 0; u < 8; ++u) L += ml[u].y * fast_exp2(ml[u].x - Mn);
            M = Mn;
            s0 += 8 * kWaves;
            if (s0 >= it.nchunk) break;
            load_ml(s0);
        }
        gml[wave][rr] = make_float2(M, L);
        __syncthreads();
        if (threadIdx.x < kRowCap) {
            float Mx = kEmpty, Lx = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) ml_merge(Mx, Lx, gml[w][threadIdx.x].x, gml[w][threadIdx.x].y);
            const bool counts = it.qoff + (int)threadIdx.x / a.group >= it.qfull - min(a.window, it.qfull);
            lse_row[threadIdx.x] = Lx > 0.f && counts ? Mx + fast_log2(Lx) : INFINITY;
        }
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) lse[rt] = *reinterpret_cast<const f32x4*>(&lse_row[rt * 16 + 4 * G]);
    };
    auto tile_scores = [&](const KCodes& b, int key0, float ks) __attribute__((always_inline)) {
        const float scale = logit_scale(a.scale_log2, ks);
        const int place = q_place(m16, G);
        f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        // Both half tiles for each read of the rows; with three row tiles, which
        // spilled so, one after the other (us, two halves / one: 48 rows with scores
        // per query head 198 / 171, without 150 / 149; 64 rows 182 / 188).
        constexpr int kAtOnce = NRT == 3 ? 1 : 2;
#pragma unroll
        for (int t0 = 0; t0 < 2; t0 += kAtOnce) {
            u32x4 kd[kAtOnce][4];
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t) decode_k<kInt8>(b.k[t0 + t], kd[t]);
#pragma unroll
            for (int rt = 0; rt < NRT; ++rt) {
                u32x4 q[4];
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) q[kb] = q_operand(q_lds, place, rt, kb);
#pragma unroll
                for (int t = 0; t < kAtOnce; ++t) {
                    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kb = 0; kb < 4; ++kb) s = mfma_bf16(q[kb], kd[t][kb], s);
                    if (key0 + kTile - 1 > all_see) {   // wave-uniform: some row does not see some key
                        const int key = key0 + 16 * (t0 + t) + m16;
                        const int4 last = *reinterpret_cast<const int4*>(&last_key[rt * 16 + (place - m16 * kQStride) / 8]);
                        s[0] = key > last.x ? -INFINITY : s[0];
                        s[1] = key > last.y ? -INFINITY : s[1];
                        s[2] = key > last.z ? -INFINITY : s[2];
                        s[3] = key > last.w ? -INFINITY : s[3];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[t0 + t][i] += fast_exp2(__builtin_fmaf(s[i], scale, -lse[rt][i]));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (kPerHead) {
            // element i holds rows of head (4 G + i) mod group
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 v = sc[t];
                if (a.group <= 2) { v[0] += v[2]; v[1] += v[3]; }
                if (a.group == 1) v[0] += v[1];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (a.group <= 4) v[i] += shfl_xor_f(v[i], 16);
                    if (a.group <= 8) v[i] += shfl_xor_f(v[i], 32);
                }
                const int key = key0 + 16 * t + m16;
                if (key < it.key_end && 4 * G < a.group) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * G + i < a.group) {
                            float* at = srow + (size_t)(4 * G + i) * a.max_ctx + key;
                            *at = a.score_add ? *at + v[i] : v[i];
                        }
                }
            }
        } else {
            float v[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                v[t] = (sc[t][0] + sc[t][1]) + (sc[t][2] + sc[t][3]);
                v[t] += shfl_xor_f(v[t], 16);
                v[t] += shfl_xor_f(v[t], 32);
            }
            const int key = key0 + (lane & 31);
            const float val = G & 1 ? v[1] : v[0];
            if (lane < 32 && key < it.key_end) srow[key] = a.score_add ? srow[key] + val : val;
        }
    };
    u32x4 q[NRT];
    q_load<NRT>(a, it.b, it.c, it.nq, it.qoff, q);
    const TileRun run = tile_run(ca.c, table, a.n_kv_heads, it.c, a.page_size, it.key_begin, ntile, wave, lane, true);
    auto key_of = [&](int t) { return it.key_begin + (ntile - 1 - t) * kTile; };
    tile_pipeline<2, KCodes>(
        wave, ntile, kWaves,
        [&](KCodes& b, int t) __attribute__((always_inline)) {
            load_k_codes<false>(ca.c.k + tile_off(run, t), it.T - key_of(t), G, m16, b.k);
        },
        [&](const KCodes& b, int t) __attribute__((always_inline)) {
            tile_scores(b, key_of(t), lane_f(run.ks, (t - wave) / kWaves));
        },
        [&] {
            q_store<NRT>(q, q_lds);
            if (threadIdx.x < NRT * 16) last_key[threadIdx.x] = all_see + (int)threadIdx.x / a.group;
            row_lse();
        });
}

// kMost: row tiles of the call's largest item; each workgroup runs the body for
// its own sequence's.  A chunk is two workgroups, its later keys' first, and each
// goes from its last tile to its first: what the sweep read last is the likeliest
// to be in a cache still.  (us per call, one workgroup in order / two backwards: a
// ragged batch of 8 196 / 190, 4 x 64K keys and 48 rows 153 / 145, 120000 keys and
// 28 rows 71 / 66.)
constexpr int kParts = 2;
template <int kMost, bool kInt8, bool kPerHead>
__global__ __launch_bounds__(kThreads, kMost <= 3 ? 4 : 3) void coded_finish_kernel(CodedVerifyArgs ca) {
    constexpr size_t kLds = offsetof(ScoreLds, q) + kMost * 16 * kQStride;
    static_assert(kLds >= kRowGroups * (sizeof(float2) + 32 * sizeof(f32x4)), "finish_row's share");
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const int n_parts = kParts * ca.n_items;
    if ((int)blockIdx.x >= n_parts) {
        finish_row(ca.v, blockIdx.x - n_parts, reinterpret_cast<f32x4(*)[32]>(lds),
                   reinterpret_cast<float2*>(lds + kRowGroups * 32 * sizeof(f32x4)));
        return;
    }
    const int turn = (int)blockIdx.x >= ca.n_items ? 1 : 0;
    Item it = coded_item(ca.v, blockIdx.x - turn * ca.n_items);
    const int part = ca.v.chunk / kParts;
    it.key_begin += (kParts - 1 - turn) * part;
    it.key_end = min(it.key_begin + part, it.key_end);
    if (it.key_begin >= it.key_end) return;
    const int R = it.nq * ca.v.group;
    if (R <= 16) score_item<1, kInt8, kPerHead>(ca, it, lds);
    else if (kMost == 2 || R <= 32) score_item<kMost >= 2 ? 2 : 1, kInt8, kPerHead>(ca, it, lds);
    else if (kMost == 3 || R <= 48) score_item<kMost >= 3 ? 3 : 1, kInt8, kPerHead>(ca, it, lds);
    else score_item<kMost, kInt8, kPerHead>(ca, it, lds);
}

template <int NRT, bool kInt8>
hipError_t launch_nrt(const CodedVerifyArgs& a, int n_rows_total, hipStream_t stream) {
    hipLaunchKernelGGL((coded_sweep_kernel<NRT, kInt8>), dim3(a.n_items), dim3(kThreads), 0, stream, a);
    const dim3 grid(kParts * a.n_items + n_rows_total);
    if (a.v.per_head)
        hipLaunchKernelGGL((coded_finish_kernel<NRT, kInt8, true>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((coded_finish_kernel<NRT, kInt8, false>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool kInt8>
hipError_t launch_code(const CodedVerifyArgs& a, int n_rows_total, int row_tiles, hipStream_t stream) {
    switch (row_tiles) {
        case 1: return launch_nrt<1, kInt8>(a, n_rows_total, stream);
        case 2: return launch_nrt<2, kInt8>(a, n_rows_total, stream);
        case 3: return launch_nrt<3, kInt8>(a, n_rows_total, stream);
        default: return launch_nrt<4, kInt8>(a, n_rows_total, stream);
    }
}

}  // namespace

hipError_t launch_verify_coded(const CodedVerifyArgs& a, int n_rows_total, int row_tiles, hipStream_t stream) {
    // (a wave's tiles are in one TileRun)
    if (a.v.chunk > kPageRunTiles * kTile || a.v.chunk % (kParts * kTile) != 0) return hipErrorInvalidValue;
    return a.c.int8 ? launch_code<true>(a, n_rows_total, row_tiles, stream) : launch_code<false>(a, n_rows_total, row_tiles, stream);
}

}  // namespace ssl
