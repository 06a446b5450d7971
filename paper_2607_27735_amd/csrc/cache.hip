// cache.hip -- filling the 8-bit paged KV cache: the pages and slots of a
// step's tokens, and the append that codes their K and V rows.
#include <algorithm>

#include "coded_common.h"

namespace ssl {
namespace {

using cc::u32x2;

// ---------------------------------------------------------------------------
// Pages and slots from the request lengths.
//
// need_b = ceil((ctx_b + new_b) / page) - ceil(ctx_b / page); the inclusive
// prefix sums of need and new say which free pages a sequence takes, where its
// tokens stand in the flattened step, and whether both fit.  Every workgroup
// forms the sums for itself (at most kMapBatch sequences), which saves the
// kernel boundary or the exchange that sharing them would take, and then writes
// its part of the slots and of the new table entries.  Bound by the launch and
// three dependent loads (lengths, table, slots): 4.1 to 4.9 us per call back to
// back for 16 sequences of 2 to 8 tokens (an empty kernel takes 3.9; the kernel
// alone 2.9), 4.6 to 5.3 for 64 sequences and 315000 tokens (5.1).
// ---------------------------------------------------------------------------
// (Slots per workgroup, the kernel alone for 64 sequences and 315000 tokens: 2048
// 9.2 us, 1024 6.4, 512 and 256 5.1.)
constexpr int kMapThreads = 256;
constexpr int kMapTokens = 512;    // slots per workgroup
constexpr int kMapFar = 1 << 30;   // sums saturate here; no capacity reaches it

__device__ __forceinline__ int sat_add(int x, int y) { return (int)min((uint32_t)x + (uint32_t)y, (uint32_t)kMapFar); }

// Inclusive saturating prefix sum over the wave (wave_incl_scan's moves).
__device__ __forceinline__ int sat_scan(int x) {
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return x;
}

// The first b with x < upto[b], of n ascending values.
__device__ __forceinline__ int find(const int* upto, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (x < upto[mid]) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// kPer: sequences per thread.
template <int kPer>
__global__ __launch_bounds__(kMapThreads) void page_map_kernel(PageMapArgs a) {
    constexpr int kBatch = kPer * kMapThreads;
    __shared__ int rows[kBatch], pages[kBatch], ctx[kBatch], held[kBatch];
    __shared__ int2 wsum[kMapThreads / kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // Thread t has sequences kPer t ...
    int c[kPer], n[kPer], need[kPer], have[kPer], sn = 0, sp = 0;
    bool ok[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = kPer * tid + i;
        c[i] = b < a.batch ? a.ctx_len[b] : 0;
        n[i] = b < a.batch ? a.new_len[b] : 0;
    }
    // (the range is the device's word: pages that it claims past the list are not there)
    const int first = a.free_range[0], end = a.free_range[1];
    const int last = min(end, a.n_free);
    const int avail = first >= 0 && first < last ? min(last - first, kMapFar - 1) : 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int64_t total = (int64_t)c[i] + n[i];
        ok[i] = c[i] >= 0 && n[i] >= 0 && total <= (int64_t)a.page_size * a.max_blocks;
        n[i] = min(max(n[i], 0), kMapFar);
        // (up to 2^31 - 1, so the roundings up fit 32 bits unsigned)
        have[i] = ok[i] ? (int)(((uint32_t)c[i] + a.page_size - 1) / (uint32_t)a.page_size) : 0;
        need[i] = ok[i] ? (int)(((uint32_t)total + a.page_size - 1) / (uint32_t)a.page_size) - have[i] : 0;
        sn = sat_add(sn, n[i]);
        sp = sat_add(sp, need[i]);
    }
    const int in = sat_scan(sn), ip = sat_scan(sp);
    if (lane == kWave - 1) wsum[wave] = make_int2(in, ip);
    // what stands before the thread's first sequence
    int at = __shfl_up(in, 1, kWave), ap = __shfl_up(ip, 1, kWave);
    if (lane == 0) at = ap = 0;
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        at = sat_add(at, wsum[w].x);
        ap = sat_add(ap, wsum[w].y);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = kPer * tid + i;
        at = sat_add(at, n[i]);
        ap = sat_add(ap, need[i]);
        const bool served = ok[i] && (need[i] == 0 || ap <= avail) && at <= a.max_tokens;
        rows[b] = at;
        pages[b] = ap;
        ctx[b] = c[i];
        held[b] = served ? have[i] : -1;   // pages before the step, -1: not served
    }
    __syncthreads();
    const int total_rows = rows[a.batch - 1], total_pages = pages[a.batch - 1];

    for (int64_t y = (int64_t)blockIdx.x * kMapThreads + tid; y < min(total_pages, avail); y += gridDim.x * kMapThreads) {
        const int x = (int)y;
        const int b = find(pages, a.batch, x);
        const int before = b ? pages[b - 1] : 0;
        if (held[b] >= 0) a.block_table[(size_t)b * a.max_blocks + held[b] + x - before] = a.free_pages[first + x];
    }
    // Slots: a page that is new in this step is read from the free list (its
    // table entry may be another workgroup's to write).
    for (int64_t x = (int64_t)blockIdx.x * kMapTokens; x < a.max_tokens; x += (int64_t)gridDim.x * kMapTokens) {
#pragma unroll
        for (int i = 0; i < kMapTokens / kMapThreads; ++i) {
            const int t = (int)x + i * kMapThreads + tid;
            if (t >= a.max_tokens) continue;
            int slot = -1;
            if (t < total_rows) {
                const int b = find(rows, a.batch, t);
                if (held[b] >= 0) {
                    const int pos = ctx[b] + t - (b ? rows[b - 1] : 0);
                    const int blk = pos / a.page_size, fresh = blk - held[b];
                    const int page = fresh >= 0 ? a.free_pages[first + (b ? pages[b - 1] : 0) + fresh]
                                                : a.block_table[(size_t)b * a.max_blocks + blk];
                    slot = (int)((uint32_t)page * (uint32_t)a.page_size + (uint32_t)(pos - blk * a.page_size));   // (any page id)
                }
            }
            a.slot_map[t] = slot;
        }
    }
    if (blockIdx.x == 0) {
        // pages taken: the served sequences that need any are a leading run
        int taken = 0;
        for (int b = tid; b < a.batch; b += kMapThreads) {
            const int before = b ? pages[b - 1] : 0, nb = rows[b] - (b ? rows[b - 1] : 0);
            a.total_len[b] = ctx[b] + (held[b] >= 0 ? nb : 0);
            a.row_start[b + 1] = rows[b];
            if (held[b] >= 0 && pages[b] > before) taken = max(taken, pages[b]);
        }
        for (int o = 32; o; o >>= 1) taken = max(taken, __shfl_xor(taken, o, kWave));
        __syncthreads();
        if (lane == 0) wsum[wave].x = taken;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kMapThreads / kWave; ++w) taken = max(taken, wsum[w].x);
            a.row_start[0] = 0;
            a.free_range_out[0] = first + taken;
            a.free_range_out[1] = end;
        }
    }
}

// ---------------------------------------------------------------------------
// Append.
//
// Per scale block and KV head, for K and for V: need = the smallest power of
// two s >= 2^-126 with max |x| <= top s over the new rows; s = need where the
// block starts with a new row, else max(need, the block's scale), its older
// rows coded again by s_old / s where that is not 1; new codes = rn(x / s).
// A power of two makes x / s exact, so a code is rounded once, and a re-coded
// one once more.
//
// A wave codes the new rows of one block and head: they stay in its registers
// between the maximum and the codes, so K and V are read once, with no LDS.
// Bound by those reads and writes, 2 + 1 bytes per element: 73635 tokens of 8
// heads, 453 MB, take 92.4 us (4.90 TB/s; a copy on the device reaches 5.14), 64
// sequences of 2 to 8 tokens 5.3 us, one of 7 3.9 to 4.6, the launch.
// ---------------------------------------------------------------------------
constexpr int kAppendWaves = 4;
constexpr int kAppendThreads = kAppendWaves * kWave;

constexpr float kBf16Max = 3.38953139e38f;

// The scale for a largest magnitude m >= 0: top = 1.75 * 2^8 (e4m3) or 127/64 * 2^6 (int8).
template <bool kInt8>
__device__ __forceinline__ float scale_for(float m) {
    const uint32_t bits = __float_as_uint(fminf(m, kBf16Max));
    const int x = (int)(bits >> 23) - (kInt8 ? 6 : 8) + ((bits & 0x7FFFFFu) > (kInt8 ? 0x7E0000u : 0x600000u) ? 1 : 0);
    return __uint_as_float((uint32_t)max(x, 1) << 23);
}

// Four values, already divided by the scale, as codes.
template <bool kInt8>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    if constexpr (kInt8) {
        auto code = [](float x) { return (uint32_t)(int)__builtin_rintf(x) & 0xFFu; };
        return code(a) | code(b) << 8 | code(c) << 16 | code(d) << 24;
    } else {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
    }
}

// x * inv, infinities taken as the largest bf16 and NaN as 0: within the codes'
// range, as the scale is at least scale_for(|x|).
__device__ __forceinline__ float scaled(float x, float inv) {
    const float y = fminf(fmaxf(x, -kBf16Max), kBf16Max) * inv;
    return x == x ? y : 0.f;
}

// Four codes times a factor, coded again.
template <bool kInt8>
__device__ __forceinline__ uint32_t recode4(uint32_t w, float f) {
    if constexpr (kInt8) {
        return encode4<true>((float)(int8_t)w * f, (float)(int8_t)(w >> 8) * f, (float)(int8_t)(w >> 16) * f,
                             (float)(int8_t)(w >> 24) * f);
    } else {
        const f32x2 lo = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false));
        const f32x2 hi = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true));
        return encode4<false>(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
    }
}

// kRows: rows of a scale block.  Workgroup x looks at tokens window * x ..; a
// token leads a run when it is its block's first in the step; wave w of
// workgroup (x, y) codes the runs led there for unit 4 y + w = 2 * head + (1
// for V).  A call of few tokens has a window of 1, so that every block has
// waves of its own; in a long one most tokens lead nothing, and windows of 16
// keep the workgroups that find nothing few.
template <int kRows, bool kInt8>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(AppendArgs a) {
    const int lane = threadIdx.x & 63;
    const int unit = blockIdx.y * kAppendWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= 2 * a.n_kv_heads) return;
    const int head = unit >> 1;
    const uint16_t* src = (unit & 1 ? a.v_new : a.k_new) + (size_t)head * kHeadDim;
    const int64_t stride = unit & 1 ? a.v_stride : a.k_stride;
    uint8_t* codes = unit & 1 ? a.v : a.k;
    float* scales = unit & 1 ? a.v_scale : a.k_scale;
    const int m16 = lane & 15, G = lane >> 4;

    // One load has the slots from before the window on: lane l that of token
    // t0 - 1 + l.  A run is found there as far as it reaches, and the rest of a
    // long one with another load.
    auto slot_at = [&](int t) { return t >= 0 && t < a.n_tokens ? a.slot_map[t] : -1; };
    auto usable = [&](int s) { return s >= 0 && s < a.n_slots; };
    const int t0 = blockIdx.x * a.window;
    const int s_here = slot_at(t0 - 1 + lane), s_before = __shfl_up(s_here, 1, kWave);
    const bool lead = lane >= 1 && lane <= a.window && usable(s_here) &&
                      (!usable(s_before) || s_here != s_before + 1 || s_here % kRows == 0);
    for (uint64_t todo = __ballot(lead); todo; todo &= todo - 1) {
        const int l0 = __builtin_ctzll(todo), t = t0 - 1 + l0;
        const int slot = __builtin_amdgcn_readlane(s_here, l0);
        const int old = slot % kRows;            // rows that the block holds before the run
        const int room = kRows - old;
        int n;                                   // rows of the run
        {
            const uint64_t m = __ballot((uint32_t)s_here == (uint32_t)slot + lane - l0 && usable(s_here)) >> l0;   // bit i: row i
            n = m == ~0ull ? kWave : __builtin_ctzll(~m);
        }
#pragma unroll 1
        for (int have = kWave - l0; n == have && n < room; have += kWave) {
            const int s = slot_at(t + have + lane);
            const uint64_t m = __ballot((uint32_t)s == (uint32_t)slot + have + lane && usable(s));
            n += m == ~0ull ? kWave : __builtin_ctzll(~m);
        }
        n = min(n, room);
        const int page = slot / a.page_size, o = slot - page * a.page_size;
        const size_t row0 = ((size_t)page * a.n_kv_heads + head) * a.page_size + o;
        float* scale = scales + ((size_t)page * a.n_kv_heads + head) * (a.page_size / kRows) + o / kRows;
        const float was = old ? *scale : 0.f;

        u32x4 x[kRows / 4];
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
            x[i] = u32x4{0u, 0u, 0u, 0u};
            if (4 * i + G < n) x[i] = ld_u32x4(src + (int64_t)(t + 4 * i + G) * stride + 8 * m16);
        }
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
            if (4 * i < n) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    mx = fmaxf(mx, fmaxf(fabsf(bf16_lo(x[i][d])), fabsf(bf16_hi(x[i][d]))));
            }
        }
        for (int m = 32; m; m >>= 1) mx = fmaxf(mx, shfl_xor_f(mx, m));
        const float s = fmaxf(scale_for<kInt8>(mx), was);
        if (old && s != was) {   // the older rows, eight at a time: 16 codes per lane
            const float f = was / s;
            for (int r = lane >> 3; r < old; r += 8) {
                u32x4* p = reinterpret_cast<u32x4*>(codes + (row0 - old + r) * kHeadDim + 16 * (lane & 7));
                u32x4 w = *p;
#pragma unroll
                for (int d = 0; d < 4; ++d) w[d] = recode4<kInt8>(w[d], f);
                *p = w;
            }
        }
        const float inv = 1.f / s;
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
            if (4 * i + G < n) {
                u32x2 w;
#pragma unroll
                for (int d = 0; d < 2; ++d)
                    w[d] = encode4<kInt8>(scaled(bf16_lo(x[i][2 * d]), inv), scaled(bf16_hi(x[i][2 * d]), inv),
                                          scaled(bf16_lo(x[i][2 * d + 1]), inv), scaled(bf16_hi(x[i][2 * d + 1]), inv));
                *reinterpret_cast<u32x2*>(codes + (row0 + 4 * i + G) * kHeadDim + 8 * m16) = w;
            }
        }
        if (lane == 0 && s != was) *scale = s;
    }
}

template <int kRows>
void launch_append(const AppendArgs& a, dim3 grid, hipStream_t stream) {
    if (a.int8)
        hipLaunchKernelGGL((cache_append_kernel<kRows, true>), grid, dim3(kAppendThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((cache_append_kernel<kRows, false>), grid, dim3(kAppendThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream) {
    const int64_t most = std::max<int64_t>(a.max_tokens, 1);
    const int blocks = (int)std::min<int64_t>(1024, (most + kMapTokens - 1) / kMapTokens);
    if (a.batch <= kMapThreads)
        hipLaunchKernelGGL((page_map_kernel<1>), dim3(blocks), dim3(kMapThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((page_map_kernel<kMapBatch / kMapThreads>), dim3(blocks), dim3(kMapThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_cache_append(const AppendArgs& args, int scale_block, hipStream_t stream) {
    AppendArgs a = args;
    const int y = (2 * a.n_kv_heads + kAppendWaves - 1) / kAppendWaves;
    a.window = (int64_t)a.n_tokens * y <= 8192 ? 1 : 16;
    const dim3 grid((a.n_tokens + a.window - 1) / a.window, y);
    if (scale_block == 32) launch_append<32>(a, grid, stream);
    else if (scale_block == 64) launch_append<64>(a, grid, stream);
    else launch_append<128>(a, grid, stream);
    return hipGetLastError();
}

}  // namespace ssl
