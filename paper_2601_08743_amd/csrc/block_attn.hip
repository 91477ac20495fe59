// Attention of single tokens over listed blocks of the paged cache, and the lists: blocks chosen by a cheap score.
//
// Score.  For a query row q of one head, qi = rint(q / 2^f) with f the smallest exponent that leaves |qi| <= 127, and a
// block's bounds hi, lo (step_ops.hip):  2^e 2^f sum_d (max(qi_d, 0) hi_d + min(qi_d, 0) lo_d), an upper bound, to the rounding
// of q, of what any key of the block scores; a block's score is the largest over the heads that share its KV head.
// The sum is one of integers below 2^24 and the rest are powers of two, so a score does not depend on who computes it in
// which order, and equal scores go to the lower block.
#include <algorithm>

#include "arrive.h"
#include "kv_append.h"
#include "step_ops.h"

namespace tc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// The blocks a token at `pos` may choose from: [first, w0); those before and the ones up to its own are always listed.
struct Window {
    int own, w0, first;
    __device__ __forceinline__ Window(int pos, int n_sink, int n_local) : own(pos >> 4), w0(max((pos >> 4) - (n_local - 1), 0)), first(min(w0, n_sink)) {}
    __device__ __forceinline__ int candidates() const { return w0 - first; }
};

// A token's request and position, or false for a padded row (and for one that names no place of the tables).
__device__ __forceinline__ bool token_place(const int32_t *token_seq, const int32_t *token_pos, int n, int B, int max_blocks, int &seq, int &pos)
{
    seq = token_seq[n];
    pos = token_pos[n];
    return seq >= 0 && seq < B && pos >= 0 && (pos >> 4) < max_blocks;
}

// ------------------------------------------------------------------------------------ scores
// i8 matrix instructions, 16 query rows x 16 blocks x 64: A the query rows as [max(qi, 0) | min(qi, 0)], B the bounds [hi | lo]
// of 16 blocks, straight from memory (a block's 2D bytes are whole lines).  Bound: reading the bounds, 1/16 of the cache's
// bytes in bf16.  A work-group takes one token and KV head and a range of its candidates, a wave 16 blocks at a time.
constexpr int kScoreBlocks = 256;                        // candidates of a work-group

template <bool kBf16, int kD>
__global__ __launch_bounds__(256) void score_kernel(Geom g, SelectArgs a)
{
    constexpr int kSteps = 2 * kD / 64;                  // matrix instructions along the 2D products
    const int item = blockIdx.x / a.score_parts, part = blockIdx.x - item * a.score_parts;
    const int n = a.n0 + item / g.Hkv, kvh = item % g.Hkv;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int j0 = win.first + part * kScoreBlocks;
    if (win.candidates() <= a.n_top || j0 >= win.w0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r16 = lane & 15, q4 = lane >> 4;
    const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks;
    const int8_t *bounds = a.digests + ((int64_t)a.layer * g.Hkv + kvh) * g.n_blocks * (2 * kD);
    const int8_t *exps = a.digests + a.exps_at + ((int64_t)a.layer * g.Hkv + kvh) * g.n_blocks;
    uint32_t *scores = a.scores + ((int64_t)(n - a.n0) * g.Hkv + kvh) * a.score_stride;
    float best[kScoreBlocks / 64];
#pragma unroll
    for (int i = 0; i < kScoreBlocks / 64; ++i) best[i] = -INFINITY;
    for (int row0 = 0; row0 < g.G; row0 += 16) {
        // lane (row r16, quarter q4) holds channels 16 q4 .. and 64 + 16 q4 .. (kD = 64: the first only) of its row
        const int row = min(row0 + r16, g.G - 1);
        const char *qr = a.q + ((int64_t)n * g.Hq + kvh * g.G + row) * g.head_bytes;
        float x[kSteps / 2][16];
        uint32_t size = 0;
#pragma unroll
        for (int s = 0; s < kSteps / 2; ++s)
#pragma unroll
            for (int c = 0; c < (kBf16 ? 2 : 4); ++c) {
                const uint4 v = *(const uint4 *)(qr + (64 * s + 16 * q4) * (kBf16 ? 2 : 4) + c * 16);
                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (kBf16) {
                        x[s][8 * c + 2 * k] = __uint_as_float(u[k] << 16);
                        x[s][8 * c + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
                    } else {
                        x[s][4 * c + k] = __uint_as_float(u[k]);
                    }
                }
            }
#pragma unroll
        for (int s = 0; s < kSteps / 2; ++s)
#pragma unroll
            for (int k = 0; k < 16; ++k) size = max(size, __float_as_uint(x[s][k]) & 0x7fffffffu);
        size = max(size, (uint32_t)__shfl_xor((int)size, 16));
        size = max(size, (uint32_t)__shfl_xor((int)size, 32));
        const bool finite = size < 0x7f800000u;
        const int f = finite ? step_exponent(__uint_as_float(size)) : 0;
        const float by = finite ? step_pow2(-f) : 0.f;
        i32x4 qa[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps / 2; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t plus = 0, minus = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = finite ? (int)rintf(x[s][4 * k + e] * by) : 0;
                    plus |= (uint32_t)max(i, 0) << (8 * e);
                    minus |= ((uint32_t)min(i, 0) & 0xffu) << (8 * e);
                }
                qa[s][k] = (int)plus;
                qa[kSteps / 2 + s][k] = (int)minus;
            }
        // rows 4 q4 + e of the products stand in this lane: their powers of two, and whether they count
        float scale[4];
        bool counts[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int src = 4 * q4 + e;
            scale[e] = step_pow2(__shfl(f, src));
            counts[e] = row0 + src < g.G && __shfl((int)finite, src) != 0;
        }
#pragma unroll
        for (int i = 0; i < kScoreBlocks / 64; ++i) {
            const int j = j0 + i * 64 + w * 16 + r16;
            if (j0 + i * 64 + w * 16 >= win.w0) break;
            const int32_t entry = j < win.w0 ? table[j] : -1;
            const int bid = entry >= 0 ? entry_bid(entry) : -1;
            const bool ok = bid >= a.first_block && bid < g.n_blocks;
            const i32x4 *src = (const i32x4 *)(bounds + (int64_t)(ok ? bid : a.first_block) * (2 * kD) + 16 * q4);
            i32x4 acc = {0, 0, 0, 0}, b[kSteps];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) b[s] = src[4 * s];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[s], b[s], acc, 0, 0, 0);
            float m = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (counts[e]) m = fmaxf(m, (float)acc[e] * scale[e]);
            best[i] = fmaxf(best[i], m);
        }
    }
#pragma unroll
    for (int i = 0; i < kScoreBlocks / 64; ++i) {
        const int j = j0 + i * 64 + w * 16 + r16;
        float m = best[i];
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        if (q4 != 0 || j >= win.w0) continue;
        const int32_t entry = table[j];
        const int bid = entry >= 0 ? entry_bid(entry) : -1;
        if (bid >= a.first_block && bid < g.n_blocks) {
            const int e = exps[bid];
            m = e == 127 ? INFINITY : m * step_pow2(e) + 0.f;       // (+ 0: the two zeros are equal)
        } else {
            m = -INFINITY;                               // no block: last of all
        }
        const uint32_t u = __float_as_uint(m);
        scores[j - win.first] = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    }
}

// ------------------------------------------------------------------------------------ lists
// The n_top best of a token's candidates and, behind ties, the lower ones; written in ascending order between the first
// blocks and the last.  A work-group per (token, KV head).  The n_top-th largest score is found by bins over the range that
// still holds it: a histogram of 1024 equal bins between its ends, the bin that the count falls into, and again inside that
// (at most four rounds; scores that are spread out take two).  A thread holds an odd number of neighbouring candidates, so that
// one prefix sum over the threads places them and LDS banks do not collide.
constexpr int kSelectBins = 1024, kSelectLds = 16384;    // candidates kept in LDS; more are read again from the scores

template <bool kLds>
__global__ __launch_bounds__(256) void select_kernel(Geom g, SelectArgs a)
{
    extern __shared__ uint32_t s_key[];
    __shared__ uint32_t s_bins[kSelectBins];
    __shared__ uint32_t s_wave[8], s_found[3];
    const int n = a.n0 + blockIdx.x / g.Hkv, kvh = blockIdx.x % g.Hkv;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int cand = win.candidates(), n_list = a.n_sink + a.n_top + a.n_local;
    int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * n_list;
    const int n_chosen = min(cand, a.n_top), n_all = win.first + n_chosen + (win.own - win.w0 + 1);
    for (int i = tid; i < n_list; i += 256)
        if (i < win.first) list[i] = i;
        else if (i >= n_all) list[i] = -1;
        else if (i >= win.first + n_chosen) list[i] = win.w0 + (i - win.first - n_chosen);
        else if (cand <= a.n_top) list[i] = i;
    if (cand <= a.n_top || a.n_top == 0) return;
    const uint32_t *scores = a.scores + ((int64_t)(n - a.n0) * g.Hkv + kvh) * a.score_stride;
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int i = tid; i < cand; i += 256) {
        const uint32_t k = scores[i];
        if (kLds) s_key[i] = k;
        lo = min(lo, k);
        hi = max(hi, k);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, m));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, m));
    }
    if (lane == 0) { s_wave[w] = lo; s_wave[4 + w] = hi; }
    __syncthreads();
    lo = min(min(s_wave[0], s_wave[1]), min(s_wave[2], s_wave[3]));
    hi = max(max(s_wave[4], s_wave[5]), max(s_wave[6], s_wave[7]));
    const uint32_t *keys = kLds ? s_key : scores;
    const int per = ((cand + 255) / 256) | 1, c0 = min(tid * per, cand), c1 = min(c0 + per, cand);
    // keys above `hi` are chosen; `want` of those in [lo, hi] are still to be found
    uint32_t want = a.n_top;
    while (lo < hi) {
        const uint32_t span = hi - lo;
        const int shift = max(0, 22 - (int)__builtin_clz(span));        // span >> shift < 1024
        for (int i = tid; i < kSelectBins; i += 256) s_bins[i] = 0;
        __syncthreads();
        for (int i = c0; i < c1; ++i) {
            const uint32_t k = keys[i];
            if (k >= lo && k <= hi) atomicAdd(&s_bins[(k - lo) >> shift], 1u);
        }
        __syncthreads();
        // counted from the top: thread t holds bins 1023 - 4t .. 1020 - 4t
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) { c[k] = s_bins[kSelectBins - 1 - 4 * tid - k]; sum += c[k]; }
        uint32_t x = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t y = (uint32_t)__shfl_up((int)x, d);
            if (lane >= d) x += y;
        }
        if (lane == 63) s_wave[w] = x;
        __syncthreads();
        uint32_t above = x - sum;
        for (int k = 0; k < w; ++k) above += s_wave[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (above < want && above + c[k] >= want) { s_found[0] = kSelectBins - 1 - 4 * tid - k; s_found[1] = above; s_found[2] = c[k]; }
            above += c[k];
        }
        __syncthreads();
        const uint32_t bin = s_found[0];
        const bool whole = want - s_found[1] == s_found[2];             // all of the bin: its lower end is the threshold
        want -= s_found[1];
        lo += bin << shift;
        hi = shift == 0 ? lo : min(hi, lo + ((1u << shift) - 1));
        if (whole) { want = 0xffffffffu; break; }
    }
    // chosen: keys above hi, and in [lo, hi] the first `want` (there lo == hi, or the whole range is)
    const uint32_t at = lo;
    uint64_t mine = 0;                                   // (keys at the threshold, keys above it)
    const bool whole = want == 0xffffffffu;
    for (int i = c0; i < c1; ++i) {
        const uint32_t k = keys[i];
        mine += (whole ? k >= at : k > at) ? 1u : (!whole && k == at) ? 1ull << 32 : 0;
    }
    uint64_t x = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t y = __shfl_up((unsigned long long)x, d);
        if (lane >= d) x += y;
    }
    __shared__ uint64_t s_sum[4];
    if (lane == 63) s_sum[w] = x;
    __syncthreads();
    uint64_t before = x - mine;
    for (int k = 0; k < w; ++k) before += s_sum[k];
    uint32_t above = (uint32_t)before, ties = (uint32_t)(before >> 32);
    for (int i = c0; i < c1; ++i) {
        const uint32_t k = keys[i];
        const bool over = whole ? k >= at : k > at, tie = !whole && k == at;
        if (over || (tie && ties < want)) list[win.first + above + min(ties, want)] = win.first + i;
        above += over;
        ties += tie;
    }
}

hipError_t launch_select(const Geom &g, SelectArgs a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    const int most = a.max_blocks;                       // candidates of any token
    a.score_parts = (most + kScoreBlocks - 1) / kScoreBlocks;
    const int64_t grid64 = (int64_t)a.n_tokens * g.Hkv * std::max(a.score_parts, 1);
    if (grid64 > INT32_MAX) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)grid64;
    if (most > a.n_top && a.n_top > 0) {
        if (g.esize == 2) TC_LAUNCH((score_kernel<true, 128>), grid, 0, L, g, a);
        else if (g.D == 64) TC_LAUNCH((score_kernel<false, 64>), grid, 0, L, g, a);
        else TC_LAUNCH((score_kernel<false, 128>), grid, 0, L, g, a);
    }
    static PerDeviceOnce configured;
    const hipError_t e = configured.run([] {
        return hipFuncSetAttribute((const void *)select_kernel<true>, hipFuncAttributeMaxDynamicSharedMemorySize, kSelectLds * 4);
    });
    if (e != hipSuccess) return e;
    if (most <= kSelectLds) TC_LAUNCH(select_kernel<true>, a.n_tokens * g.Hkv, most * 4, L, g, a);
    else TC_LAUNCH(select_kernel<false>, a.n_tokens * g.Hkv, 0, L, g, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ attention
// out = softmax(sm_scale q . k) v over the keys of the listed blocks at positions up to the token's own that hold a token;
// zeros where there are none.  A token and KV head have G rows that share a list, so as in the decode kernel the work is
// reading the listed keys and values once, and a short list is a chain of round trips.
//
// A work-group is (token, KV head, 16 rows, range of the list); its four waves take the range's units in turn, keep their own
// running maximum and sum, and are combined through LDS at the end.  K and V go straight from memory into the registers that
// the matrix instructions read: a wave's lists are short, 16 KB of loads are in flight from one unit, and no wave waits for
// another before the end.
struct ListUnit { int32_t j, entry; int valid; };

// Block `i` of the list: its logical number, its table entry and how many of its positions the token sees (0: none).
__device__ __forceinline__ ListUnit list_unit(const Geom &g, const BlockAttnArgs &a, const int32_t *list, const int32_t *table, int i, int end, int pos)
{
    ListUnit u{-1, -1, 0};
    if (i < end) u.j = list[i];
    if (u.j >= 0 && u.j <= pos >> 4) u.entry = table[u.j];
    const int bid = entry_bid(u.entry);
    if (u.entry >= 0 && bid >= a.first_block && bid < g.n_blocks) u.valid = min(kBlockTokens - entry_pad(u.entry), pos - u.j * kBlockTokens + 1);
    return u;
}

// bf16, heads of 128.  A unit is two blocks, 32 keys, against 16 query rows: S^T = K Q^T by 16x16x32 matrix instructions whose
// 16 keys are tokens 0..7 of both blocks, then 8..15, so that a lane's eight scores (quarter q4 of the wave: block q4 / 2,
// half q4 % 2) belong to the eight tokens whose values stand in one 16-byte piece of the pool's V rows, and O^T += V^T P^T
// takes both as they are.  Weights are rounded to bf16 for that product (as in every attention kernel here; their sum is of
// the fp32 ones).  Values at positions that the token does not see are replaced by zeros, whatever stands there.
constexpr int kBaRow = 132;

template <bool kSplit>
__global__ __launch_bounds__(256, 2) void block_attn_bf16_kernel(Geom g, BlockAttnArgs a)
{
    __shared__ __attribute__((aligned(16))) float s_o[4][16 * kBaRow];
    __shared__ float s_ml[4][16][2];
    const int chunks = (g.G + 15) >> 4;
    const int item = blockIdx.x / a.n_splits, split = blockIdx.x - item * a.n_splits;
    const int n = item / (g.Hkv * chunks), hc = item - n * (g.Hkv * chunks), kvh = hc / chunks, row0 = (hc - kvh * chunks) * 16;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q4 = lane >> 4;
    const int rows = min(16, g.G - row0);
    const int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * a.n_list;
    const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks;
    const int n_units = (a.n_list + 1) >> 1;
    const int u0 = (int)((int64_t)n_units * split / a.n_splits), u1 = (int)((int64_t)n_units * (split + 1) / a.n_splits);
    const int end = min(2 * u1, a.n_list);
    const char *pool = g.pool + (int64_t)a.layer * g.layer_stride + (int64_t)kvh * (kBlockTokens * 256);
    const int64_t v_half = g.block_bytes >> 1;

    bf16x8 qf[4];
    {
        const char *qr = a.q + ((int64_t)n * g.Hq + kvh * g.G + row0 + min(r16, rows - 1)) * 256 + q4 * 16;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qf[ks] = *(const bf16x8 *)(qr + ks * 64);
    }
    f32x4 o[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_lane = 0.f;

    const uint32_t k_off = (uint32_t)(r16 & 7) * 256 + q4 * 16, v_off = (uint32_t)r16 * 32 + (q4 & 1) * 16;
    // a wave's units 32 at a time: lane 2k + b looks up block b of unit k
    for (int k0 = u0 + w; k0 < u1; k0 += 4 * 32) {
        const ListUnit mine = list_unit(g, a, list, table, 2 * (k0 + 4 * (lane >> 1)) + (lane & 1), end, pos);
        const int n_mine = min(32, (u1 - k0 + 3) >> 2);
        bf16x8 kf[8], vf[8];
        int valid0 = 0, valid1 = 0;
        auto fetch = [&](int k, int &v0, int &v1) {      // a unit whose blocks are both empty loads nothing
            v0 = __builtin_amdgcn_readlane(mine.valid, 2 * k);
            v1 = __builtin_amdgcn_readlane(mine.valid, 2 * k + 1);
            if (v0 <= 0 && v1 <= 0) return;
            int b0 = entry_bid(__builtin_amdgcn_readlane(mine.entry, 2 * k)), b1 = entry_bid(__builtin_amdgcn_readlane(mine.entry, 2 * k + 1));
            if (v0 <= 0) b0 = b1;                        // (what is loaded in an empty block's place is masked)
            if (v1 <= 0) b1 = b0;
            const char *p0 = pool + (int64_t)b0 * g.block_bytes, *p1 = pool + (int64_t)b1 * g.block_bytes;
            const char *kp = (r16 < 8 ? p0 : p1) + k_off, *vp = (q4 < 2 ? p0 : p1) + v_half + v_off;
#pragma unroll
            for (int i = 0; i < 8; ++i) kf[i] = *(const bf16x8 *)(kp + (i >> 2) * 2048 + (i & 3) * 64);
#pragma unroll
            for (int i = 0; i < 8; ++i) vf[i] = *(const bf16x8 *)(vp + i * 512);
        };
        for (int k = 0; k < n_mine; ++k) {
            fetch(k, valid0, valid1);
            if (valid0 <= 0 && valid1 <= 0) continue;
            f32x4 s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[4 * h + ks], qf[ks], s[h], 0, 0, 0);
            }
            if (valid0 < kBlockTokens || valid1 < kBlockTokens) {
                const int seen = (q4 < 2 ? valid0 : valid1) - 4 * (q4 & 1);      // of this lane's tokens 0..3 and 8..11
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool sees = 8 * h + e < seen;
                        s[h][e] = sees ? s[h][e] : -INFINITY;
#pragma unroll
                        for (int i = 0; i < 8; ++i) vf[i][4 * h + e] = sees ? vf[i][4 * h + e] : (__bf16)0.f;
                    }
            }
            float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run, mx * a.scale_log2);
            if (__any(m_new > m_run)) {
                const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
                l_lane *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[db][e] *= alpha;
                m_run = m_new;
            }
            const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
            bf16x8 pf;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[h][e], a.scale_log2, neg_m));
                    l_lane += p;
                    pf[4 * h + e] = (__bf16)p;
                }
#pragma unroll
            for (int db = 0; db < 8; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[db], pf, o[db], 0, 0, 0);
        }
    }

    // the waves' (maximum, sum, output) rows, combined by 16 threads a row, eight columns each
    float l_row = l_lane + __shfl_xor(l_lane, 16);
    l_row += __shfl_xor(l_row, 32);
#pragma unroll
    for (int db = 0; db < 8; ++db) *(f32x4 *)&s_o[w][r16 * kBaRow + 16 * db + 4 * q4] = o[db];
    if (q4 == 0) { s_ml[w][r16][0] = m_run; s_ml[w][r16][1] = l_row; }
    __syncthreads();
    const int row = tid >> 4, d = 8 * (tid & 15);
    if (row >= rows) return;
    float M = -INFINITY, sum = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, s_ml[k][row][0]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float mk = s_ml[k][row][0];
        // (no maximum: no keys - its sums are zeros - or only scores that are NaN, and so are they)
        const float wgt = mk == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mk - M);
        sum += wgt * s_ml[k][row][1];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += wgt * s_o[k][row * kBaRow + d + e];
    }
    const int64_t out_row = (int64_t)n * g.Hq + kvh * g.G + row0 + row;
    if (kSplit) {
        float *po = a.part_o + (out_row * a.n_splits + split) * 128 + d;
        *(f32x4 *)po = f32x4{acc[0], acc[1], acc[2], acc[3]};
        *(f32x4 *)(po + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
        if (d == 0) *(float2 *)(a.part_ml + (out_row * a.n_splits + split) * 2) = make_float2(M, sum);
    } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (__bf16)(acc[e] * inv);
        *(bf16x8 *)(a.out + out_row * 256 + d * 2) = y;
    }
}

// fp32, heads of 64 or 128: a unit is one block.  A key row is four channels for each of kD / 4 lanes, so a wave scores
// 64 / (kD / 4) keys at a time, for up to eight rows, and each of its lane groups keeps a maximum and a sum of its own.
template <int kD, bool kSplit>
__global__ __launch_bounds__(256, 2) void block_attn_f32_kernel(Geom g, BlockAttnArgs a)
{
    constexpr int kLanes = kD / 4, kGroups = 64 / kLanes, kSteps = kBlockTokens / kGroups, kRows = 8, kParts = 4 * kGroups;
    __shared__ __attribute__((aligned(16))) float s_o[kParts][kRows][kD];
    __shared__ float s_ml[kParts][kRows][2];
    const int chunks = (g.G + kRows - 1) / kRows;
    const int item = blockIdx.x / a.n_splits, split = blockIdx.x - item * a.n_splits;
    const int n = item / (g.Hkv * chunks), hc = item - n * (g.Hkv * chunks), kvh = hc / chunks, row0 = (hc - kvh * chunks) * kRows;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane % kLanes, grp = lane / kLanes;
    const int rows = min(kRows, g.G - row0);
    const int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * a.n_list;
    const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks;
    const int u0 = (int)((int64_t)a.n_list * split / a.n_splits), u1 = (int)((int64_t)a.n_list * (split + 1) / a.n_splits);
    const char *pool = g.pool + (int64_t)a.layer * g.layer_stride + (int64_t)kvh * (kBlockTokens * kD * 4) + c * 16;
    const int64_t v_half = g.block_bytes >> 1;
    f32x4 qf[kRows], o[kRows];
    float m_run[kRows], l_run[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        qf[r] = *(const f32x4 *)(a.q + ((int64_t)n * g.Hq + kvh * g.G + row0 + min(r, rows - 1)) * (kD * 4) + c * 16);
        o[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[r] = -INFINITY;
        l_run[r] = 0.f;
    }
    for (int k0 = u0 + w; k0 < u1; k0 += 4 * 64) {
        const ListUnit mine = list_unit(g, a, list, table, k0 + 4 * lane, u1, pos);
        const int n_mine = min(64, (u1 - k0 + 3) >> 2);
        for (int k = 0; k < n_mine; ++k) {
            const int valid = __builtin_amdgcn_readlane(mine.valid, k);
            if (valid <= 0) continue;
            const char *p = pool + (int64_t)entry_bid(__builtin_amdgcn_readlane(mine.entry, k)) * g.block_bytes;
            f32x4 kf[kSteps], vf[kSteps];
#pragma unroll
            for (int t = 0; t < kSteps; ++t) kf[t] = *(const f32x4 *)(p + (t * kGroups + grp) * (kD * 4));
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                vf[t] = *(const f32x4 *)(p + v_half + (t * kGroups + grp) * (kD * 4));
                if (t * kGroups + grp >= valid) vf[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (r >= rows) break;
                float s[kSteps], mx = -INFINITY;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const f32x4 x = kf[t] * qf[r];
                    float y = (x[0] + x[1]) + (x[2] + x[3]);
                    y = kLanes == 32 ? sum32(y) : sum16(y);
                    s[t] = t * kGroups + grp < valid ? y * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, s[t]);
                }
                const float m_new = fmaxf(m_run[r], mx);
                const float alpha = m_run[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[r] - m_new);
                const float base = m_new == -INFINITY ? 0.f : m_new;
                float l = l_run[r] * alpha;
                f32x4 acc = o[r] * alpha;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const float e = __builtin_amdgcn_exp2f(s[t] - base);
                    l += e;
                    acc += e * vf[t];
                }
                m_run[r] = m_new;
                l_run[r] = l;
                o[r] = acc;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        *(f32x4 *)&s_o[w * kGroups + grp][r][4 * c] = o[r];
        if (c == 0) { s_ml[w * kGroups + grp][r][0] = m_run[r]; s_ml[w * kGroups + grp][r][1] = l_run[r]; }
    }
    __syncthreads();
    constexpr int kThreadsRow = kD / 4;
    for (int row = tid / kThreadsRow; row < rows; row += 256 / kThreadsRow) {
        const int d = 4 * (tid % kThreadsRow);
        RowSum x{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < kParts; ++k) x.add(s_ml[k][row][0], s_ml[k][row][1], *(const f32x4 *)&s_o[k][row][d]);
        const int64_t out_row = (int64_t)n * g.Hq + kvh * g.G + row0 + row;
        if (kSplit) {
            *(f32x4 *)(a.part_o + (out_row * a.n_splits + split) * kD + d) = x.acc;
            if (d == 0) *(float2 *)(a.part_ml + (out_row * a.n_splits + split) * 2) = make_float2(x.M, x.L);
        } else {
            *(f32x4 *)(a.out + (out_row * kD + d) * 4) = x.acc * (x.L == 0.f ? 0.f : 1.f / x.L);
        }
    }
}

// Ranges of a list combined: kD / 4 threads a row.
template <bool kBf16, int kD>
__global__ __launch_bounds__(256) void block_merge_kernel(Geom g, BlockAttnArgs a)
{
    constexpr int kThreadsRow = kD / 4;
    const int64_t row = (int64_t)blockIdx.x * (256 / kThreadsRow) + threadIdx.x / kThreadsRow;
    const int d = 4 * (threadIdx.x % kThreadsRow);
    if (row >= (int64_t)a.n_tokens * g.Hq) return;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, (int)(row / g.Hq), a.B, a.max_blocks, seq, pos)) return;
    RowSum x{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    for (int s = 0; s < a.n_splits; ++s) {
        const float2 ml = *(const float2 *)(a.part_ml + (row * a.n_splits + s) * 2);
        x.add(ml.x, ml.y, *(const f32x4 *)(a.part_o + (row * a.n_splits + s) * kD + d));
    }
    const float inv = x.L == 0.f ? 0.f : 1.f / x.L;
    if (kBf16) {
        unsigned short r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __builtin_bit_cast(unsigned short, (__bf16)(x.acc[e] * inv));
        *(uint2 *)(a.out + (row * kD + d) * 2) = make_uint2(r[0] | ((uint32_t)r[1] << 16), r[2] | ((uint32_t)r[3] << 16));
    } else {
        *(f32x4 *)(a.out + (row * kD + d) * 4) = x.acc * inv;
    }
}

// As many ranges as give the chip about two work-groups a CU, none shorter than four units (one for each wave).
int block_attn_splits(int Hq, int Hkv, int esize, int n_tokens, int n_list)
{
    const int G = Hq / Hkv, rows = esize == 2 ? 16 : 8;
    const int64_t items = (int64_t)n_tokens * Hkv * ((G + rows - 1) / rows);
    const int units = esize == 2 ? (n_list + 1) / 2 : n_list;
    const int64_t want = items > 0 ? 512 / items : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, (units + 3) / 4), 32));
}

hipError_t launch_block_attn(const Geom &g, const BlockAttnArgs &a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    const int rows = g.esize == 2 ? 16 : 8, chunks = (g.G + rows - 1) / rows;
    const int64_t grid = (int64_t)a.n_tokens * g.Hkv * chunks * a.n_splits;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    const bool split = a.n_splits > 1;
    if (g.esize == 2) {
        if (split) TC_LAUNCH(block_attn_bf16_kernel<true>, (unsigned)grid, 0, L, g, a);
        else TC_LAUNCH(block_attn_bf16_kernel<false>, (unsigned)grid, 0, L, g, a);
    } else if (g.D == 64) {
        if (split) TC_LAUNCH((block_attn_f32_kernel<64, true>), (unsigned)grid, 0, L, g, a);
        else TC_LAUNCH((block_attn_f32_kernel<64, false>), (unsigned)grid, 0, L, g, a);
    } else {
        if (split) TC_LAUNCH((block_attn_f32_kernel<128, true>), (unsigned)grid, 0, L, g, a);
        else TC_LAUNCH((block_attn_f32_kernel<128, false>), (unsigned)grid, 0, L, g, a);
    }
    return hipGetLastError();
}

hipError_t launch_block_merge(const Geom &g, const BlockAttnArgs &a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    const int64_t rows = (int64_t)a.n_tokens * g.Hq, per = 256 / (g.D / 4), blocks = (rows + per - 1) / per;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    if (g.esize == 2) TC_LAUNCH((block_merge_kernel<true, 128>), (unsigned)blocks, 0, L, g, a);
    else if (g.D == 64) TC_LAUNCH((block_merge_kernel<false, 64>), (unsigned)blocks, 0, L, g, a);
    else TC_LAUNCH((block_merge_kernel<false, 128>), (unsigned)blocks, 0, L, g, a);
    return hipGetLastError();
}

}  // namespace tc
