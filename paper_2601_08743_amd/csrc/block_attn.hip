// Attention of single tokens over listed blocks of the paged cache, and the lists: blocks chosen by a cheap score.
//
// Score.  For a query row q of one head, qi = rint(q / 2^f) with f the smallest exponent that leaves |qi| <= 127, and a
// block's bounds hi, lo (step_ops.hip):  2^e 2^f sum_d (max(qi_d, 0) hi_d + min(qi_d, 0) lo_d), an upper bound, to the rounding
// of q, of what any key of the block scores; a block's score is the largest over the heads that share its KV head.
// The sum is one of integers below 2^24 and the rest are powers of two, so a score does not depend on who computes it in
// which order, and equal scores go to the lower block.
#include <algorithm>

#include "arrive.h"
#include "lds_dma.h"
#include "score_route.h"
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

// Over lanes 32 apart, and 16 as well where kApart is 16, by exchanging rows of a wave (a shuffle through LDS takes ten times as
// long).
template <int kApart, typename F>
__device__ __forceinline__ float over_lanes(float x, F op)
{
    unsigned u = __float_as_uint(x);
    if (kApart == 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const unsigned p = a[0], q = a[1];
        u = __float_as_uint(op(__uint_as_float(p), __uint_as_float(q)));
    }
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned p = b[0], q = b[1];
    return op(__uint_as_float(p), __uint_as_float(q));
}
template <int kApart> __device__ __forceinline__ float max_over(float x) { return over_lanes<kApart>(x, [](float p, float q) { return fmaxf(p, q); }); }
template <int kApart> __device__ __forceinline__ float sum_over(float x) { return over_lanes<kApart>(x, [](float p, float q) { return p + q; }); }

// ------------------------------------------------------------------------------------ scores
// i8 matrix instructions, 16 query rows x 16 blocks x 64: A the query rows as [max(qi, 0) | min(qi, 0)], B the bounds [hi | lo]
// of 16 blocks (a block's 2D bytes are whole lines).  Bound: reading the bounds, 1/16 of the cache's bytes in bf16, and for a token
// or a few the chain of round trips to them: place, table entry, bounds.
template <int kD>
struct QueryRows {                                       // 16 rows as a wave holds them
    static constexpr int kSteps = 2 * kD / 64;           // matrix instructions along the 2D products
    i32x4 a[kSteps];
    float scale[4];                                      // of rows 4 q4 + e, whose products stand in this lane: 2^f, NaN for a row that takes no part
};

// 16 query rows made ready in LDS by 256 threads, 16 a row: [max(qi, 0) | min(qi, 0)], 16-byte chunk c of row r at c ^ r.  (Made by every
// wave for itself they were most of a short call's vector work.)
template <bool kBf16, int kD>
struct QueryTile {
    static constexpr int kChunks = 2 * kD / 16, kOwn = kD / 16;          // channels of a thread
    int8_t (&rows)[16 * 2 * kD];
    float (&scale)[16];

    // tid 0 .. 255; `qr`: the channels of row tid / 16, `counts`: whether it is one
    __device__ __forceinline__ void make(const char *qr, bool counts, int tid) const
    {
        const int r = tid >> 4, c = tid & 15;
        float x[kOwn];
        if (kBf16) {
            const uint4 v = *(const uint4 *)(qr + c * 16);
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < kOwn; ++k) x[k] = __uint_as_float(k & 1 ? u[k >> 1] & 0xffff0000u : u[k >> 1] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < kOwn / 4; ++j) {
                const f32x4 v = *(const f32x4 *)(qr + c * (4 * kOwn) + 16 * j);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[4 * j + k] = v[k];
            }
        }
        float size = 0.f;                                // (as bits: they order like the sizes, those of infinities and NaN above all)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) size = __uint_as_float(max(__float_as_uint(size), __float_as_uint(x[k]) & 0x7fffffffu));
        size = reduce16(size, [](float p, float q) { return __uint_as_float(max(__float_as_uint(p), __float_as_uint(q))); });
        const bool finite = __float_as_uint(size) < 0x7f800000u;
        const int f = finite ? step_exponent(size) : 0;
        const float by = step_pow2(-f);
        if (c == 0) scale[r] = finite && counts ? step_pow2(f) : __builtin_nanf("");
        uint32_t plus[kOwn / 4], minus[kOwn / 4];
#pragma unroll
        for (int j = 0; j < kOwn / 4; ++j) {
            plus[j] = minus[j] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = finite ? (int)rintf(x[4 * j + e] * by) : 0;
                plus[j] |= (uint32_t)max(i, 0) << (8 * e);
                minus[j] |= ((uint32_t)min(i, 0) & 0xffu) << (8 * e);
            }
        }
        const int at = c * kOwn, chunk = at >> 4, in = at & 15;
        int8_t *row = rows + r * (2 * kD);
#pragma unroll
        for (int j = 0; j < kOwn / 4; ++j) {
            *(uint32_t *)(row + ((chunk ^ (r % kChunks)) << 4) + in + 4 * j) = plus[j];
            *(uint32_t *)(row + (((chunk + kChunks / 2) ^ (r % kChunks)) << 4) + in + 4 * j) = minus[j];
        }
    }
    __device__ __forceinline__ QueryRows<kD> operands(int r16, int q4) const
    {
        QueryRows<kD> q;
#pragma unroll
        for (int s = 0; s < QueryRows<kD>::kSteps; ++s) q.a[s] = *(const i32x4 *)(rows + r16 * (2 * kD) + (((4 * s + q4) ^ (r16 % kChunks)) << 4));
        const f32x4 y = *(const f32x4 *)(scale + 4 * q4);
#pragma unroll
        for (int e = 0; e < 4; ++e) q.scale[e] = y[e];
        return q;
    }
};

// Whether an entry names a block, and where that block's digest stands among those of the layer and KV head; one that does not reads
// another's.
__device__ __forceinline__ bool is_block(const Geom &g, const SelectArgs &a, int32_t entry)
{
    return entry >= 0 && entry_bid(entry) >= a.first_block && entry_bid(entry) < g.n_blocks;
}
__device__ __forceinline__ int32_t digest_row(const Geom &g, const SelectArgs &a, int32_t entry) { return is_block(g, a, entry) ? entry_bid(entry) : a.first_block; }
__device__ __forceinline__ int64_t digest_rows(const Geom &g, const SelectArgs &a, int kvh) { return ((int64_t)a.layer * g.Hkv + kvh) * g.n_blocks; }
constexpr int kNoBlock = 128;                            // in the place of an exponent; 127 marks a key that is not finite
__device__ __forceinline__ int block_exponent(const Geom &g, const SelectArgs &a, int kvh, int32_t entry)
{
    const int e = a.digests[a.exps_at + digest_rows(g, a, kvh) + digest_row(g, a, entry)];
    return is_block(g, a, entry) ? e : kNoBlock;
}

// The bounds of 16 blocks in LDS: row r of 2D bytes is block r's, its 16-byte chunk c at position c ^ r (so that the operand reads of
// neighbouring rows meet different banks).  By direct loads of whole rows: read straight as operands, 64 bytes of each of 16 rows
// at a time, they take a CU's address path four times as long (see the attention below).
template <int kD>
struct BoundsTile {
    static constexpr int kChunks = 2 * kD / 16, kBytes = 16 * 2 * kD, kLoads = kBytes / 1024;
    uint32_t lds;                                        // 16-byte aligned address of the tile
    // `rows`: the layer and KV head's first digest; row_of(r): the number of block r's
    template <typename F>
    __device__ __forceinline__ void load(const char *rows, int lane, F row_of) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * (64 / kChunks) + lane / kChunks, c = (lane % kChunks) ^ (r % kChunks);
            load_to_lds_each(lds + i * 1024, rows + (uint64_t)(uint32_t)row_of(r) * (2 * kD) + c * 16);
        }
    }
    // The operands of block r16, quarter q4.
    __device__ __forceinline__ void operands(i32x4 (&b)[QueryRows<kD>::kSteps], int r16, int q4) const
    {
        typedef const __attribute__((address_space(3))) i32x4 *lds_chunk;
#pragma unroll
        for (int s = 0; s < QueryRows<kD>::kSteps; ++s)
            b[s] = *(lds_chunk)(uintptr_t)(lds + r16 * (2 * kD) + (((4 * s + q4) ^ (r16 % kChunks)) << 4));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // tile read out
    }
};

// Products of this lane's four rows of each tile with its block, each by its row's power of two (the tiles' chains side by side); NaN of
// a row that takes no part, which no maximum of two numbers picks.
template <int kD, int kTiles>
__device__ __forceinline__ void tile_products(f32x4 (&p)[kTiles], const QueryRows<kD> (&q)[kTiles], const i32x4 (&b)[QueryRows<kD>::kSteps])
{
    i32x4 acc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < QueryRows<kD>::kSteps; ++s)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t].a[s], b[s], acc[t], 0, 0, 0);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[t][e] = (float)acc[t][e] * q[t].scale[e];
}
__device__ __forceinline__ float column_max(f32x4 p)     // over the 16 rows, in every quarter
{
    return max_over<16>(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])));
}

// A block's score as bits that order like it: the largest product of its rows, by the block's own power of two.
struct BlockScale {
    float by, fixed;                                     // 2^e; what stands for the score where there is no e
    bool none;
    __device__ __forceinline__ explicit BlockScale(int e) : by(step_pow2(min(e, 126))), fixed(e == 127 ? INFINITY : -INFINITY), none(e >= 127) {}
    __device__ __forceinline__ uint32_t key(float m) const
    {
        const float x = m * by + 0.f;                    // (+ 0: the two zeros are equal)
        const uint32_t u = __float_as_uint(none ? fixed : x);
        return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    }
};

// Scores to memory, where one launch for scores and list (below) does not do: a work-group takes a KV head and a range of candidates,
// a wave 16 blocks at a time.  Ranges come behind one another in the grid: the last ones are short or empty, and as neighbours
// each would belong to chiplets of its own (the case of many tokens below: 28 us).
// One token (its heads 16 at a time): tokens of many requests, long tables (four tokens, 8 KV heads, 1.4 to 1.7 k blocks: 9.5 us with the
// lists).
template <bool kBf16, int kD>
__global__ __launch_bounds__(256) void score_token_kernel(Geom g, SelectArgs a)
{
    typedef BoundsTile<kD> Tile;
    constexpr int kRounds = kScoreBlocks / 64;
    __shared__ __attribute__((aligned(256))) char s_tile[4][2][Tile::kBytes];
    __shared__ __attribute__((aligned(16))) int8_t s_q[16 * 2 * kD];
    __shared__ __attribute__((aligned(16))) float s_scale[16];
    __shared__ int32_t s_row[kScoreBlocks];
    __shared__ float s_prod[kScoreBlocks];
    const int part = a.parts(blockIdx.x), item = blockIdx.x - part * (int)a.parts.by, token = a.heads(item), kvh = item - token * g.Hkv, n = a.n0 + token;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q4 = lane >> 4;
    const QueryTile<kBf16, kD> rows{s_q, s_scale};
    auto make_rows = [&](int row0) {
        const int r = row0 + (tid >> 4);
        rows.make(a.q + ((int64_t)n * g.Hq + kvh * g.G + min(r, g.G - 1)) * g.head_bytes, r < g.G, tid);
    };
    make_rows(0);                                        // (while the token's place is looked up)
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int j0 = win.first + part * kScoreBlocks;
    if (win.candidates() <= a.n_top || j0 >= win.w0) return;
    const int count = min(kScoreBlocks, win.w0 - j0), rounds = count > 16 * w ? (count - 16 * w + 63) >> 6 : 0;
    const int32_t entry = tid < count ? a.block_table[(int64_t)seq * a.max_blocks + j0 + tid] : -1;
    s_row[tid] = digest_row(g, a, entry);
    __syncthreads();
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)s_tile[w][0];
    auto tile = [&](int k) { return Tile{ring + (uint32_t)(k & 1) * Tile::kBytes}; };
    const char *digests = (const char *)a.digests + digest_rows(g, a, kvh) * (2 * kD);
    auto load = [&](int k) { tile(k).load(digests, lane, [&](int r) { return s_row[64 * k + 16 * w + r]; }); };
    float best[kRounds];
    int exponent = kNoBlock;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) best[k] = -INFINITY;
    for (int row0 = 0; row0 < g.G; row0 += 16) {
        if (row0 > 0) {
            __syncthreads();
            make_rows(row0);
            __syncthreads();
        }
        const QueryRows<kD> q[1] = {rows.operands(r16, q4)};
        for (int k = 0; k < 2 && k < rounds; ++k) load(k);
        if (row0 == 0) exponent = block_exponent(g, a, kvh, entry);      // (needed last: behind the first bounds)
#pragma unroll
        for (int k = 0; k < kRounds; ++k) {
            if (k >= rounds) break;
            if (k + 1 < rounds) wait_loads<Tile::kLoads>();
            else wait_loads<0>();
            i32x4 b[QueryRows<kD>::kSteps];
            tile(k).operands(b, r16, q4);
            if (k + 2 < rounds) load(k + 2);
            f32x4 p[1];
            tile_products<kD>(p, q, b);
            best[k] = fmaxf(best[k], column_max(p[0]));
        }
    }
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
        if (q4 == 0) s_prod[64 * k + 16 * w + r16] = best[k];
    __syncthreads();
    if (tid < count) a.scores[((int64_t)token * g.Hkv + kvh) * a.score_stride + j0 + tid] = BlockScale(exponent).key(s_prod[tid]);
}

// 4 (16 / G) neighbouring tokens, four tiles of query rows: suffixes, whose tokens read the same digests.  Tokens of another request
// follow with a pass of their own.  (681 tokens of eight requests, 8 KV heads, 380 to 849 blocks: 31 us with the lists, of which the
// profiler, under which both launches are slower, gives this one 22 of 36.)  The products of rows 4 q4 + e of tile t stand in quarter q4 of a wave, so these sixteen
// are the heads of 16 / G whole tokens, one after the other, and a token's largest is found in registers.
constexpr int kTiles = 4;

template <bool kBf16, int kD>
__global__ __launch_bounds__(256, 2) void score_group_kernel(Geom g, SelectArgs a)
{
    typedef BoundsTile<kD> Tile;
    __shared__ __attribute__((aligned(256))) char s_tile[4][2][Tile::kBytes];
    __shared__ int32_t s_row[kScoreBlocks], s_exp[kScoreBlocks];
    const int part = a.parts(blockIdx.x), item = blockIdx.x - part * (int)a.parts.by, group = a.heads(item), kvh = item - group * g.Hkv;
    const int n0 = a.n0 + group * a.group_tokens, n1 = min(n0 + a.group_tokens, a.n0 + a.n_tokens);
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q4 = lane >> 4;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)s_tile[w][0];
    auto tile = [&](int k) { return Tile{ring + (uint32_t)(k & 1) * Tile::kBytes}; };
    // lane l looks up the group's token l, and what it chooses from
    int seq_l = -1, pos_l = 0;
    if (lane < n1 - n0 && !token_place(a.token_seq, a.token_pos, n0 + lane, a.B, a.max_blocks, seq_l, pos_l)) seq_l = -1;
    __shared__ __attribute__((aligned(16))) int8_t s_q[kTiles][16 * 2 * kD];
    __shared__ __attribute__((aligned(16))) float s_scale[kTiles][16];
    const int of_group = a.group_tokens / 4;             // tokens of a quarter
    auto make_rows = [&](int t) {
        const int place = 4 * t + ((tid >> 4) & 3), of_quarter = place / g.G;            // among the quarter's sixteen
        const int tok = of_quarter < of_group ? (tid >> 6) * of_group + of_quarter : a.group_tokens, head = place - of_quarter * g.G;
        QueryTile<kBf16, kD>{s_q[t], s_scale[t]}.make(a.q + ((int64_t)min(n0 + tok, n1 - 1) * g.Hq + kvh * g.G + head) * g.head_bytes, n0 + tok < n1, tid);
    };
    QueryRows<kD> q[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) make_rows(t);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) q[t] = QueryTile<kBf16, kD>{s_q[t], s_scale[t]}.operands(r16, q4);
    const char *digests = (const char *)a.digests + digest_rows(g, a, kvh) * (2 * kD);
    const Window win_l(seq_l >= 0 ? pos_l : 0, a.n_sink, a.n_local);
    const bool scores_l = seq_l >= 0 && win_l.candidates() > a.n_top;
    for (int t0 = n0, t1; t0 < n1; t0 = t1) {
        // tokens t0 .. t1 - 1 of one request, and the candidates that one of them chooses from
        const int seq = __builtin_amdgcn_readlane(seq_l, t0 - n0);
        const uint64_t other = ~(__ballot(seq_l == seq && lane < n1 - n0) >> (t0 - n0));
        t1 = t0 + (other ? __builtin_ctzll(other) : 64);
        const bool mine = scores_l && lane >= t0 - n0 && lane < t1 - n0;
        int j0 = (int)~wave_max(mine ? ~(uint32_t)win_l.first : 0u);
        const int j1 = (int)wave_max(mine ? (uint32_t)win_l.w0 : 0u);
        if (j1 == 0 || j0 + part * kScoreBlocks >= j1) continue;       // (0: none has too many)
        j0 += part * kScoreBlocks;
        const uint32_t in_run = (uint32_t)(__ballot(mine) >> (q4 * of_group));     // of this quarter's tokens (16 at most)
        const int count = min(kScoreBlocks, j1 - j0), rounds = count > 16 * w ? (count - 16 * w + 63) >> 6 : 0;
        const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks + j0;
        __syncthreads();                                 // (another request's entries were read)
        const int32_t entry = tid < count ? table[tid] : -1;
        s_row[tid] = digest_row(g, a, entry);
        s_exp[tid] = block_exponent(g, a, kvh, entry);
        __syncthreads();
        auto load = [&](int k) { tile(k).load(digests, lane, [&](int r) { return s_row[64 * k + 16 * w + r]; }); };
        for (int k = 0; k < 2 && k < rounds; ++k) load(k);
        for (int k = 0; k < rounds; ++k) {
            if (k + 1 < rounds) wait_loads<Tile::kLoads>();
            else wait_loads<0>();
            i32x4 b[QueryRows<kD>::kSteps];
            tile(k).operands(b, r16, q4);
            if (k + 2 < rounds) load(k + 2);
            const int i = 64 * k + 16 * w + r16, j = j0 + i;
            f32x4 p[kTiles];
            tile_products<kD>(p, q, b);
            const BlockScale block(i < count ? s_exp[i] : kNoBlock);
            int head = 0;
            uint32_t left = i < count ? in_run : 0;
            uint32_t *out = a.scores + ((int64_t)(n0 - a.n0 + q4 * of_group) * g.Hkv + kvh) * a.score_stride + j;
            float m = -INFINITY;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    m = fmaxf(m, p[t][e]);
                    if (++head < g.G) continue;  // (the same for the whole wave)
                    head = 0;
                    if (left & 1) *out = block.key(m);
                    left >>= 1;
                    out += a.score_stride * g.Hkv;
                    m = -INFINITY;
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------ lists
// All of a list but the chosen candidates; where all candidates are listed, those too.
__device__ __forceinline__ void write_fixed(const SelectArgs &a, const Window &win, int32_t *list, int tid, int threads)
{
    const int cand = win.candidates(), n_list = a.n_sink + a.n_top + a.n_local;
    const int n_chosen = min(cand, a.n_top), n_all = win.first + n_chosen + (win.own - win.w0 + 1);
    for (int i = tid; i < n_list; i += threads)
        if (i < win.first) list[i] = i;
        else if (i >= n_all) list[i] = -1;
        else if (i >= win.first + n_chosen) list[i] = win.w0 + (i - win.first - n_chosen);
        else if (cand <= a.n_top) list[i] = i;
}

// The n_top best of a token's candidates and, behind ties, the lower ones; written in ascending order between the first
// blocks and the last.  The n_top-th largest score is found by bins over the range that still holds it: a histogram of 1024 equal
// bins between its ends, the bin that the count falls into, and again inside that (at most four rounds; scores that are spread
// out take two).  A thread holds kPer neighbouring candidates, so that one prefix sum over the threads places them.
constexpr int kSelectBins = 1024;

template <int kThreads, int kBins>
struct PickShared {
    __attribute__((aligned(16))) uint32_t bins[kBins], lo[kThreads / 64], hi[kThreads / 64], wave[kThreads / 64], found[3];
};

// The sum of the waves' values before wave w.
template <int kWaves>
__device__ __forceinline__ uint32_t before_wave(const uint32_t (&wave)[kWaves], int w)
{
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) sum += k < w ? wave[k] : 0;
    return sum;
}

// key: of `have` candidates from c0 on (of 65535 at most in all threads); s.bins are zero, in all threads' sight.
template <int kThreads, int kAll, int kPer>
__device__ __forceinline__ void pick(PickShared<kThreads, kAll> &s, const uint32_t (&key)[kPer], int c0, int have, int n_top, int first, int32_t *list, int tid)
{
    constexpr int kBins = kAll / kThreads;               // of a thread
    constexpr int kBits = __builtin_ctz(kAll);
    const int lane = tid & 63, w = tid >> 6;
    uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (k < have) {
            lo = min(lo, key[k]);
            hi = max(hi, key[k]);
        }
    hi = wave_max(hi);
    lo = ~wave_max(~lo);
    if (lane == 0) { s.lo[w] = lo; s.hi[w] = hi; }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) { lo = min(lo, s.lo[k]); hi = max(hi, s.hi[k]); }
    // keys above `hi` are chosen; `want` of those in [lo, hi] are still to be found
    uint32_t want = n_top;
    bool whole = false;
    while (lo < hi) {
        const int shift = max(0, 32 - kBits - (int)__builtin_clz(hi - lo));     // (hi - lo) >> shift < kAll
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (k < have && key[k] >= lo && key[k] <= hi) atomicAdd(&s.bins[(key[k] - lo) >> shift], 1u);
        __syncthreads();
        // counted from the top: thread t holds bins kAll - 1 - kBins t and the next lower ones
        uint32_t c[kBins], sum = 0;
#pragma unroll
        for (int k = 0; k < kBins; ++k) { c[k] = s.bins[kAll - 1 - kBins * tid - k]; sum += c[k]; }
        const uint32_t x = wave_prefix(sum);
        if (lane == 63) s.wave[w] = x;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kBins; ++k) s.bins[kAll - 1 - kBins * tid - k] = 0;
        uint32_t above = before_wave(s.wave, w) + x - sum;
#pragma unroll
        for (int k = 0; k < kBins; ++k) {
            if (above < want && above + c[k] >= want) { s.found[0] = kAll - 1 - kBins * tid - k; s.found[1] = above; s.found[2] = c[k]; }
            above += c[k];
        }
        __syncthreads();
        whole = want - s.found[1] == s.found[2];         // all of the bin: its lower end is the threshold
        want -= s.found[1];
        lo += s.found[0] << shift;
        hi = shift == 0 ? lo : min(hi, lo + ((1u << shift) - 1));
        if (whole) break;
    }
    // chosen: keys above the threshold, and the first `want` of those at it
    uint32_t mine = 0;                                   // (keys at the threshold << 16) + keys above it
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const bool is = k < have;
        mine += is && (whole ? key[k] >= lo : key[k] > lo) ? 1u : is && !whole && key[k] == lo ? 0x10000u : 0u;
    }
    const uint32_t x = wave_prefix(mine);
    if (lane == 63) s.wave[w] = x;                       // (its last reads were before the loop's last barrier)
    __syncthreads();
    const uint32_t before = before_wave(s.wave, w) + x - mine;
    uint32_t above = before & 0xffffu, ties = before >> 16;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const bool is = k < have, over = is && (whole ? key[k] >= lo : key[k] > lo), tie = is && !whole && key[k] == lo;
        if (over || (tie && ties < want)) list[first + above + min(ties, want)] = first + c0 + k;
        above += over;
        ties += tie;
    }
}

// Lists from scores in memory: a work-group a (token, KV head).  Times of this launch under the profiler, of passes without it:
//   kThreads 256: eight candidates a thread, 1024 bins, a chain of barriers (32 items, 118 of 1.7 k each: 5.9 us)
//   kThreads 64: a wave, which waits for no other, up to 16 a thread, 256 bins.  Longer from start to end, but beyond four waves a CU
//   what counts is what they do together (5.4 k items, 60 of some 600: 14.3 us, 17.6 by 256 threads; a pass of scores, list and
//   attention for 640 items 41.0 against 39.6, for 1088 50.0 against 50.5, for 15 k 325 against 341)
constexpr int kSelectWave = 64 * 16, kSelectFew = 256 * 8;              // table entries that each does for
constexpr int kSelectItems = 1024;

template <int kThreads, int kPer, int kBins>
__global__ __launch_bounds__(kThreads) void select_kernel(Geom g, SelectArgs a)
{
    __shared__ PickShared<kThreads, kBins> s;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(4)));
    const int token = a.heads(blockIdx.x), n = a.n0 + token, kvh = blockIdx.x - token * g.Hkv, tid = threadIdx.x;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int cand = win.candidates();
    int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * (a.n_sink + a.n_top + a.n_local);
    if (cand > a.n_top && a.n_top > 0) {
        const uint32_t *scores = a.scores + ((int64_t)(n - a.n0) * g.Hkv + kvh) * a.score_stride + win.first;
        const int per = (cand + 4 * kThreads - 1) / (4 * kThreads) * 4, c0 = per * tid;
        uint32_t key[kPer];
#pragma unroll
        for (int k = 0; k < kPer; k += 4) {
            u32x4 v = {0, 0, 0, 0};
            if (k >= per) {                              // (the same for all)
            } else if (c0 + k + 3 < cand) v = *(const u32x4 *)(scores + c0 + k);
            else if (c0 + k < cand) {                    // (the row's last few)
                v[0] = scores[c0 + k];
                v[1] = c0 + k + 1 < cand ? scores[c0 + k + 1] : 0;
                v[2] = c0 + k + 2 < cand ? scores[c0 + k + 2] : 0;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) key[k + e] = v[e];
        }
        static_assert(kBins == 4 * kThreads, "a thread clears four bins");
        *(uint4 *)&s.bins[4 * tid] = make_uint4(0, 0, 0, 0);             // (seen behind pick's first barrier)
        pick(s, key, c0, min(max(cand - c0, 0), per), a.n_top, win.first, list, tid);
    }
    write_fixed(a, win, list, tid, kThreads);
}

// The same for tables of more than kSelectFew entries: the scores stay in memory and are read again in every round.
__global__ __launch_bounds__(256) void select_long_kernel(Geom g, SelectArgs a)
{
    __shared__ uint32_t s_bins[kSelectBins];
    __shared__ uint32_t s_wave[8], s_found[3];
    const int token = a.heads(blockIdx.x), n = a.n0 + token, kvh = blockIdx.x - token * g.Hkv;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int cand = win.candidates(), n_list = a.n_sink + a.n_top + a.n_local;
    int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * n_list;
    write_fixed(a, win, list, tid, 256);
    if (cand <= a.n_top || a.n_top == 0) return;
    const uint32_t *scores = a.scores + ((int64_t)(n - a.n0) * g.Hkv + kvh) * a.score_stride + win.first;
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int i = tid; i < cand; i += 256) {
        const uint32_t k = scores[i];
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
    const uint32_t *keys = scores;
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

// Scores and list in one launch, for few tokens whose tables are not long: a work-group of sixteen waves a (token, KV head), the
// scores in LDS.  A CU takes its digests at some 80 GB/s, so beyond kFusedBlocks table entries launches that spread them over the chip
// are as good or better (four tokens of 8 KV heads, 1.7 k entries: 12.4 us so, 12.0 in two), and many tokens of a request should
// read them once (above kFusedItems).  One token of 4 KV heads, 288 entries: 6.6 us a call;
// 32 tokens of up to 311: 7.0.
constexpr int kFusedBlocks = 1536, kFusedItems = 512;

template <bool kBf16, int kD>
__global__ __launch_bounds__(1024) void score_select_kernel(Geom g, SelectArgs a)
{
    extern __shared__ __attribute__((aligned(256))) char s_ring[];       // two tiles a wave
    __shared__ PickShared<1024, kSelectBins> s_pick;
    __shared__ int32_t s_row[kFusedBlocks];
    __shared__ float s_prod[kFusedBlocks];
    const int token = a.heads(blockIdx.x), n = a.n0 + token, kvh = blockIdx.x - token * g.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q4 = lane >> 4;
    __shared__ __attribute__((aligned(16))) int8_t s_q[16 * 2 * kD];
    __shared__ __attribute__((aligned(16))) float s_scale[16];
    const QueryTile<kBf16, kD> rows{s_q, s_scale};
    auto make_rows = [&](int row0) {
        const int r = row0 + (tid >> 4);
        if (tid < 256) rows.make(a.q + ((int64_t)n * g.Hq + kvh * g.G + min(r, g.G - 1)) * g.head_bytes, r < g.G, tid);
    };
    make_rows(0);                                        // (while the token's place is looked up)
    s_pick.bins[tid] = 0;
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const Window win(pos, a.n_sink, a.n_local);
    const int cand = win.candidates(), n_list = a.n_sink + a.n_top + a.n_local;
    int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * n_list;
    if (cand <= a.n_top || a.n_top == 0) {
        write_fixed(a, win, list, tid, 1024);
        return;
    }
    const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks + win.first;

    // ---- scores: wave w takes blocks 16 w .. 16 w + 15 of every 256; thread t makes keys of those of candidates 2t and 2t + 1
    typedef BoundsTile<kD> Tile;
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)s_ring + w * 2 * Tile::kBytes;
    auto tile = [&](int k) { return Tile{ring + (uint32_t)(k & 1) * Tile::kBytes}; };
    const char *digests = (const char *)a.digests + digest_rows(g, a, kvh) * (2 * kD);
    const int c0 = 2 * tid;
    int32_t entry[2] = {-1, -1};
    int exponent[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (c0 + k < cand) s_row[c0 + k] = digest_row(g, a, entry[k] = table[c0 + k]);
    __syncthreads();
    const int rounds = cand > 16 * w ? (cand - 16 * w + 255) >> 8 : 0;
    auto load = [&](int k) {
        tile(k).load(digests, lane, [&](int r) { return s_row[min(256 * k + 16 * w + r, cand - 1)]; });
    };
    for (int row0 = 0; row0 < g.G; row0 += 16) {
        if (row0 > 0) {
            __syncthreads();
            make_rows(row0);
            __syncthreads();
        }
        const QueryRows<kD> q[1] = {rows.operands(r16, q4)};
        for (int k = 0; k < 2 && k < rounds; ++k) load(k);
        if (row0 == 0) {                                 // (needed last: behind the first bounds)
#pragma unroll
            for (int k = 0; k < 2; ++k) exponent[k] = block_exponent(g, a, kvh, entry[k]);
        }
        for (int k = 0; k < rounds; ++k) {
            if (k + 1 < rounds) wait_loads<Tile::kLoads>();
            else wait_loads<0>();
            i32x4 b[QueryRows<kD>::kSteps];
            tile(k).operands(b, r16, q4);
            if (k + 2 < rounds) load(k + 2);
            f32x4 p[1];
            tile_products<kD>(p, q, b);
            float m = fmaxf(column_max(p[0]), -INFINITY);      // (no row takes part)
            const int i = 256 * k + 16 * w + r16;
            if (q4 == 0 && i < cand) {
                if (row0 > 0) m = fmaxf(m, s_prod[i]);   // (of this wave's own earlier rows)
                s_prod[i] = m;
            }
        }
    }
    __syncthreads();
    uint32_t key[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (c0 + k < cand) key[k] = BlockScale(exponent[k]).key(s_prod[c0 + k]);
    pick(s_pick, key, c0, min(cand - c0, 2), a.n_top, win.first, list, tid);
    write_fixed(a, win, list, tid, 1024);                // (last: a barrier behind a store to memory waits for it)
}

template <bool kBf16, int kD>
static hipError_t launch_score_select(const Geom &g, const SelectArgs &a, const Launch &L)
{
    constexpr int kLds = 16 * 2 * BoundsTile<kD>::kBytes;
    static PerDeviceOnce configured;
    const hipError_t e = configured.run([] {
        return hipFuncSetAttribute((const void *)score_select_kernel<kBf16, kD>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    });
    if (e != hipSuccess) return e;
    TC_LAUNCH_N((score_select_kernel<kBf16, kD>), a.n_tokens * g.Hkv, 1024, kLds, L, g, a);
    return hipGetLastError();
}

template <bool kBf16, int kD>
static hipError_t launch_scores(const Geom &g, SelectArgs a, const Launch &L)
{
    const bool grouped = scores_by_group(a.n_tokens, a.B, g.G, g.Hkv, a.max_blocks);
    a.group_tokens = grouped ? score_group_tokens(g.G) : 1;
    a.score_parts = (int32_t)score_parts(a.max_blocks);
    const int64_t grid = (int64_t)((a.n_tokens + a.group_tokens - 1) / a.group_tokens) * g.Hkv * a.score_parts;
    if (grid > kStepMaxGroups) return hipErrorInvalidValue;
    a.parts = FastDiv((uint32_t)(grid / a.score_parts));
    if (grouped) TC_LAUNCH((score_group_kernel<kBf16, kD>), (unsigned)grid, 0, L, g, a);
    else TC_LAUNCH((score_token_kernel<kBf16, kD>), (unsigned)grid, 0, L, g, a);
    return hipGetLastError();
}

int64_t select_groups(int Hkv, int max_blocks) { return (int64_t)Hkv * std::max<int64_t>(1, score_parts(max_blocks)); }

hipError_t launch_select(const Geom &g, SelectArgs a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    a.heads = FastDiv((uint32_t)g.Hkv);
    const int most = a.max_blocks;                       // candidates of any token
    const int64_t items = (int64_t)a.n_tokens * g.Hkv;
    if (items > kStepMaxGroups) return hipErrorInvalidValue;
    if (most <= kFusedBlocks && items <= kFusedItems)
        return g.esize == 2 ? launch_score_select<true, 128>(g, a, L)
             : g.D == 64 ? launch_score_select<false, 64>(g, a, L) : launch_score_select<false, 128>(g, a, L);
    if (most > a.n_top && a.n_top > 0) {
        const hipError_t e = g.esize == 2 ? launch_scores<true, 128>(g, a, L)
                           : g.D == 64 ? launch_scores<false, 64>(g, a, L) : launch_scores<false, 128>(g, a, L);
        if (e != hipSuccess) return e;
    }
    if (most <= kSelectWave && items > kSelectItems) TC_LAUNCH_N((select_kernel<64, 16, 256>), (unsigned)items, 64, 0, L, g, a);
    else if (most <= kSelectFew) TC_LAUNCH_N((select_kernel<256, 8, kSelectBins>), (unsigned)items, 256, 0, L, g, a);
    else TC_LAUNCH(select_long_kernel, (unsigned)items, 0, L, g, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ attention
__device__ __forceinline__ uint32_t bf16_pair(float x, float y)
{
    return (uint32_t)__builtin_bit_cast(unsigned short, (__bf16)x) | ((uint32_t)__builtin_bit_cast(unsigned short, (__bf16)y) << 16);
}
__device__ __forceinline__ void write_bf16x4(char *dst, f32x4 x) { *(uint2 *)dst = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])); }

// out = softmax(sm_scale q . k) v over the keys of the listed blocks at positions up to the token's own that hold a token;
// zeros where there are none.  A token and KV head have G rows that share a list, so as in the decode kernel the work is
// reading the listed keys and values once, and a short list is a chain of round trips.
//
// A work-group is (token, KV head, 16 rows, range of the list); its waves take the range's units in turn, keep their own
// running maximum and sum, and are combined through LDS at the end.  No wave waits for another before that.
// A row's partial outputs, maxima and sums of kParts waves: four columns of each, `apart` floats from wave to wave, and the two at `ml`,
// `ml_apart` floats apart.  `rest`: a wave's sums that belong to those `rest` floats before them, where they are finite (0: none).
template <int kParts>
__device__ __forceinline__ RowSum fold_rows(const float *part, int apart, const float *ml, int ml_apart, int rest)
{
    RowSum x{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    f32x4 rests = {0.f, 0.f, 0.f, 0.f};
    float2 of[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        of[k] = *(const float2 *)(ml + k * ml_apart);
        x.M = fmaxf(x.M, of[k].x);
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        // (no maximum: no keys - its sums are zeros - or only scores that are NaN, and so are they)
        const float wgt = of[k].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(of[k].x - x.M);
        x.L += wgt * of[k].y;
        x.acc += wgt * *(const f32x4 *)(part + k * apart);
        if (rest != 0) rests += wgt * *(const f32x4 *)(part + rest + k * apart);
    }
    if (rest != 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x.acc[e] += __builtin_isfinite(rests[e]) ? rests[e] : 0.f;
    }
    return x;
}

// Block j of a list: its table entry (-1: none), and how many of its positions the token sees (0: none).
__device__ __forceinline__ int32_t listed_entry(const int32_t *table, int32_t j, int pos) { return j >= 0 && j <= pos >> 4 ? table[j] : -1; }
__device__ __forceinline__ int listed_keys(const Geom &g, const BlockAttnArgs &a, int32_t j, int32_t entry, int pos)
{
    const int bid = entry_bid(entry);
    return entry >= 0 && bid >= a.first_block && bid < g.n_blocks ? min(kBlockTokens - entry_pad(entry), pos - j * kBlockTokens + 1) : 0;
}

// bf16, heads of 128.  A unit is two blocks, 32 keys, against 16 query rows: S^T = K Q^T by 16x16x32 matrix instructions whose
// 16 keys are tokens 0..7 of both blocks, then 8..15, so that a lane's eight scores (quarter q4 of the wave: block q4 / 2,
// half q4 % 2) belong to the eight tokens whose values stand in one 16-byte piece of the pool's V rows, and O^T += V^T P^T
// takes both as they are.  A weight goes into that product as a sum of two bf16 numbers, itself rounded and what that leaves out, so
// that 16 bits of it count and the output's own rounding is the one that shows.  Up to eight rows have their rests in the columns that
// would be copies (kRest: rows behind the eighth), more rows in instructions of their own.  The rests' sums are kept apart and left out where they
// are no finite number: an infinite value times a rest of zero, or of the other sign, is not what the formula has.  Values at positions that the
// token does not see are replaced by zeros, whatever stands there.
//
// A unit's 16 KB come by direct loads into the wave's own piece of LDS, a kilobyte of neighbouring bytes each, and the operands
// from there: loaded straight into the operands' registers, where neighbouring lanes are neighbouring rows of 256 bytes, keys take a
// CU's address path 64 cycles a kilobyte instead of 16.  The next unit's keys are requested as soon as this one's are in
// registers, and so the values.  (Values straight to registers, 32-byte rows, and twice the waves: slower for every list tried.)
// Bound: 53 blocks for each of 4 items, 7.7 us a call, what one CU takes; 49 for each of 128, 51 MB, 11.8 us = 4.4 TB/s, likewise;
// 64 for each of 5.4 k items, 151 us, 2.9 GB through the L2s = 19 TB/s, of which a fifth misses there (counters: 22.6 M requests of 128
// bytes, 4.7 M misses).
constexpr int kBaBlock = 4096;                           // one head's K (or V) in one block
constexpr int kBaWaves = 4;
constexpr int kBaWave = 4 * kBaBlock;                    // K of a unit: rows of 256 bytes, 16-byte chunk c of row r at c ^ r; V: two blocks verbatim
constexpr int kBaChunk = 32 * kBaWaves;                  // units that a work-group looks up at a time, 32 a wave: lane 2k + b looks up block b of unit k

constexpr float kBaRescale = 8.f;                        // weights grow to 2^8 before the reference moves

template <bool kSplit, bool kRest>
__global__ __launch_bounds__(64 * kBaWaves, 2) void block_attn_bf16_kernel(Geom g, BlockAttnArgs a)
{
    extern __shared__ __attribute__((aligned(256))) char lds[];          // (the XOR addressing of the K rows needs them 256-byte aligned)
    __shared__ float2 s_ml[kBaWaves][16];
    const int chunks = (int)a.chunks.by;
    const int item = a.splits(blockIdx.x), split = blockIdx.x - item * a.n_splits;
    const int head = a.chunks(item), n = a.heads(head), kvh = head - n * g.Hkv, row0 = (item - head * chunks) * 16;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q4 = lane >> 4;
    const int rows = min(16, g.G - row0);
    const int32_t *list = a.lists + ((int64_t)n * g.Hkv + kvh) * a.n_list;
    const int n_units = (a.n_list + 1) >> 1;
    const int u0 = (int)((int64_t)n_units * split / a.n_splits), u1 = (int)((int64_t)n_units * (split + 1) / a.n_splits);
    auto listed = [&](int k0) {                          // this lane's block of the units from k0 on
        const int i = 2 * (k0 + kBaWaves * (lane >> 1)) + (lane & 1);
        return i < min(2 * u1, a.n_list) ? list[i] : -1;
    };
    int32_t j = listed(u0 + w);                          // (while the token's place is looked up)
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, n, a.B, a.max_blocks, seq, pos)) return;
    const int32_t *table = a.block_table + (int64_t)seq * a.max_blocks;
    const char *pool = g.pool + (int64_t)a.layer * g.layer_stride + (int64_t)kvh * kBaBlock;
    const int64_t v_half = g.block_bytes >> 1;
    const uint32_t lds_w = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + w * kBaWave;
    typedef const __attribute__((address_space(3))) bf16x8 *lds_frag;

    int32_t entry = listed_entry(table, j, pos);
    bf16x8 qf[4];
    {
        const char *qr = a.q + ((int64_t)n * g.Hq + kvh * g.G + row0 + min(kRest ? r16 & 7 : r16, rows - 1)) * 256 + q4 * 16;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qf[ks] = *(const bf16x8 *)(qr + ks * 64);
    }
    f32x4 o[8], o_rest[8];                               // by the weights in bf16, and by what they leave out (kRest: both in o)
#pragma unroll
    for (int db = 0; db < 8; ++db) o[db] = o_rest[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool rests = !kRest || r16 >= 8;               // what of a weight in bf16, in the lower and upper half of a register, is taken from it
    const uint32_t low_half = rests ? 0x01000c0cu : 0x0c0c0c0cu, high_half = rests ? 0xffff0000u : 0u;
    float m_run = -INFINITY, l_lane = 0.f;

    uint32_t k_off[4], v_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k_off[i] = (uint32_t)((lane >> 4) * 256 + (((lane & 15) ^ (4 * i + (lane >> 4))) * 16));
        v_off[i] = (uint32_t)lane * 16;
    }
    // the operands of this lane: K row r16 & 7 (+ 8) of block r16 / 8, chunk 4 ks + q4; V row 16 db + r16 of block q4 / 2, half q4 & 1
    const uint32_t kr = (uint32_t)(r16 & 7), kb = lds_w + (r16 >> 3) * kBaBlock + kr * 256 + ((q4 ^ kr) << 4);
    const uint32_t vb = lds_w + 2 * kBaBlock + (q4 >> 1) * kBaBlock + r16 * 32 + (q4 & 1) * 16;

    int keys;
    const char *src[2];
    auto sources = [&](int k) {
        const int v0 = __builtin_amdgcn_readlane(keys, 2 * k), v1 = __builtin_amdgcn_readlane(keys, 2 * k + 1);
        const int b0 = entry_bid(__builtin_amdgcn_readlane(entry, 2 * k)), b1 = entry_bid(__builtin_amdgcn_readlane(entry, 2 * k + 1));
        // (what is loaded in an empty block's place is masked)
        src[0] = pool + (int64_t)(v0 > 0 ? b0 : v1 > 0 ? b1 : a.first_block) * g.block_bytes;
        src[1] = pool + (int64_t)(v1 > 0 ? b1 : v0 > 0 ? b0 : a.first_block) * g.block_bytes;
    };
    auto issue_k = [&]() {
        load4_to_lds(lds_w, src[0], k_off);
        load4_to_lds(lds_w + kBaBlock, src[1], k_off);
    };
    auto issue_v = [&]() {
        load4_to_lds(lds_w + 2 * kBaBlock, src[0] + v_half, v_off);
        load4_to_lds(lds_w + 3 * kBaBlock, src[1] + v_half, v_off);
    };
    // Unit k, whose keys and values were requested before; those of the next one, where there are more, as the areas become free.
    auto unit = [&](int k, bool more) __attribute__((always_inline)) {
        const int valid0 = __builtin_amdgcn_readlane(keys, 2 * k), valid1 = __builtin_amdgcn_readlane(keys, 2 * k + 1);
        wait_loads<8>();                                 // K is there, V may be on its way
        bf16x8 kf[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) kf[i] = *(lds_frag)(uintptr_t)(((kb ^ ((i & 3) << 6)) ^ ((i >> 2) << 7)) + (i >> 2) * 2048);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K area read out
        if (more) {
            sources(k + 1);
            issue_k();
        }
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[4 * h + ks], qf[ks], s[h], 0, 0, 0);
        }
        if (more) wait_loads<8>();
        else wait_loads<0>();
        bf16x8 vf[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) vf[i] = *(lds_frag)(uintptr_t)(vb + i * 512);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V area read out
        if (more) issue_v();
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
        const float mxs = max_over<16>(mx) * a.scale_log2;
        if (__any(mxs > m_run + kBaRescale)) {   // also taken while m_run is still -inf
            const float m_new = fmaxf(m_run, mxs);
            const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
            l_lane *= alpha;
#pragma unroll
            for (int db = 0; db < 8; ++db)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[db][e] *= alpha;
                    if (!kRest) o_rest[db][e] *= alpha;
                }
            m_run = m_new;
        }
        const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
        bf16x8 pf, rest;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(s[h][e], a.scale_log2, neg_m)), p1 = __builtin_amdgcn_exp2f(fmaf(s[h][e + 1], a.scale_log2, neg_m));
                l_lane += p0;
                l_lane += p1;
                const uint32_t both = bf16_pair(p0, p1);
                // (kRest: the lanes of the first eight columns subtract nothing)
                const float r0 = p0 - __uint_as_float(__builtin_amdgcn_perm(0u, both, low_half)), r1 = p1 - __uint_as_float(both & high_half);
                const uint32_t left = bf16_pair(r0, r1);
                ((uint32_t *)&pf)[2 * h + e / 2] = kRest ? left : both;
                ((uint32_t *)&rest)[2 * h + e / 2] = left;
            }
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[db], pf, o[db], 0, 0, 0);
            if (!kRest) o_rest[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[db], rest, o_rest[db], 0, 0, 0);
        }
    };
    for (int k0 = u0 + w; k0 < u1; k0 += kBaChunk) {
        keys = listed_keys(g, a, j, entry, pos);
        const uint64_t some = __ballot(keys > 0);
        const int units = some ? (65 - __builtin_clzll(some)) >> 1 : 0;      // up to the last one with a key
        asm volatile("" : "+v"(qf[0]), "+v"(qf[1]), "+v"(qf[2]), "+v"(qf[3]));      // (in registers: nothing but the counted loads is outstanding from here on)
        if (units > 0) {
            sources(0);
            issue_k();
            issue_v();
            for (int k = 0; k + 1 < units; ++k) unit(k, true);
            unit(units - 1, false);
        }
        if (k0 + kBaChunk < u1) entry = listed_entry(table, j = listed(k0 + kBaChunk), pos);
    }

    // the waves' (output, maximum, sum) rows, combined by 32 threads a row, four columns each: chunk c of row r at c ^ r of the V area
    const float l_row = sum_over<16>(l_lane);
    if (!kRest) {
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][e] += __builtin_isfinite(o_rest[db][e]) ? o_rest[db][e] : 0.f;
    }
    if ((kRest ? r16 & 7 : r16) < rows) {                // (kRest: the rests as rows eight further on)
        char *mine = lds + w * kBaWave + 2 * kBaBlock + r16 * 512;
#pragma unroll
        for (int db = 0; db < 8; ++db) *(f32x4 *)(mine + (((4 * db + q4) ^ r16) << 4)) = o[db];
        if (q4 == 0) s_ml[w][r16] = make_float2(m_run, l_row);
    }
    __syncthreads();
    const int c = tid & 31, d = 4 * c;
    for (int row = tid >> 5; row < rows; row += 2 * kBaWaves) {
        const float *part = (const float *)(lds + 2 * kBaBlock + row * 512 + ((c ^ row) << 4));
        const int to_rest = kRest ? 8 * 128 + ((c & 8) ? -32 : 32) : 0;          // row + 8's chunk c stands at c ^ (row + 8)
        const RowSum x = fold_rows<kBaWaves>(part, kBaWave / (int)sizeof(float), (const float *)&s_ml[0][row], 16 * 2, to_rest);
        const int64_t out_row = (int64_t)n * g.Hq + kvh * g.G + row0 + row;
        if (kSplit) {
            *(f32x4 *)(a.part_o + (out_row * a.n_splits + split) * 128 + d) = x.acc;
            if (d == 0) *(float2 *)(a.part_ml + (out_row * a.n_splits + split) * 2) = make_float2(x.M, x.L);
        } else {
            write_bf16x4(a.out + out_row * 256 + d * 2, x.acc * (x.L == 0.f ? 0.f : 1.f / x.L));
        }
    }
}

// fp32, heads of 64 or 128: a unit is one block.  A key row is four channels for each of kD / 4 lanes, so a wave scores
// 64 / (kD / 4) keys at a time, for up to eight rows, and each of its lane groups keeps a maximum and a sum of its own.
constexpr int kBaF32Rows = 8;

template <int kD, bool kSplit>
__global__ __launch_bounds__(256, 2) void block_attn_f32_kernel(Geom g, BlockAttnArgs a)
{
    constexpr int kLanes = kD / 4, kGroups = 64 / kLanes, kSteps = kBlockTokens / kGroups, kRows = kBaF32Rows, kRow = kD + 4, kWaves = 4;
    __shared__ __attribute__((aligned(16))) float s_part[kWaves * kRows * kRow];         // output, maximum, sum
    const int chunks = (int)a.chunks.by;
    const int item = a.splits(blockIdx.x), split = blockIdx.x - item * a.n_splits;
    const int head = a.chunks(item), n = a.heads(head), kvh = head - n * g.Hkv, row0 = (item - head * chunks) * kRows;
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
    for (int k0 = u0 + w; k0 < u1; k0 += kWaves * 64) {
        const int32_t j = k0 + kWaves * lane < u1 ? list[k0 + kWaves * lane] : -1, entry = listed_entry(table, j, pos);
        const int keys = listed_keys(g, a, j, entry, pos);
        const int n_mine = min(64, (u1 - k0 + kWaves - 1) / kWaves);
        for (int k = 0; k < n_mine; ++k) {
            const int valid = __builtin_amdgcn_readlane(keys, k);
            if (valid <= 0) continue;
            const char *p = pool + (int64_t)entry_bid(__builtin_amdgcn_readlane(entry, k)) * g.block_bytes;
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
    // the lane groups' rows, then the waves'
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (r >= rows) break;
        const float M = max_over<kLanes>(m_run[r]);
        const float wgt = m_run[r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[r] - M);
        const float l = sum_over<kLanes>(l_run[r] * wgt);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = sum_over<kLanes>(o[r][e] * wgt);
        float *mine = s_part + (w * kRows + r) * kRow;
        if (grp == 0) *(f32x4 *)(mine + 4 * c) = y;
        if (lane == 0) *(float2 *)(mine + kD) = make_float2(M, l);
    }
    __syncthreads();
    constexpr int kThreadsRow = kD / 4;
    for (int row = tid / kThreadsRow; row < rows; row += 64 * kWaves / kThreadsRow) {
        const int d = 4 * (tid % kThreadsRow);
        const RowSum x = fold_rows<kWaves>(s_part + row * kRow + d, kRows * kRow, s_part + row * kRow + kD, kRows * kRow, 0);
        const int64_t out_row = (int64_t)n * g.Hq + kvh * g.G + row0 + row;
        if (kSplit) {
            *(f32x4 *)(a.part_o + (out_row * a.n_splits + split) * kD + d) = x.acc;
            if (d == 0) *(float2 *)(a.part_ml + (out_row * a.n_splits + split) * 2) = make_float2(x.M, x.L);
        } else {
            *(f32x4 *)(a.out + (out_row * kD + d) * 4) = x.acc * (x.L == 0.f ? 0.f : 1.f / x.L);
        }
    }
}

// Ranges of a list combined: kD / 4 threads a row, all of a row's first partials requested at once (bound: the launch and one round trip;
// 128 rows of four ranges 3.7 us under the profiler).
template <bool kBf16, int kD>
__global__ __launch_bounds__(256) void block_merge_kernel(Geom g, BlockAttnArgs a)
{
    constexpr int kThreadsRow = kD / 4;
    const int64_t row = (int64_t)blockIdx.x * (256 / kThreadsRow) + threadIdx.x / kThreadsRow;
    const int d = 4 * (threadIdx.x % kThreadsRow);
    if (row >= (int64_t)a.n_tokens * g.Hq) return;
    RowSum x{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    constexpr int kBatch = 8;                            // partials requested before the first is used
    float2 ml[kBatch];
    f32x4 po[kBatch];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t at = row * a.n_splits + min(s0 + j, a.n_splits - 1);
            ml[j] = *(const float2 *)(a.part_ml + at * 2);
            po[j] = *(const f32x4 *)(a.part_o + at * kD + d);
        }
    };
    fetch(0);                                            // (a padded row's are left over from another call, and not used)
    int seq, pos;
    if (!token_place(a.token_seq, a.token_pos, (int)(row / g.Hq), a.B, a.max_blocks, seq, pos)) return;
    for (int s0 = 0; s0 < a.n_splits; s0 += kBatch) {
        if (s0 > 0) fetch(s0);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (s0 + j < a.n_splits) x.add(ml[j].x, ml[j].y, po[j]);
    }
    const float inv = x.L == 0.f ? 0.f : 1.f / x.L;
    if (kBf16) {
        write_bf16x4(a.out + (row * kD + d) * 2, x.acc * inv);
    } else {
        *(f32x4 *)(a.out + (row * kD + d) * 4) = x.acc * inv;
    }
}

// Ranges of a list.  Four waves to a work-group: two of them share a CU where items fill the chip, and their starts and ends overlap
// (5.4 k bf16 items of 64 blocks, weights in one part yet: 155 us; with eight waves 205), and for few items eight waves are no faster.
//   bf16: a work-group reads a list at what a CU takes from memory, some 80 GB/s, so ranges of eight units, two a wave, for work-groups of
//   their own pay for the launch that combines them (4 us with the gap) where lists are long and few: a call takes, in ranges and in
//   one, for 4 lists of 44 blocks 7.4 and 6.9 us, of 56 7.4 and 7.5, of 80 7.6 and 9.1, of 160 8.7 and 14.7; for 32 of 56 8.0 and 7.9, of 80
//   8.2 and 9.6, of 128 9.5 and 13.2; for 48 of 64 8.7 and 8.7, of 80 9.4 and 10.3, of 160 16.0 and 17.6; for 64 of 80 12.4 and 10.9, of 160
//   19.6 and 17.8.
//   fp32: bound by its own vector work, 400 instructions a block of four rows, so a unit a wave up to two work-groups a CU (24 blocks
//   for each of 20 items 7.7 us a call; in one range of eight waves 9.8).
constexpr int kBaRangeItems = 48, kBaRangeUnits = 28;

// 16 rows of a token and KV head, or 8, to a work-group
int block_attn_groups(int Hq, int Hkv, int esize)
{
    const int G = Hq / Hkv, rows = esize == 2 ? 16 : kBaF32Rows;
    return Hkv * ((G + rows - 1) / rows);
}

int block_attn_splits(int Hq, int Hkv, int esize, int n_tokens, int n_list)
{
    const int64_t items = std::max<int64_t>((int64_t)n_tokens * block_attn_groups(Hq, Hkv, esize), 1);
    const int units = esize == 2 ? (n_list + 1) / 2 : n_list;
    auto ranges = [&](int64_t most, int64_t at_least) {  // up to `most` work-groups, none with fewer units
        return (int)std::max<int64_t>(1, std::min<int64_t>({most / items, (units + at_least - 1) / at_least, 32}));
    };
    if (esize != 2) return ranges(512, 4);
    return items > kBaRangeItems || units <= kBaRangeUnits ? 1 : ranges(256, 8);
}

int block_attn_parts(int Hq, int Hkv, int esize, int n_tokens, int n_list)
{
    int most = 0;                                        // (beyond 256 tokens no list is in ranges)
    for (int n = 1; n <= std::min(n_tokens, 256); ++n) {
        const int splits = block_attn_splits(Hq, Hkv, esize, n, n_list);
        if (splits > 1) most = std::max(most, n * splits);
    }
    return most;
}

template <int kD, bool kSplit>
static hipError_t launch_attn_f32(const Geom &g, const BlockAttnArgs &a, unsigned grid, const Launch &L)
{
    TC_LAUNCH((block_attn_f32_kernel<kD, kSplit>), grid, 0, L, g, a);
    return hipGetLastError();
}

template <bool kSplit, bool kRest>
static hipError_t launch_attn_bf16(const Geom &g, const BlockAttnArgs &a, unsigned grid, const Launch &L)
{
    static PerDeviceOnce configured;
    const hipError_t e = configured.run([] {
        return hipFuncSetAttribute((const void *)block_attn_bf16_kernel<kSplit, kRest>, hipFuncAttributeMaxDynamicSharedMemorySize, kBaWaves * kBaWave);
    });
    if (e != hipSuccess) return e;
    TC_LAUNCH_N((block_attn_bf16_kernel<kSplit, kRest>), grid, 64 * kBaWaves, kBaWaves * kBaWave, L, g, a);
    return hipGetLastError();
}

hipError_t launch_block_attn(const Geom &g, BlockAttnArgs a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    const int groups = block_attn_groups(g.Hq, g.Hkv, g.esize), chunks = groups / g.Hkv;
    const int64_t grid = (int64_t)a.n_tokens * groups * a.n_splits;
    if (grid > kStepMaxGroups) return hipErrorInvalidValue;
    a.splits = FastDiv((uint32_t)a.n_splits);
    a.chunks = FastDiv((uint32_t)chunks);
    a.heads = FastDiv((uint32_t)g.Hkv);
    const bool split = a.n_splits > 1;
    const unsigned n = (unsigned)grid;
    if (g.esize == 2 && g.G <= 8) return split ? launch_attn_bf16<true, true>(g, a, n, L) : launch_attn_bf16<false, true>(g, a, n, L);
    if (g.esize == 2) return split ? launch_attn_bf16<true, false>(g, a, n, L) : launch_attn_bf16<false, false>(g, a, n, L);
    if (g.D == 64) return split ? launch_attn_f32<64, true>(g, a, n, L) : launch_attn_f32<64, false>(g, a, n, L);
    return split ? launch_attn_f32<128, true>(g, a, n, L) : launch_attn_f32<128, false>(g, a, n, L);
}

hipError_t launch_block_merge(const Geom &g, const BlockAttnArgs &a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    const int64_t rows = (int64_t)a.n_tokens * g.Hq, per = 256 / (g.D / 4), blocks = (rows + per - 1) / per;
    if (blocks > kStepMaxGroups) return hipErrorInvalidValue;
    if (g.esize == 2) TC_LAUNCH((block_merge_kernel<true, 128>), (unsigned)blocks, 0, L, g, a);
    else if (g.D == 64) TC_LAUNCH((block_merge_kernel<false, 64>), (unsigned)blocks, 0, L, g, a);
    else TC_LAUNCH((block_merge_kernel<false, 128>), (unsigned)blocks, 0, L, g, a);
    return hipGetLastError();
}

}  // namespace tc
