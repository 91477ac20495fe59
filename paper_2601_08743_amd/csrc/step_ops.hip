// A token step that stays on the GPU: block tables and slot maps from the requests' lengths, queries and keys encoded by
// position with the append to the pool, and 8-bit bounds of the keys of pool blocks.  (Lists by those bounds and the
// attention over them: block_attn.hip.)
#include "arrive.h"
#include "kv_append.h"
#include "step_ops.h"

namespace tc {

// ------------------------------------------------------------------------------------ tables
// Request b holds len_b tokens in have_b = ceil(len_b / 16) blocks and brings new_b; blocks have_b .. ceil((len_b + new_b) / 16)
// are spare ones, taken in order, requests in order.  A block is new to its sequence exactly if its position 0 is among the
// step's tokens, so whoever writes that token's slot writes the table entry, and nobody reads an entry that the step writes.
//
// Two prefix sums over the requests, of new tokens and of blocks; then a thread for every token, which finds its request by bisection
// in LDS, four tokens side by side.  Everything is a few kilobytes: a few tokens are a chain of dependent steps, one work-group and
// one launch (four requests: 3.6 to 4.3 us a call); of many the instructions count, 150 a token, so each of several work-groups repeats the sums
// and writes its part (300 requests, 5.0 k tokens: 5.9 us so, 10 in one work-group).  Where the results are to stand in place of
// the inputs that the other work-groups still read, the sums are a launch of their own and the second takes the lengths from its
// results.
//
// A token whose block is none - a spare id, or an entry under a partial last block, that names no sequence block - is no token to any call
// behind this one, and the status says that there are such.  One work-group knows when it has written its rows; of several one has no rows
// and looks at the blocks instead, while the others write.
template <int kThreads, bool kScan, bool kFill>
__global__ __launch_bounds__(kThreads) void step_tables_kernel(StepTables s)
{
    constexpr int kWaves = kThreads / 64;
    extern __shared__ int32_t lds[];                    // [B + 1] first token, [B] tokens held, [B] first spare block
    __shared__ uint32_t s_tok[2][kWaves], s_blk[2][kWaves], s_bad[2][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, B = s.B;
    int32_t *cu = lds, *held = lds + B + 1, *first = held + B;
    // (a fill launch of its own finds the step's end lengths, and the cursor behind the step's blocks)
    const bool refused = !kScan && s.status[0] < 0;
    const bool alone = kScan && kFill && gridDim.x == 1, sums = kScan && blockIdx.x == gridDim.x - 1;    // (the work-group that writes the sums)
    const int32_t used = kScan ? s.spare_used[0] : s.spare_next[0] - (refused ? 0 : s.status[1]);
    uint64_t n_new = 0;                                 // of the requests so far; a request counts n_tokens at most, a round of them 2^30
    uint32_t n_blocks = 0;
    bool bad = refused || used < 0 || used > s.n_spare;
    int32_t next_new = 0, next_len = 0;                 // the next round's request, ahead
    auto look_up = [&](int b) {
        if (b < B) { next_new = s.new_len[b]; next_len = kScan ? s.seq_len[b] : s.end_len[b]; }
    };
    look_up(tid);
    for (int b0 = 0, round = 0; b0 < B; b0 += kThreads, round ^= 1) {
        const int b = b0 + tid;
        const int32_t fresh = b < B ? next_new : 0, len = b < B ? next_len - (kScan || refused ? 0 : fresh) : 0;
        look_up(b + kThreads);
        bool mine_bad = false;
        if (b < B) {
            mine_bad = len < 0 || fresh < 0 || (int64_t)len + fresh > (int64_t)s.max_blocks * kBlockTokens || fresh > s.n_tokens;
        }
        const uint32_t tok = mine_bad ? 0 : fresh, blk = mine_bad ? 0 : (uint32_t)((len + fresh + 15) >> 4) - (uint32_t)((len + 15) >> 4);
        const uint32_t upto_tok = wave_prefix(tok), upto_blk = wave_prefix(blk);
        const bool any_bad = __any(mine_bad);
        if (lane == 63) { s_tok[round][w] = upto_tok; s_blk[round][w] = upto_blk; s_bad[round][w] = any_bad; }
        __syncthreads();
        uint32_t before_tok = 0, before_blk = 0, all_tok = 0, all_blk = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const uint32_t t = s_tok[round][k], c = s_blk[round][k];
            before_tok += k < w ? t : 0;
            before_blk += k < w ? c : 0;
            all_tok += t;
            all_blk += c;
            bad |= s_bad[round][k] != 0;
        }
        if (b < B) {
            cu[b] = (int32_t)min(n_new + before_tok + upto_tok - tok, (uint64_t)INT32_MAX);
            first[b] = (int32_t)(n_blocks + before_blk + upto_blk - blk);
            held[b] = len;
        }
        n_new += all_tok;
        n_blocks += all_blk;
    }
    int32_t code = bad || n_new > (uint64_t)s.n_tokens ? -1 : 0;
    if (code == 0 && (int32_t)n_blocks > s.n_spare - used) code = -3;
    const int32_t total = code == 0 ? (int32_t)n_new : 0;
    auto is_block = [&](int32_t id) { return id >= s.first_seq && id < s.n_blocks; };
    bool none = false;                                  // a token's block is none
    if (sums) {
        for (int b = tid; b < B; b += kThreads) {       // (a thread's own requests)
            const int32_t fresh = code == 0 ? s.new_len[b] : 0, len = held[b];
            s.cu_new[b] = code == 0 ? cu[b] : 0;
            s.end_len[b] = len + fresh;
            if (!alone && fresh > 0 && (len & 15) != 0) {
                const int32_t id = s.block_table[(int64_t)b * s.max_blocks + (len >> 4)];
                none |= id < 0 || !is_block(entry_bid(id));
            }
        }
        if (!alone && code == 0)
            for (int i = tid; i < (int)n_blocks; i += kThreads) none |= !is_block(s.spare[used + i]);
        if (tid == 0) {
            s.cu_new[B] = total;
            s.spare_next[0] = used + (code == 0 ? (int32_t)n_blocks : 0);
            s.status[1] = code == -1 ? 0 : (int32_t)n_blocks;
        }
    }
    auto report = [&]() {
        const bool any = __any(none);
        __syncthreads();                                // (s_bad was read)
        if (lane == 0) s_bad[0][w] = any;
        __syncthreads();
        if (tid != 0) return;
        int32_t is = code;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) is = s_bad[0][k] != 0 && is == 0 ? 1 : is;
        s.status[0] = is;
    };
    if (sums && !alone) {                               // (of several work-groups the last has no tokens)
        report();
        return;
    }
    if (!kFill) return;
    if (tid == 0) cu[B] = INT32_MAX;
    __syncthreads();
    const int groups = kScan && !alone ? gridDim.x - 1 : gridDim.x;
    constexpr int kSide = 4;
    int top = 1;
    while (2 * top < B) top *= 2;
    for (int n0 = blockIdx.x * (kSide * kThreads) + tid; n0 < s.n_tokens; n0 += groups * (kSide * kThreads)) {
        int lo[kSide] = {0, 0, 0, 0};                   // the last request whose first token is not behind the token
        for (int step = top; step > 0; step >>= 1)
#pragma unroll
            for (int k = 0; k < kSide; ++k) {           // (behind the last request stands a number above all)
                const int mid = min(lo[k] + step, B);
                lo[k] = cu[mid] <= n0 + k * kThreads ? mid : lo[k];
            }
        int32_t pos[kSide], id[kSide];
        int32_t *entry[kSide];
        bool fresh[kSide];
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const int n = n0 + k * kThreads;
            pos[k] = id[k] = -1;
            if (n >= total) continue;
            const int b = lo[k];
            pos[k] = held[b] + (n - cu[b]);
            const int j = pos[k] >> 4, have = (held[b] + 15) >> 4;
            entry[k] = s.block_table + (int64_t)b * s.max_blocks + j;
            fresh[k] = j >= have;
            id[k] = fresh[k] ? s.spare[used + first[b] + (j - have)] : *entry[k];
        }
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const int n = n0 + k * kThreads;
            if (n >= s.n_tokens) continue;
            int64_t slot = -1;
            int32_t full = -1;
            if (n < total) {
                const int32_t block = id[k] < 0 || fresh[k] ? id[k] : entry_bid(id[k]);
                const bool is = is_block(block);
                if (fresh[k] && (pos[k] & 15) == 0) *entry[k] = is ? block : -1;
                if (is) {
                    slot = (int64_t)block * kBlockTokens + (pos[k] & 15);
                    if ((pos[k] & 15) == 15) full = block;
                }
                none |= !is;
            }
            s.slot_map[n] = slot;
            s.token_pos[n] = slot < 0 ? -1 : pos[k];
            s.token_seq[n] = slot < 0 ? -1 : lo[k];
            s.full_block[n] = full;
        }
    }
    if (alone) report();
}

constexpr int kTablesOneWg = 2048;

template <int kThreads, bool kScan, bool kFill>
static hipError_t launch_tables(const StepTables &s, const Launch &L)
{
    static PerDeviceOnce configured;
    const hipError_t e = configured.run([] {
        return hipFuncSetAttribute((const void *)step_tables_kernel<kThreads, kScan, kFill>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                   (3 * kStepMaxSeqs + 1) * (int)sizeof(int32_t));
    });
    if (e != hipSuccess) return e;
    const int fill = (s.n_tokens + 4 * kThreads - 1) / (4 * kThreads), grid = !kFill || s.n_tokens <= kTablesOneWg ? 1 : fill + (kScan ? 1 : 0);
    TC_LAUNCH_N((step_tables_kernel<kThreads, kScan, kFill>), grid, kThreads, (3 * (size_t)s.B + 1) * sizeof(int32_t), L, s);
    return hipGetLastError();
}

hipError_t launch_step_tables(const StepTables &s, const Launch &L)
{
    const bool few = s.B <= 1024;                       // requests: four rounds of 256 at most
    if (s.n_tokens > kTablesOneWg && (s.end_len == s.seq_len || s.spare_next == s.spare_used)) {
        const hipError_t e = launch_tables<1024, true, false>(s, L);
        if (e != hipSuccess) return e;
        return few ? launch_tables<256, false, true>(s, L) : launch_tables<1024, false, true>(s, L);
    }
    if (s.n_tokens > kTablesOneWg ? few : s.B <= 256 && s.n_tokens <= 1024) return launch_tables<256, true, true>(s, L);
    return launch_tables<1024, true, true>(s, L);
}

// ------------------------------------------------------------------------------------ encode and append
// Queries and keys turned by position - pair (j, j + D/2) of every head by pos * theta^(-2j/D), the position being that of the
// axis whose section j falls into - and keys and values written to their slots, in one pass over the rows.  As in the
// re-encoding stitch the turn is a fraction of a revolution taken in fp64, sine and cosine and the rotation are fp32 and the
// result is rounded once.  The fraction is the one of the smaller size, -1/2 to 1/2, so that turns just below a whole one keep their
// bits; what its fp32 form leaves out, up to 2 pi 2^-26, is more than the rounding of a sine, and goes into fp32 results by the
// derivatives.
//
// A work-group a token: its (cos, sin) table in LDS, then a thread for every pair of 16-byte chunks.  The values of a bf16 block are
// stored transposed, two bytes of a token in each row of 32; tokens that go to the same block therefore share its KV heads
// out among their work-groups, each of which takes those heads' rows of all of them and writes whole rows.  Bound: memory, for many tokens
// (2048, 32 / 8 heads, 50 MB: 11.0 us = 4.6 TB/s; 21.8 with two-byte stores); for few the chain that a work-group makes of
// slot, position and row, though all three follow from the token's number (32 tokens 4.6 us).
struct Run { int first, len; };                          // the step's tokens of one block

// The tokens around token n (slot `slot`) that stand behind one another in the same block: one load for the wave.
__device__ __forceinline__ Run run_of(const RopeAppend &a, int n, int64_t slot, int lane)
{
    const int m = n + lane - 15;
    const bool near = lane < 31 && m >= 0 && m < a.n_tokens;
    const int64_t other = near ? a.slot_map[m] : -1, want = slot + (lane - 15);
    const uint32_t same = (uint32_t)__ballot(near && other == want && (want >> 4) == (slot >> 4));
    const uint32_t before = ~same & 0x7fffu, behind = ~(same >> 16) & 0x7fffu;       // the nearest that does not belong
    const int left = before ? 14 - (31 - __builtin_clz(before)) : 15, right = behind ? __builtin_ctz(behind) : 15;
    return Run{n - left, left + 1 + right};
}

template <bool kBf16>
__global__ __launch_bounds__(256) void rope_append_kernel(Geom g, RopeAppend a)
{
    __shared__ float2 cs[64];
    __shared__ uint4 s_v[kBf16 ? kBlockTokens * 17 : 1];  // one head's values, rows of 17 chunks
    const int tid = threadIdx.x, n = blockIdx.x;
    const int64_t slot = a.slot_map[n];
    const int64_t blk = slot >> 4;
    if (slot < 0 || blk < g.first_seq || blk >= g.n_blocks) return;     // a padded row, or no block of a sequence
    const int t = (int)(slot & 15);
    const int half_d = g.D >> 1, cph = g.head_bytes >> 4, half_c = cph >> 1, half_log = __builtin_ctz(half_c);   // (chunks of a head: 16 or 32)
    const int rot_units = (g.Hq + g.Hkv) * half_c;
    auto source = [&](int u) {                           // of a pair of chunks
        const int h = u >> half_log, cc = u & (half_c - 1);
        return (h < g.Hq ? a.q + n * a.q_stride + (int64_t)h * g.head_bytes : a.k + n * a.k_stride + (int64_t)(h - g.Hq) * g.head_bytes) + (cc << 4);
    };
    auto values = [&](int r) { return *(const uint4 *)(a.v + n * a.v_stride + (int64_t)(r >> (half_log + 1)) * g.head_bytes + ((r & (cph - 1)) << 4)); };
    const Run run = run_of(a, n, slot, tid & 63);
    const int t_run = t - (n - run.first);               // the run's first position; 0: the block begins here, and is zero behind the run
    const bool by_run = kBf16 && t_run == 0;
    const int v_units = by_run ? 0 : g.Hkv * cph;
    // a thread's first chunks, requested while the turns are computed
    uint4 x, y, v;
    if (tid < rot_units) {
        const char *src = source(tid);
        x = *(const uint4 *)src;
        y = *(const uint4 *)(src + (half_c << 4));
    }
    if (tid < v_units) v = values(tid);
    if (tid < half_d) {
        int axis = 0;
        while (tid >= a.section_end[axis]) ++axis;
        const double turns = (double)a.pos[(int64_t)axis * a.n_tokens + n] * (a.rev_coarse[tid >> 3] * a.rev_fine[tid & 7]);
        const double part = turns - rint(turns);
        const float frac = (float)part;
        float sn, c;
        if (kBf16) {
            sn = __builtin_amdgcn_sinf(frac);
            c = __builtin_amdgcn_cosf(frac);
        } else {
            const float left = 6.28318531f * (float)(part - (double)frac);
            float sn0, c0;
            sincospif(2.0f * frac, &sn0, &c0);
            sn = fmaf(left, c0, sn0);
            c = fmaf(-left, sn0, c0);
        }
        cs[tid] = make_float2(c, sn);
    }
    char *kd = g.pool + (int64_t)a.layer * g.layer_stride + blk * g.block_bytes;
    char *vd = kd + (g.block_bytes >> 1);
    constexpr int kElems = kBf16 ? 8 : 4;
    __syncthreads();
    for (int u = tid; u < rot_units; u += 256) {
        const int h = u >> half_log, cc = u & (half_c - 1);
        char *dst = (h < g.Hq ? a.q_out + ((int64_t)n * g.Hq + h) * g.head_bytes : kd + (int64_t)((h - g.Hq) * kBlockTokens + t) * g.head_bytes) + (cc << 4);
        if (u != tid) {
            const char *src = source(u);
            x = *(const uint4 *)src;
            y = *(const uint4 *)(src + (half_c << 4));
        }
        turn_chunk<kBf16>(x, y, cs + cc * kElems);
        *(uint4 *)dst = x;
        *(uint4 *)(dst + (half_c << 4)) = y;
    }
    for (int r = tid; r < v_units; r += 256) {
        if (r != tid) v = values(r);
        const int h = r >> (half_log + 1), cc = r & (cph - 1);
        if (!kBf16) {
            *(uint4 *)(vd + (int64_t)(h * kBlockTokens + t) * g.head_bytes + (cc << 4)) = v;
        } else {
            const unsigned e[4] = {v.x, v.y, v.z, v.w};
            unsigned short *v16 = (unsigned short *)vd;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v16[((int64_t)(h * g.D + cc * 8 + k) << 4) + vperm(t)] = (unsigned short)(e[k >> 1] >> ((k & 1) * 16));
        }
    }
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (by_run) {
        // heads n - run.first, .. + run.len, ..: 16 chunks of each token, then 8 tokens of each row
        for (int h = n - run.first; h < g.Hkv; h += run.len) {
            const int tok = tid >> 4, c = tid & 15;
            uint4 v = zero;
            if (tok < run.len) v = *(const uint4 *)(a.v + (run.first + tok) * a.v_stride + (int64_t)h * 256 + (c << 4));
            __syncthreads();
            s_v[tok * 17 + c] = v;                       // (the run begins the block: a token's position is its number)
            __syncthreads();
            const unsigned short *v16 = (const unsigned short *)s_v;
            const int d = tid >> 1, half = tid & 1;
            unsigned e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t0 = vperm(8 * half + 2 * k), t1 = vperm(8 * half + 2 * k + 1);
                e[k] = v16[t0 * 136 + d] | ((unsigned)v16[t1 * 136 + d] << 16);
            }
            *(uint4 *)(vd + (int64_t)h * 4096 + tid * 16) = make_uint4(e[0], e[1], e[2], e[3]);
        }
    }
    if (t == 0 && run.len < kBlockTokens) {
        const int chunks = (kBlockTokens - run.len) * cph;               // behind one another in a head's rows
        for (int h = 0; h < g.Hkv; ++h) {
            const int64_t at = (int64_t)(h * kBlockTokens + run.len) * g.head_bytes;
            for (int c = tid; c < chunks; c += 256) {
                *(uint4 *)(kd + at + (c << 4)) = zero;
                if (!kBf16) *(uint4 *)(vd + at + (c << 4)) = zero;
            }
        }
    }
}

hipError_t launch_rope_append(const Geom &g, const RopeAppend &a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    if (g.esize == 2) TC_LAUNCH(rope_append_kernel<true>, a.n_tokens, 0, L, g, a);
    else TC_LAUNCH(rope_append_kernel<false>, a.n_tokens, 0, L, g, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ digests
// Bounds of a block's keys, channel by channel, in 8 bits with one power of two for all: hi = max over the block's tokens, lo =
// min; e the smallest integer, -126 at least, with max(|hi|, |lo|) <= 127 * 2^e; stored are ceil(hi / 2^e) and
// floor(lo / 2^e), so that they stay bounds, and e (127 where some key is not finite).  Dividing by a power of two is exact, but for
// quotients too small for fp32, and those are bounded by 1 as any up to 1 are: the bytes follow from the keys alone, whatever computes
// them.
//
// One read of the keys: a wave takes one block of one KV head, 16 rows that stand behind one another, and holds 16 bytes of each
// fourth (or second) row in a lane.  Maximum and minimum are taken on the bits, made to order like integers, in which
// an infinity or a NaN is an extreme of its sign and so is seen at the end; in that order the complement stands for the negative
// value, so the lower bounds are upper bounds too from there on.  Between lanes two registers at a time are combined by
// exchanging rows, after which each lane holds its own two or four bounds and makes bytes of those alone: half the vector
// work of a reduction in which every lane ends up with all.  Bound: memory.  6168 blocks, 8 heads, two layers, 404 MB read and 25
// written: 85.5 us = 5.0 TB/s, a large copy's 5.2 (68 us without the writes; loops over several pairs a wave, with the
// next one's loads ahead, 90 .. 95).
template <bool kBf16>
struct Sortable;
template <>
struct Sortable<true> {                                  // two bf16 in a register
    typedef short vec __attribute__((ext_vector_type(2)));
    static constexpr int kPerWord = 2;
    __device__ static __forceinline__ vec flip(vec x) { return x ^ ((x >> 15) & (short)0x7fff); }
    __device__ static __forceinline__ float value(vec x, int i) { return __uint_as_float((uint32_t)(unsigned short)flip(x)[i] << 16); }
};
template <>
struct Sortable<false> {
    typedef int vec __attribute__((ext_vector_type(1)));
    static constexpr int kPerWord = 1;
    __device__ static __forceinline__ vec flip(vec x) { return x ^ ((x >> 31) & 0x7fffffff); }
    __device__ static __forceinline__ float value(vec x, int) { return __int_as_float(flip(x)[0]); }
};

// Two registers, each to be combined over lanes kApart apart (16 or 32): the first one's result in the lower lanes, the second one's in
// the others.
template <int kApart, typename V>
__device__ __forceinline__ V max_both(V x, V y)
{
    const unsigned u = __builtin_bit_cast(unsigned, x), v = __builtin_bit_cast(unsigned, y);
    unsigned p, q;
    if (kApart == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, v, false, false);
        p = r[0]; q = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, v, false, false);
        p = r[0]; q = r[1];
    }
    return __builtin_elementwise_max(__builtin_bit_cast(V, p), __builtin_bit_cast(V, q));
}

template <bool kBf16, int kLanes>                        // kLanes: 16-byte chunks of a key row, 16 or 32
__global__ __launch_bounds__(256) void digest_kernel(Geom g, DigestArgs a)
{
    typedef typename Sortable<kBf16>::vec vec;
    constexpr int kRowsAt = 64 / kLanes, kLoads = kBlockTokens / kRowsAt, kPer = Sortable<kBf16>::kPerWord;
    constexpr int kWords = kLanes == 16 ? 2 : 4, kOwn = kWords * kPer;       // bounds a lane ends up with
    const int lane = threadIdx.x & 63, row = lane / kLanes, c = lane % kLanes;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int i = a.heads(unit), h = unit - i * g.Hkv, layer = a.l0 + blockIdx.y;
    if (i >= a.n) return;
    const int32_t entry = a.entries[i];
    const int bid = entry_bid(entry), last = kBlockTokens - 1 - entry_pad(entry);        // the last row that holds a key
    if (entry < 0 || bid >= g.n_blocks || bid < a.first_block) return;
    const char *k = g.pool + (int64_t)layer * g.layer_stride + (int64_t)bid * g.block_bytes + (int64_t)h * kBlockTokens * g.head_bytes;
    union { uint4 u; vec v[4]; } x[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) x[j].u = *(const uint4 *)(k + min(row + j * kRowsAt, last) * g.head_bytes + c * 16);
    vec hi[4], lo[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) hi[w] = lo[w] = Sortable<kBf16>::flip(x[0].v[w]);
#pragma unroll
    for (int j = 1; j < kLoads; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const vec y = Sortable<kBf16>::flip(x[j].v[w]);
            hi[w] = __builtin_elementwise_max(hi[w], y);
            lo[w] = __builtin_elementwise_min(lo[w], y);
        }
    vec own[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) own[w] = max_both<kLanes>(hi[w], ~lo[w]);
    if (kLanes == 16) {
#pragma unroll
        for (int w = 0; w < 2; ++w) own[w] = max_both<32>(own[w], own[w + 2]);
    }
    const bool is_lo = (lane & kLanes) != 0;
    const int at = (is_lo ? g.D : 0) + c * (4 * kPer) + (kLanes == 16 ? (lane >> 5) * kOwn : 0);
    float bound[kOwn];                                   // upper bounds, and lower ones negated
    uint32_t size = 0;                                   // of the largest, as bits (they order like the sizes)
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        bound[e] = Sortable<kBf16>::value(own[e / kPer], e % kPer);
        size = max(size, __float_as_uint(bound[e]) & 0x7fffffffu);
    }
    size = wave_max(size);
    const bool finite = size < 0x7f800000u;
    const int e = finite ? step_exponent(__uint_as_float(size)) : 127;
    const float by = finite ? step_pow2(-e) : 0.f;
    uint32_t bytes = 0;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        const float y = fmaxf(ceilf(bound[q] * by), (int)__float_as_uint(bound[q]) > 0 ? 1.f : -INFINITY);
        bytes |= ((uint32_t)(finite ? (int)(is_lo ? -y : y) : 0) & 0xffu) << (8 * q);
    }
    const int64_t to = ((int64_t)layer * g.Hkv + h) * g.n_blocks + bid;
    int8_t *dst = a.digests + to * 2 * g.D + at;
    if (kOwn == 4) *(uint32_t *)dst = bytes;
    else *(uint16_t *)dst = (uint16_t)bytes;
    if (lane == 0) a.digests[a.exps_at + to] = (int8_t)e;
}

hipError_t launch_digest(const Geom &g, DigestArgs a, int l1, const Launch &L)
{
    if (a.n == 0 || l1 <= a.l0) return hipSuccess;
    const int64_t units = (int64_t)a.n * g.Hkv;
    if ((units + 3) / 4 > kStepMaxGroups) return hipErrorInvalidValue;
    a.heads = FastDiv((uint32_t)g.Hkv);
    const dim3 grid((unsigned)((units + 3) / 4), l1 - a.l0);
    if (g.esize == 2) TC_LAUNCH((digest_kernel<true, 16>), grid, 0, L, g, a);
    else if (g.D == 64) TC_LAUNCH((digest_kernel<false, 16>), grid, 0, L, g, a);
    else TC_LAUNCH((digest_kernel<false, 32>), grid, 0, L, g, a);
    return hipGetLastError();
}

}  // namespace tc
