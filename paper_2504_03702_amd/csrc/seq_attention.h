// What the kernels of ps_attention_forward() and ps_attention_backward() share: arguments, sequences, tiles in LDS and their
// products on the matrix cores, which tiles a block of rows sees, scores.
//
// The rows of a key head's queries are those of all its heads, r = G i + g for row i and head g of the G: keys and values are
// read once for all of them, and their gradients add the heads up without a word of traffic.  "Fixed" rows belong to lanes: a
// wavefront owns 32, a lane one of them (and the other half of the wavefront the same 32), in registers.  "Passing" rows come
// by in tiles through LDS.  A product of a tile with the fixed rows (v_mfma_f32_32x32x16_bf16, v_mfma_f32_32x32x2_f32; A = the
// tile, B = the fixed rows) leaves a lane with the scores of its own row: accumulator element e of half-wavefront h is passing
// row 8 (e / 4) + 4 h + e % 4 of 32.  Row maxima and sums are then a lane's own, and the weights are the B operand of the second
// product (A = the tile's transpose) as they stand: the order of the contracted rows is free, so it is the accumulator's.
#pragma once

#include <type_traits>

#include "device_util.h"
#include "internal.h"

namespace seqatt {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int FIXED = 128;             // fixed rows of a workgroup, 32 a wavefront
constexpr int FEW = 512;               // keys that a row sees where the rounding of their weights' gradients does not average out
constexpr int DOC_BLOCK = 64;          // tokens to a summary of their documents

struct Args {
    const void *q, *k, *v, *out, *dout;
    void *out_w, *dq, *dk, *dv;
    void* rest_w;                      // bf16 calls: what rounding left of out, dense, or null
    const void* rest;
    float* lse_w;
    const float* lse;
    const int32_t *q_offsets, *k_offsets, *k_lengths, *q_start, *prefix, *q_docs, *k_docs;
    const float* slopes;
    int2 *q_blocks, *k_blocks;         // smallest and largest document of every DOC_BLOCK tokens
    float *row_lse, *row_delta;        // [heads][n_q]: lse in powers of two (+infinity for rows that see nothing); dout . out
    float* part_o;                     // [parts][n_q * heads][head_dim]: unnormalised out, or dq
    float2* part_ml;                   // [parts][n_q * heads]: reference exponent, sum
    float *part_dk, *part_dv;          // [key_parts][n_k * kv_heads][head_dim]
    ps_status* status;
    ps_strides qs, ks, vs, os, gs, dqs, dks, dvs;
    int64_t n_q, n_k;
    int32_t n_seq, seq0, seqs, together;   // sequences; the first one of a launch, how many it has, how many of them take turns
    int32_t heads, kv_heads, head_dim, group, max_q, max_k, causal;
    int32_t row_blocks;                // blocks of FIXED rows that the grid has for every sequence
    int32_t parts, part_tiles;         // shares of a row block's key tiles, and tiles of a share
    int32_t key_parts, key_part_tiles; // shares of a key block's row tiles
    int32_t listed;                    // workgroups find their work by adding up what there is
    int32_t few;                       // at most 32 rows to a key head
    int32_t tile, key_tile;            // rows of a tile that passes by fixed queries, by fixed keys
    uint32_t by_group;                 // 2^32 / group + 1 (group > 1)
    float scale, cap;
    float slope_by, cap_in;            // see Row and Cap
    // ps_local_attention_*() alone, whose kernels are the same with LOCAL:
    int32_t left, right, sinks;        // a row's window, and the first keys that it sees all the same
    int32_t local;                     // 1
    int32_t sorted;                    // sequences' work goes by their lengths: the longest first, if workgroups find it by adding up
    int32_t few_first, few_last;       // see few_in_window()
    int32_t sink_blocks, sink_parts, sink_part_tiles;   // those in blocks of 32, shares of their tiles of 32 rows
    float *sink_dk, *sink_dv;          // [sink_parts][n_seq][sink_blocks * 32][kv_heads][head_dim]
    const float* table;                // [heads][2 reach + 1]: the learned bias of a distance, null without one (see Learned)
    const int32_t* bucket_words;       // [2 reach + 1]: where in a lane's sums the distance's bucket is
    float* bias_parts;                 // [parts][blocks of rows][buckets][heads]: sums of a bucket's gradients, null if not wanted
    int64_t bias_blocks;
    int32_t reach, n_buckets, sum_columns;   // sums of a bucket that a wavefront has: 64, or 32
    int32_t bias_width, bias_words;    // distances that a head has in a tile; words of all heads of a tile, in whole wavefronts
    uint32_t by_width;                 // 2^32 / bias_width + 1
};

// The arguments read again where they are used, by what the compiler takes for another address each time: what is wanted once a tile and no more does not wait
// in scalar registers, of which the gradients' kernels have too few.  (All kernels have them as their first argument.)
typedef const __attribute__((address_space(4))) Args* ArgsAgain;
__device__ __forceinline__ ArgsAgain again() {
    ArgsAgain a = (ArgsAgain)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
}

// (scalars: the compiler does not see that all lanes have the same, and would count and address tiles in vector registers)
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Seq {
    int q0, qn, k0, kn, start, prefix;
};

// Sequence s, checked against the tensors and the host's bounds; false if it is faulty.  All its words are asked for at once, without a
// branch: a workgroup of a short sequence waits for them a tenth of its time.
__device__ __forceinline__ bool sequence(const Args& a, int s, Seq& r) {
    typedef const __attribute__((address_space(4))) int32_t* Words;       // (written by no kernel that reads them: scalar loads)
    const int32_t *lengths = a.k_lengths ? a.k_lengths : a.k_offsets, *starts = a.q_start ? a.q_start : a.q_offsets, *prefixes = a.prefix ? a.prefix : a.q_offsets;
    const Words qo = (Words)(a.q_offsets + s), ko = (Words)(a.k_offsets + s);
    const int q0 = qo[0], q1 = qo[1], k0 = ko[0], k1 = ko[1], length = *(Words)(lengths + s), start = *(Words)(starts + s), prefix = *(Words)(prefixes + s);
    r.q0 = q0;
    r.k0 = k0;
    r.qn = (int)((unsigned)q1 - (unsigned)q0);
    const int room = (int)((unsigned)k1 - (unsigned)k0);
    r.kn = a.k_lengths ? length : room;
    r.start = a.q_start ? start : (int)((unsigned)r.kn - (unsigned)r.qn);
    r.prefix = a.prefix ? prefix : 0;
    // (ends before starts: a negative offset, or one that falls, fails one of these; places and distances are 32 bits)
    const bool offsets = (q0 >= 0) & (q1 >= q0) & (q1 <= a.n_q) & (k0 >= 0) & (k1 >= k0) & (k1 <= a.n_k);
    return offsets & (r.kn >= 0) & (r.kn <= room) & (r.kn <= a.max_k) & (r.qn <= a.max_q) & (r.start >= -(1 << 30)) & (r.start <= 1 << 30);
}

__device__ __forceinline__ unsigned over_group(const Args& a, unsigned r) { return a.group == 1 ? r : __umulhi(r, a.by_group); }

// Keys in front of this one are seen from a place, if their documents are.  (The largest place, 2^30 rows from 2^30 on, has none behind it.)
__device__ __forceinline__ int seen_end(const Args& a, const Seq& q, int place) {
    return a.causal ? min(q.kn, max(min(place, q.kn) + 1, q.prefix)) : q.kn;
}

// With a window, keys from `window_begin` on and in front of `seen_to`, and those in front of a.sinks that are in front of seen_to too.  Both never
// fall from place to place.  (A window without an end has 2^31 - 1 places.)
__device__ __forceinline__ int window_begin(const Args& a, int place) { return (int)max((int64_t)0, (int64_t)place - a.left); }
template <bool LOCAL>
__device__ __forceinline__ int seen_to(const Args& a, const Seq& q, int place) {
    const int end = seen_end(a, q, place);
    return LOCAL ? min(end, max((int)min((int64_t)q.kn, (int64_t)place + a.right + 1), a.sinks)) : end;
}
// Whether some of the rows from place `near` to place `far` have FEW keys or less in their windows: the first ones, whose windows begin with the keys, or the last ones, whose
// windows end with them, or all rows (few_first is then above all places).  The arguments as they are, or read again.  (A place is from -2^30 to 2^31 - 1, keys are 2^30 at most.)
template <typename A>
__device__ __forceinline__ bool few_in_window(const A& a, const Seq& q, int near, int far) {
    return q.kn <= FEW || near < a.few_first || far - q.kn >= a.few_last;
}

// Tiles of keys that some of the FIXED rows from r0 on may see: `tiles` of them, `front` from the first on and the others `skip` further on (without
// a window there is nothing between).
struct Span {
    int tiles, front, skip;
    template <bool LOCAL>
    __device__ __forceinline__ int at(int t) const { return LOCAL && t >= front ? t + skip : t; }
};
template <bool LOCAL>
__device__ __forceinline__ Span key_tiles(const Args& a, const Seq& q, int r0) {
    const int far = q.start + (int)over_group(a, min(r0 + FIXED, q.qn * a.group) - 1);
    const int end = max(0, seen_to<LOCAL>(a, q, far));
    Span s = {(end + a.tile - 1) / a.tile, 0, 0};
    if (LOCAL) {
        s.front = (min(a.sinks, end) + a.tile - 1) / a.tile;
        s.skip = max(0, min(window_begin(a, q.start + (int)over_group(a, r0)) / a.tile, s.tiles) - s.front);
        s.tiles -= s.skip;
    }
    return s;
}
// Tiles of rows, from `first` on and in front of the returned one, that may see some of the FIXED keys from k0 on (in their windows: the first keys
// have a launch of their own).  Shares are of these.
template <bool LOCAL>
__device__ __forceinline__ int row_tiles(const Args& a, const Seq& q, int k0, int& first) {
    const int rows = q.qn * a.group, n = (rows + a.key_tile - 1) / a.key_tile;
    first = a.causal && k0 >= q.prefix ? (int)min((int64_t)n, max((int64_t)0, (int64_t)(k0 - q.start) * a.group / a.key_tile)) : 0;
    if (!LOCAL) return n;
    auto tile_of = [&](int64_t place) { return (int)min((int64_t)n, max((int64_t)0, (place - q.start) * a.group / a.key_tile)); };
    first = max(first, tile_of((int64_t)k0 - a.right));
    const int64_t behind = (int64_t)min(k0 + FIXED, q.kn) + a.left - q.start;   // the first token that none of them is seen by
    return max(first, behind >= q.qn ? n : behind <= 0 ? 0 : (int)((behind * a.group + a.key_tile - 1) / a.key_tile));
}
__device__ __forceinline__ int shares(int tiles, int parts, int part_tiles) { return max(1, min(parts, (tiles + part_tiles - 1) / part_tiles)); }

// A workgroup's part of a launch over blocks of rows (of keys, with KEYS) and shares of their tiles.
// Sequence and block as the grid counts them: `together` sequences take turns, block by block, then the next so many.  Blocks come in order
// of their work, most first.  In a launch of few blocks all sequences take turns, so that the last to start are short (two rows of 8192
// tokens, forwards / queries' / keys' gradients: 99 / 159 / 171 us one after the other, 85 / 144 / 160 in turns; 16 x 2048, keys' eight at a
// time 1035, 977); in one of many only as many as fill the chip, so that blocks that run at a time read the same keys from the caches
// (16 x 2048, forwards / queries': 390 / 589 us two at a time, 438 / 665 sixteen).
inline int32_t turns(int64_t blocks_a_seq, int32_t seqs) {
    if (blocks_a_seq * seqs <= 2048) return seqs;
    return (int32_t)(blocks_a_seq >= 512 ? 1 : 512 / blocks_a_seq);
}
struct Work {
    int s, hk, block, part;
};
template <bool KEYS, bool LOCAL>
__device__ __forceinline__ int shares_of(const Args& a, const Seq& q, int block) {
    const int n = KEYS ? q.kn : q.qn * a.group;
    if (block * FIXED >= n) return 0;
    if ((KEYS ? a.key_parts : a.parts) == 1) return 1;
    int first = 0;
    const int tiles = KEYS ? row_tiles<LOCAL>(a, q, block * FIXED, first) : key_tiles<LOCAL>(a, q, block * FIXED).tiles;
    return shares(tiles - first, KEYS ? a.key_parts : a.parts, KEYS ? a.key_part_tiles : a.part_tiles);
}
// a.listed (at most 64 sequences of at most 64 blocks): the grid has a workgroup for what there could be, and the first so many take
// what there is, found by adding it up a sequence to a lane.  Counted as the grid counts, what there is lay anywhere among it, and
// three or more long workgroups on one unit beside empty ones (8 sequences of 100 to 1023 tokens, 408 workgroups of 2048 with work to do: 26 to
// 40 tiles on the fullest units, 10 on average; forwards / queries' / keys' gradients in fp32 with heads of 80 128 / 173 / 293 us, 77 / 104 / 157
// added up).
template <bool KEYS, bool LOCAL>
__device__ __forceinline__ bool look_for_work(const Args& a, Seq& q, Work& w) {
    const int blocks = KEYS ? (a.max_k + FIXED - 1) / FIXED : a.row_blocks, parts = KEYS ? a.key_parts : a.parts, lane = threadIdx.x & 63;
    unsigned id = blockIdx.x;
    w.hk = id % a.kv_heads;
    id /= a.kv_heads;
    if (!a.listed) {
        w.part = id % parts;
        id /= parts;
        const unsigned turn = id / (unsigned)(blocks * a.together), first = turn * a.together, rest = id - first * blocks;
        const unsigned here = min((unsigned)a.together, a.seqs - first);
        w.block = rest / here;
        if (!KEYS) w.block = blocks - 1 - w.block;
        w.s = a.seq0 + first + rest % here;
        if (!sequence(a, w.s, q)) {
            if (!KEYS && threadIdx.x == 0 && w.hk == 0 && w.block == 0 && w.part == 0) report_fault(a.status, PS_ST_BAD_LENGTH, w.s);
            return false;
        }
        return w.block * FIXED < (KEYS ? q.kn : q.qn * a.group);
    }
    auto sum_in_front = [&](int v, int& upto) {                            // over the lanes
        upto = v;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int u = __shfl_up(upto, o, 64);
            if (lane >= o) upto += u;
        }
        return upto - v;
    };
    Seq mine = {};
    const bool there = lane < a.seqs, good = there && sequence(a, a.seq0 + lane, mine);
    if (there && !good && !KEYS && blockIdx.x == 0 && threadIdx.x < 64) report_fault(a.status, PS_ST_BAD_LENGTH, a.seq0 + lane);
    int n = 0, upto;
    if (LOCAL && good && parts == 1)
        n = ((KEYS ? mine.kn : mine.qn * a.group) + FIXED - 1) / FIXED;
    else if (good)
        for (int b = 0; b < blocks; ++b) {
            const int c = shares_of<KEYS, LOCAL>(a, mine, b);
            if (c == 0) break;
            n += c;
        }
    // LOCAL: the longest sequences first, in eighths of the longest there can be, so that the last to start are short (64 sequences of 4 to 512 tokens under a bias, forwards / queries' / keys'
    // gradients 46 / 98 / 62 us in the grid's order, 39 / 80 / 49 this way)
    int of = lane;
    if (LOCAL && a.sorted) {
        const int eighth = good ? (int)((float)(KEYS ? mine.qn : mine.kn) * (7.99f / (float)max(KEYS ? a.max_q : a.max_k, 1))) : -1;
        int rank = 0, longer = 0;
#pragma unroll
        for (int e = 7; e >= -1; --e) {
            const uint64_t same = __ballot(eighth == e);
            if (eighth == e) rank = longer + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(same >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)same, 0));
            longer += __popcll(same);
        }
        n = __builtin_amdgcn_ds_permute(4 * rank, n);
        of = __builtin_amdgcn_ds_permute(4 * rank, lane);
    }
    const int front = sum_in_front(n, upto), s = __popcll(__ballot(upto <= (int)id));
    if (s >= a.seqs) return false;
    id -= __builtin_amdgcn_readlane(front, s);
    w.s = a.seq0 + (LOCAL ? __builtin_amdgcn_readlane(of, s) : s);
    sequence(a, w.s, q);
    const int own = ((KEYS ? q.kn : q.qn * a.group) + FIXED - 1) / FIXED;
    if (LOCAL && parts == 1) {
        w.block = KEYS ? id : own - 1 - id;
        w.part = 0;
        return true;
    }
    const int b = KEYS ? lane : own - 1 - lane;   // (most work first)
    const int in_front = sum_in_front(b >= 0 ? shares_of<KEYS, LOCAL>(a, q, b) : 0, upto), at = __popcll(__ballot(upto <= (int)id));
    w.block = KEYS ? at : own - 1 - at;
    w.part = (int)id - __builtin_amdgcn_readlane(in_front, at);
    return true;
}

// The same, as scalars: the compiler does not see that all lanes have found the same.
template <bool KEYS, bool LOCAL>
__device__ __forceinline__ bool find_work(const Args& a, Seq& q, Work& w) {
    if (!look_for_work<KEYS, LOCAL>(a, q, w)) return false;
    int* const x[] = {&q.q0, &q.qn, &q.k0, &q.kn, &q.start, &q.prefix, &w.s, &w.hk, &w.block, &w.part};
#pragma unroll
    for (int i = 0; i < 10; ++i) *x[i] = __builtin_amdgcn_readfirstlane(*x[i]);
    return true;
}

// Where sequence summaries of documents start: sequences never share one.
__device__ __forceinline__ int64_t doc_block0(int first_token, int s) { return first_token / DOC_BLOCK + s; }

// ---- tiles in LDS: rows of DP elements (head_dim and zeros), 16-byte chunks swizzled so that 16 rows' equal chunks, and the
// transposing reads, fall into different banks -------------------------------------------------------------------------------
constexpr int tile_rows(int eb) { return eb == 2 ? 64 : 32; }
// Rows of a tile that passes by fixed keys: for heads of 128 half as many, which leaves room for a workgroup's values (below).
constexpr int key_tile_rows(int eb, int dp) { return eb == 2 && dp < 128 ? 64 : 32; }
// Rows of a tile that passes by fixed queries for their gradients: under a learned bias half as many for heads of 128, which leaves room for its sums.
constexpr int query_tile_rows(int eb, int dp, bool biased) { return biased && eb == 2 && dp == 128 ? 32 : tile_rows(eb); }
constexpr int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : 128; }   // features of a tile

template <typename T, int DP, int R = tile_rows(sizeof(T))>
struct Tile {
    static constexpr int EB = sizeof(T), ROWB = DP * EB, ROWS = R, BLOCKS = ROWS / 32, BYTES = ROWS * ROWB;
    static constexpr int CPR = ROWB / 16, PER_THREAD = BYTES / 16 / 256, EPC = 16 / EB, NF = ROWB / 32, NA = DP / 32;
    // The swizzle turns as many low bits of a chunk's number as rows of this length leave free (rows are multiples of 2^BITS chunks).
    static constexpr int BITS = ROWB % 256 == 0 ? 4 : ROWB % 128 == 0 ? 3 : 2, LOW = (1 << BITS) - 1;
    static __device__ __forceinline__ constexpr int swz(int r) {
        if (EB == 4 && BITS == 4) return ((r >> 2) & 1) << 3 | (r & 3) << 1 | ((r >> 3) & 1);
        if (EB == 4) return (r >> 1) & 7;
        if (BITS == 3) return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) | ((r >> 3) & 1) << 1;
        if (BITS == 2) return (r >> 2) & 3;
        return (r & 3) << 2 | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int r, int chunk) { return r * ROWB + ((chunk ^ swz(r)) << 4); }
    // at(r, chunk + more) from at(r, chunk), for chunk < the power of two that `more` is a multiple of.
    static __device__ __forceinline__ int further(int at, int more) { return (at ^ ((more & LOW) << 4)) + ((more & ~LOW) << 4); }
};

// A lane's fixed row: chunks 2 i + half.
template <typename T, int DP>
struct Fixed {
    static constexpr bool READS = false;
    uint4 c[Tile<T, DP>::NF];
    __device__ __forceinline__ const uint4& chunk(int i, int) const { return c[i]; }
    // This half-wavefront's share of the product with another row that is laid out the same.
    __device__ __forceinline__ float share(const Fixed& o) const {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < Tile<T, DP>::NF; ++i) {
            const T *x = (const T*)&c[i], *y = (const T*)&o.c[i];
#pragma unroll
            for (int j = 0; j < Tile<T, DP>::EPC; ++j) sum = fmaf((float)x[j], (float)y[j], sum);
        }
        return sum;
    }
    // `row` has to be readable whether `valid` or not
    __device__ __forceinline__ void load(const T* row, bool valid, int head_dim, int half) {
#pragma unroll
        for (int i = 0; i < Tile<T, DP>::NF; ++i) {
            const int e = (2 * i + half) * Tile<T, DP>::EPC;
            const uint4 x = *(const uint4*)(row + min(e, head_dim - Tile<T, DP>::EPC));
            const bool is = valid && e < head_dim;
            c[i] = make_uint4(is ? x.x : 0, is ? x.y : 0, is ? x.z : 0, is ? x.w : 0);
        }
    }
};

// Lane-constant parts of the LDS addresses.
template <typename T, int DP>
struct Lanes {
    int row, turned;
    __device__ __forceinline__ Lanes(int lane) {
        using L = Tile<T, DP>;
        const int half = lane >> 5, r = lane & 31;
        row = L::at(r, half);
        if (L::EB == 2) {
            const int li = lane & 15, g = (lane >> 4) & 1, rl = 4 * half + (li >> 2);
            turned = L::at(rl, 2 * g + ((li & 3) >> 1)) + (li & 1) * 8;
        } else {
            turned = L::at(4 * half, r >> 2) + (r & 3) * 4;
        }
    }
};

#define SEQATT_LDS __attribute__((address_space(3)))

// An address that the compiler takes for a new one: what is made of it by a few XORs is then made again where it is used, instead of
// in registers throughout the loop (16 of them for heads of 128, which the accumulators need).
template <int ROWB>
__device__ __forceinline__ int anew(int at) {
    if (ROWB > 128) asm volatile("" : "+v"(at));
    return at;
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }

// Fixed rows in LDS instead, the wavefront's own 32 of them: where registers are short.
template <typename T, int DP>
struct FixedInLds {
    static constexpr bool READS = true;
    const unsigned char* rows;
    __device__ __forceinline__ FixedInLds(unsigned char* to, const Fixed<T, DP>& f, const Lanes<T, DP>& l) : rows(to) {
#pragma unroll
        for (int i = 0; i < Tile<T, DP>::NF; ++i) *(uint4*)(to + Tile<T, DP>::further(l.row, 2 * i)) = f.c[i];
    }
    __device__ __forceinline__ uint4 chunk(int i, int row) const { return *(const uint4*)(rows + Tile<T, DP>::further(row, 2 * i)); }   // row: Lanes'
};

// What a step reads from LDS is read in one go before its products: left alone the compiler, short of registers, reads for each
// product when its turn comes and waits for LDS every time (heads of 128, gradients of keys: 60 % of a wavefront's time).
__device__ __forceinline__ void reads_first() { __builtin_amdgcn_sched_barrier(0); }

__device__ __forceinline__ f32x16 no_start() {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    return s;
}

// 32 passing rows (block b of the tile) times the fixed rows, and what the sums start from.
template <typename T, int DP, typename F>
__device__ __forceinline__ f32x16 dot(const unsigned char* tile, int b, const F& f, const Lanes<T, DP>& l, const f32x16& start = no_start()) {
    using L = Tile<T, DP>;
    constexpr int N = F::READS ? 2 : L::NF <= 8 ? L::NF : L::NF / 2;
    const int at = anew<L::ROWB>(l.row);
    f32x16 s = start;
#pragma unroll
    for (int n = 0; n < L::NF; n += N) {
        uint4 as[N], cs[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            as[i] = *(const uint4*)(tile + b * 32 * L::ROWB + L::further(at, 2 * (n + i)));
            cs[i] = f.chunk(n + i, at);
        }
        reads_first();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint4 a = as[i], c = cs[i];
            if constexpr (L::EB == 2) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(c), s, 0, 0, 0);
            } else {
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(c.x), s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(c.y), s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(c.z), s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(c.w), s, 0, 0, 0);
            }
        }
    }
    return s;
}

// Two such products, taken in turns: neither waits for its own last step, or for LDS more than once (documents in two rows of 8192, forwards
// 108 -> 100 us).
template <typename T, int DP, typename F, typename G>
__device__ __forceinline__ void dots(const unsigned char* tile, int b, const F& f, f32x16& s, const unsigned char* tile2, int b2, const G& g, f32x16& s2,
                                     const Lanes<T, DP>& l, const f32x16& start = no_start(), const f32x16& start2 = no_start()) {
    using L = Tile<T, DP>;
    if constexpr (L::EB == 4 || F::READS || G::READS) {
        s = dot<T, DP>(tile, b, f, l, start);
        s2 = dot<T, DP>(tile2, b2, g, l, start2);
    } else {
        constexpr int N = L::NF <= 4 ? L::NF : L::NF / 2;
        const int at = anew<L::ROWB>(l.row);
        s = start;
        s2 = start2;
#pragma unroll
        for (int n = 0; n < L::NF; n += N) {
            uint4 x[N], y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = *(const uint4*)(tile + b * 32 * L::ROWB + L::further(at, 2 * (n + i)));
                y[i] = *(const uint4*)(tile2 + b2 * 32 * L::ROWB + L::further(at, 2 * (n + i)));
            }
            reads_first();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x[i]), as_bf16x8(f.chunk(n + i, at)), s, 0, 0, 0);
                s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(y[i]), as_bf16x8(g.chunk(n + i, at)), s2, 0, 0, 0);
            }
        }
    }
}

// The weights of a block's 32 passing rows for a lane's fixed row, as the second product takes them: floats, or bf16 in the order of
// the accumulator's elements.  (bf16 because the matrix units take both operands alike, and a second product for what rounding leaves takes as long as the first: `out` is 2.1e-3 to
// 2.3e-3 of its norm from 64 bits, 1.65e-3 of which are its own rounding.  Where the rest does matter, a second product is made: see Row::step() and gradients().)
template <typename T>
struct Weights {
    float w[16];
    __device__ __forceinline__ void set(int j, float4 v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * j + i] = (&v.x)[i];
    }
};
template <>
struct Weights<__bf16> {
    uint32_t w[8];
    __device__ __forceinline__ void set(int j, float4 v) {
        w[2 * j] = cvt_pk_bf16(v.x, v.y);
        w[2 * j + 1] = cvt_pk_bf16(v.z, v.w);
    }
    __device__ __forceinline__ float4 get(int j) const {
        return make_float4(__uint_as_float(w[2 * j] << 16), __uint_as_float(w[2 * j] & 0xffff0000u), __uint_as_float(w[2 * j + 1] << 16),
                           __uint_as_float(w[2 * j + 1] & 0xffff0000u));
    }
};

// acc[feature][fixed row] += sum over the block's 32 passing rows of tile[row][feature] w[row].
template <typename T, int DP>
__device__ __forceinline__ void weigh(const unsigned char* tile, int b, const Weights<T>& w, f32x16 (&acc)[Tile<T, DP>::NA],
                                      const Lanes<T, DP>& l) {
    using L = Tile<T, DP>;
    const unsigned char* base = tile + b * 32 * L::ROWB;
    const int at = anew<L::ROWB>(l.turned);
    if constexpr (L::EB == 2) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            union { s16x4 h[2]; bf16x8 v; } a[L::NA];
#pragma unroll
            for (int i = 0; i < L::NA; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    a[i].h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (SEQATT_LDS s16x4*)(base + (16 * j + 8 * x) * L::ROWB + (L::further(at, 4 * i) ^ (L::swz(8 * x) << 4))));
            reads_first();
            const bf16x8 p = as_bf16x8(make_uint4(w.w[4 * j], w.w[4 * j + 1], w.w[4 * j + 2], w.w[4 * j + 3]));
#pragma unroll
            for (int i = 0; i < L::NA; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i].v, p, acc[i], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float v[4][L::NA];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < L::NA; ++i)
                    v[e][i] = *(const float*)(base + (8 * g + e) * L::ROWB + L::further(at ^ (L::swz(8 * g + e) << 4), 8 * i));
            reads_first();
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < L::NA; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e][i], w.w[4 * g + e], acc[i], 0, 0, 0);
        }
    }
}

// Keys that some of a workgroup's rows see in their windows or among the first ones.  A key outside of all windows may be anything (a cache's row that is somebody else's by
// now), and its weight of 0 is to make zeros of its values: so they are zeros in a tile.  (One token over each of 8 short caches 7.4 -> 7.7 us, two rows of 8192 in a window of 128 288 -> 289;
// with zeros in place of the keys too, and in the queries' gradients, 8.0 and 290.)
struct SeenKeys {
    int begin, end, sinks;
    __device__ __forceinline__ SeenKeys(const Args& a, const Seq& q, int near, int far)
        : begin(scalar(window_begin(a, near))), end(scalar(seen_to<true>(a, q, far))), sinks(a.sinks) {}
    __device__ __forceinline__ bool all(int k0, int n) const { return (k0 + n <= end) & ((k0 >= begin) | (k0 + n <= sinks)); }
    __device__ __forceinline__ bool has(int k) const { return (k < end) & ((k >= begin) | (k < sinks)); }
    // of a tile from k0 on, a bit each
    __device__ __forceinline__ uint64_t those(int k0) const { return __ballot(has(k0 + (int)(threadIdx.x & 63))); }
};

static __device__ const uint4 zeros = {0, 0, 0, 0};
static __device__ const uint32_t infinity_word = 0x7f800000u, minus_one = 0xffffffffu;

// Sends for tiles: 16 bytes a lane go from memory into LDS without a register (a lane picks the chunk whose swizzled place it
// fills).  Landed after vm_wait() and a barrier.  Chunks behind a head's elements repeat its last one: they meet zeros in the fixed
// rows, or make features that nobody stores.
// ROWS_ARE_TOKENS: group is 1.  A thread's chunks are then, for most lengths of a row, the same one so many rows apart.
template <typename T, int DP, int R = tile_rows(sizeof(T)), bool ROWS_ARE_TOKENS = false>
struct Sender {
    using L = Tile<T, DP, R>;
    static constexpr bool SAME = ROWS_ARE_TOKENS && 256 % L::CPR == 0 && 256 / L::CPR % 16 == 0;
    static constexpr int N = SAME ? 1 : L::PER_THREAD, ROWS_APART = 256 / L::CPR;
    unsigned off[N];                   // where a lane's chunks lie from the tile's first element on, in bytes
    int64_t apart;
    bool regular;                      // the same in every tile
    static __device__ __forceinline__ int row_of(int j, int thread) { return (j * 256 + thread) / L::CPR; }
    static __device__ __forceinline__ int element(int j, int thread, int head_dim) {
        return min((((j * 256 + thread) % L::CPR) ^ L::swz(row_of(j, thread))) * L::EPC, head_dim - L::EPC);
    }
    static __device__ __forceinline__ void send(unsigned char* tile, int j, const void* from) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                         (SEQATT_LDS void*)(tile + (j * 4 + wave) * 1024), 16, 0, 0);
    }
    // rows of `group` heads to a token
    __device__ __forceinline__ Sender(const ps_strides& s, int group, int head_dim) {
        regular = R % group == 0 && s.row < 1 << 20 && s.head < 1 << 20;
        apart = SAME ? ROWS_APART * s.row * L::EB : 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int r = row_of(j, threadIdx.x), token = r / group;
            off[j] = regular ? (unsigned)(token * (int)s.row + (r - token * group) * (int)s.head + element(j, threadIdx.x, head_dim)) * L::EB : 0u;
        }
    }
    static __device__ __forceinline__ void whole(unsigned char* tile, const T* first, const unsigned (&off)[N], int64_t apart = 0) {
#pragma unroll
        for (int j = 0; j < L::PER_THREAD; ++j) send(tile, j, (const char*)first + (SAME ? j * apart : 0) + off[SAME ? 0 : j]);
    }
    __device__ __forceinline__ void whole(unsigned char* tile, const T* first) const { whole(tile, first, off, apart); }
    // row(i): address of passing row i's element 0; there: bit i tells whether it is one, and not a row of zeros.  (Worked out anew for the few
    // tiles that need it.)
    template <typename Row>
    static __device__ __forceinline__ void rows(unsigned char* tile, int head_dim, uint64_t there, Row row) {
        const int thread = anew<256>((int)threadIdx.x);
#pragma unroll
        for (int j = 0; j < L::PER_THREAD; ++j) {
            const int i = row_of(j, thread);
            send(tile, j, there >> i & 1 ? (const void*)(row(i) + element(j, thread, head_dim)) : (const void*)&zeros);
        }
    }
    // zeros for the rows that are not among the seen keys
    __device__ __forceinline__ void whole(unsigned char* tile, const T* first, int k0, const SeenKeys& seen) const {
        const int thread = anew<256>((int)threadIdx.x);
#pragma unroll
        for (int j = 0; j < L::PER_THREAD; ++j)
            send(tile, j, seen.has(k0 + row_of(j, thread)) ? (const char*)first + (SAME ? j * apart : 0) + off[SAME ? 0 : j] : (const char*)&zeros);
    }
};
// Which rows of a tile from k0 on are keys and no padding (asked only of tiles that have some), a bit each.
__device__ __forceinline__ uint64_t keys_there(const Args& a, const Seq& q, int k0, bool padded) {
    const int k = k0 + (int)(threadIdx.x & 63), doc = padded ? a.k_docs[q.k0 + min(k, q.kn - 1)] : 0;
    return __ballot(k < q.kn && doc >= 0);
}
// A word a lane of this wavefront, sent like a tile.
__device__ __forceinline__ void send_words(void* to, const void* from) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (SEQATT_LDS void*)to, 4, 0, 0);
}
__device__ __forceinline__ void vm_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Tiles of 32 rows that a wavefront has to itself, by sends of its own.
template <typename T, int DP>
struct Few {
    using L = Tile<T, DP, 32>;
    static constexpr int SENDS = L::BYTES / 1024;                         // of 64 lanes, for a tile
    // Tiles of a wavefront in LDS: two, or one of the largest; up to 128 KB of a unit's 160, in bf16 with heads of 64 by two workgroups.
    static constexpr int STAGES = L::BYTES > 8192 ? 1 : 2, WORKGROUPS = L::BYTES > 4096 ? 1 : 2;
    // Sends whose lanes' chunks differ; the others repeat them so many rows on (sends of no whole number of rows: none does).
    static constexpr int PERIOD = 64 % L::CPR == 0 ? L::CPR / 4 : SENDS, ROWS_A_PERIOD = 64 * PERIOD / L::CPR;
    static constexpr int WAIT = (STAGES - 1) * (2 * SENDS + 1);           // sends behind the oldest tile's, and a word for documents
    unsigned off[2][PERIOD];
    int64_t step[2];                                                      // bytes from row to row
    __device__ __forceinline__ Few(const Args& a) : step{a.ks.row * L::EB, a.vs.row * L::EB} {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < PERIOD; ++j) {
#pragma unroll
            for (int x = 0; x < 2; ++x) off[x][j] = (unsigned)row_of(j, lane) * (unsigned)step[x] + element(j, lane, a.head_dim) * L::EB;
        }
    }
    static __device__ __forceinline__ int row_of(int j, int lane) { return (j * 64 + lane) / L::CPR; }
    static __device__ __forceinline__ int element(int j, int lane, int head_dim) {
        return min((((j * 64 + lane) % L::CPR) ^ L::swz(row_of(j, lane))) * L::EPC, head_dim - L::EPC);
    }
    static __device__ __forceinline__ void send(unsigned char* tile, int j, const void* from) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (SEQATT_LDS void*)(tile + j * 1024), 16, 0, 0);
    }
    __device__ __forceinline__ void whole(unsigned char* tile, int x, const void* first) const {
#pragma unroll
        for (int j = 0; j < SENDS; ++j) send(tile, j, (const char*)first + j / PERIOD * ROWS_A_PERIOD * step[x] + off[x][j % PERIOD]);
    }
    // row(i): address of row i; there: bit i tells whether it is one, and not zeros
    template <typename Address>
    static __device__ __forceinline__ void rows(unsigned char* tile, int head_dim, uint64_t there, Address row) {
        const int lane = anew<256>((int)(threadIdx.x & 63));
#pragma unroll
        for (int j = 0; j < SENDS; ++j) {
            const int i = row_of(j, lane);
            send(tile, j, there >> i & 1 ? (const void*)(row(i) + element(j, lane, head_dim)) : (const void*)&zeros);
        }
    }
    __device__ __forceinline__ void whole(unsigned char* tile, int x, const void* first, int k0, const SeenKeys& seen) const {
        const int lane = anew<256>((int)(threadIdx.x & 63));
#pragma unroll
        for (int j = 0; j < SENDS; ++j)
            send(tile, j, seen.has(k0 + row_of(j, lane)) ? (const char*)first + j / PERIOD * ROWS_A_PERIOD * step[x] + off[x][j % PERIOD] : (const char*)&zeros);
    }
};

// ---- which tiles are seen: 64 of them at a time, a lane each, as masks ----------------------------------------------------
__device__ __forceinline__ uint64_t scalars(uint64_t x) { return (uint64_t)(uint32_t)scalar((int)(x >> 32)) << 32 | (uint32_t)scalar((int)x); }
struct Walk {
    int group = -1;
    uint64_t seen = 0, one = 0, padded = 0;
    // The first tile from t on that is seen, `end` if none is.  classify(tile, one, padded): whether some of the tile is seen; whether its
    // and the fixed rows are all of one document; whether some of it is padding.
    template <typename Classify>
    __device__ __forceinline__ int next(int from, int end, Classify classify) {
        int t = scalar(from);
        while (t < scalar(end)) {
            if ((t >> 6) != group) {
                group = t >> 6;
                const int mine = group * 64 + (int)(threadIdx.x & 63);
                bool all = false, pad = false;
                const bool some = mine < end && classify(mine, all, pad);
                seen = scalars(__ballot(some));
                one = scalars(__ballot(some && all));
                padded = scalars(__ballot(some && pad));
            }
            const uint64_t m = seen >> (t & 63);
            if (m) return scalar(t + __builtin_ctzll(m));
            t = (group + 1) << 6;
        }
        return scalar(end);
    }
    __device__ __forceinline__ bool is_one(int t) const { return one >> (t & 63) & 1; }
    __device__ __forceinline__ bool is_padded(int t) const { return padded >> (t & 63) & 1; }
};

// ---- scores ------------------------------------------------------------------------------------------------------------------
// The cap.  bf16 calls take tanh u = 1 - 2 r, r = 1 / (1 + e^2u), whose absolute error of 1.4e-7 is that of a score near the cap; r is
// what they go on with.  Times a cap of up to NEAR that is 4e-5 of a score and less, a fiftieth of the rounding of its weight; above (FAR) it would
// be more, and 0.14 at 1e6.  There it is tanh itself, with its error relative: the series in front of a quarter, up to u^9 (1e-8 there), 1 - 2 r
// behind (6e-7).  (16 x 2048 with prefix, forwards / gradients 431 / 2000 us with 1 - 2 r, 546 / 2262 with the series; 8 x 2048 with heads of 64
// 128 / 459, 191 / 569.)  fp32 calls take the library's, good to the last places everywhere.
struct Cap {
    static constexpr float NEAR = 256.f;
    float inner, outer;                // what the product is multiplied by on the way in, and tanh on the way out (powers of two)
    template <typename T>
    static __device__ __forceinline__ Cap of(const Args& a) {
        return {a.cap_in * (sizeof(T) == 4 ? 1.f : 2.f * LOG2E), a.cap * LOG2E};
    }
    template <typename T>
    static __device__ __forceinline__ bool far(const Args& a) { return sizeof(T) == 2 && a.cap > NEAR; }
    template <typename T, bool FAR>
    __device__ __forceinline__ float bent(float s) const {                // r, or tanh
        if constexpr (sizeof(T) == 4) return tanhf(s * inner);
        const float r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * inner));
        if (!FAR) return r;
        const float u = s * inner * (0.5f * LN2), x = u * u;
        const float series = fmaf(u * x, fmaf(x, fmaf(x, fmaf(x, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), u);
        return fabsf(u) < 0.25f ? series : fmaf(-2.f, r, 1.f);
    }
    template <typename T, bool FAR>
    __device__ __forceinline__ float score(float b, float less) const {   // in powers of two, less something
        return sizeof(T) == 4 || FAR ? fmaf(b, outer, -less) : fmaf(b, -2.f * outer, outer - less);
    }
    template <typename T, bool FAR>
    static __device__ __forceinline__ float slope(float b) {              // 1 - tanh^2, in bf16 a quarter of it
        return sizeof(T) == 4 ? fmaf(-b, b, 1.f) : FAR ? fmaf(-0.25f * b, b, 0.25f) : fmaf(-b, b, b);
    }
};

// ---- a learned bias -----------------------------------------------------------------------------------------------------------
// The bias of a distance d = key - place, clamped to -reach .. reach, is table[head][reach + d], made from buckets and values by a launch in
// front.  A tile meets few of them, and as they are the same along its diagonals a stretch of bias_width for each head will do: it comes by DMA with the tile,
// head g's words at g bias_width, of distances from `lowest` on.
struct Learned {
    static __device__ __forceinline__ void send(int hk, int lowest, float* to) {
        const ArgsAgain a = again();
        const int lane = anew<256>((int)threadIdx.x) & 63, words = a->bias_words, width = a->bias_width, group = a->group, reach = a->reach;
        for (int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64; w < words; w += 256) {
            const int g = min((int)__umulhi((unsigned)(w + lane), a->by_width), group - 1), d = lowest + min(w + lane - g * width, width - 1);
            const float* from = a->table + (int64_t)(hk * group + g) * (2 * reach + 1) + reach + max(-reach, min(d, reach));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (SEQATT_LDS void*)(to + w), 4, 0, 0);
        }
    }
    // the same distances' places in a lane's sums of buckets
    static __device__ __forceinline__ void send_buckets(int lowest, int* to) {
        const ArgsAgain a = again();
        const int lane = anew<256>((int)threadIdx.x) & 63, width = a->bias_width, reach = a->reach;
        for (int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64; w < width; w += 256) {
            const int d = lowest + min(w + lane, width - 1);
            const int32_t* from = a->bucket_words + reach + max(-reach, min(d, reach));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (SEQATT_LDS void*)(to + w), 4, 0, 0);
        }
    }
    // The bias is what the product starts from (b(i), of passing row i of 32), if it bends no score: nothing is left to add then.  Every step of the accumulation rounds
    // at the size of bias / scale for that, where a bias added at the end would round once: with biases of a few units fp32 results are off by 6e-7 of their norm (4e-7
    // without a bias), with 20 added to all of them 3.8e-6, with 1e4 2e-3 (elementary operations in 32 bits 3.5e-7, 6e-7, 2.5e-4).
    template <typename Of>
    static __device__ __forceinline__ f32x16 start(bool is, int half, Of of) {
        f32x16 s = no_start();
        if (is) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = of(8 * (e >> 2) + (e & 3) + 4 * half);
        }
        return s;
    }
    // (places as far from all keys as any: distances stay in 32 bits)
    static __device__ __forceinline__ int place(int place) { return max(place, -(1 << 29)); }
};

// Row of accumulator element e.
__device__ __forceinline__ constexpr int row_of(int e) { return 8 * (e >> 2) + (e & 3); }   // + 4 half

// The accumulators of a wavefront, [feature][a lane's row] times the lane's `by`, to its 32 rows in memory: by way of LDS, 64 features at a
// time, so that 8 or 16 lanes write a row's lines whole (64 sequences of 512 tokens, 12 heads of 64, forwards 125 -> 107 us: from the registers
// a store has 32 pieces of 16 bytes, of 32 lines, and there are 16 of them).  own: the lane's row in memory, null if there is none.  mine: PUT_BYTES
// of LDS that no other wavefront uses.  LEFT: not the values, but what their rounding to bf16 leaves.
constexpr int PUT_BYTES = 32 * 64 * 4;
template <typename T, int DP, bool LEFT = false>
__device__ __forceinline__ void put_rows(unsigned char* mine, const f32x16 (&acc)[DP / 32], float by, int head_dim, T* own) {
    using P = Tile<T, 64, 32>;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
#pragma unroll
    for (int p = 0; p < DP / 32; p += 2) {
        const int here = DP / 32 - p < 2 ? 1 : 2, chunks = here * 32 / P::EPC;
#pragma unroll
        for (int i = 0; i < here; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[p + i][4 * g + e] * by;
                if constexpr (P::EB == 2) {
                    uint2 x;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t pair = cvt_pk_bf16(v[2 * e], v[2 * e + 1]);
                        if (LEFT) pair = cvt_pk_bf16(v[2 * e] - __uint_as_float(pair << 16), v[2 * e + 1] - __uint_as_float(pair & 0xffff0000u));
                        (&x.x)[e] = pair;
                    }
                    *(uint2*)(mine + P::at(col, 4 * i + g) + 8 * half) = x;
                } else {
                    *(float4*)(mine + P::at(col, 8 * i + 2 * g + half)) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
        __builtin_amdgcn_wave_barrier();                                  // (a wavefront's accesses to LDS keep their order)
#pragma unroll
        for (int j = 0; j < chunks / 2; ++j) {
            const int r = (j * 64 + lane) / chunks, chunk = (j * 64 + lane) % chunks, e = 32 * p + chunk * P::EPC;
            const uint4 x = *(const uint4*)(mine + P::at(r, chunk));
            T* const to = (T*)((uint64_t)(uint32_t)__shfl((int)((uint64_t)own >> 32), r, 64) << 32 | (uint32_t)__shfl((int)(uint64_t)own, r, 64));
            if (to && e < head_dim) *(uint4*)(to + e) = x;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Checked arguments as the kernels take them, and the plan of a call; PS_OK or an error.  ahead: rows may see keys behind their place.
struct Plan {
    Args a;
    size_t bytes;                      // of workspace
};
int plan(const ps_attention_desc* d, const ps_attention_seqs* s, const ps_attention_local* local, bool backward, void* workspace, Plan& p, bool ahead);
inline bool sees_ahead(const ps_attention_desc* d, const ps_attention_seqs* s) { return d && (!d->causal || s->prefix); }
void set_width(Args& a, int width);
void make_table(const Args& a, const ps_attention_local* local, float by, hipStream_t st);
int check_strides(const ps_attention_desc* d, const ps_strides& s, const void* base, int64_t rows, int64_t heads, bool written);
int check_sequences(const Args& a, hipStream_t st);
void summarise_documents(const Args& a, hipStream_t st);
bool add_up(const Args& a, int32_t seqs, int64_t blocks, int32_t parts);

}  // namespace seqatt
