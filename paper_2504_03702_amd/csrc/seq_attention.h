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
};

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

// Tiles of keys, from the first on, that some of the FIXED rows from r0 on may see; tiles of rows, from `first` on, that may see some of
// the FIXED keys from k0 on.  Shares are of these.
__device__ __forceinline__ int key_tiles(const Args& a, const Seq& q, int r0) {
    const int far = q.start + (int)over_group(a, min(r0 + FIXED, q.qn * a.group) - 1);
    return (max(0, seen_end(a, q, far)) + a.tile - 1) / a.tile;
}
__device__ __forceinline__ int row_tiles(const Args& a, const Seq& q, int k0, int& first) {
    const int rows = q.qn * a.group, n = (rows + a.key_tile - 1) / a.key_tile;
    first = a.causal && k0 >= q.prefix ? (int)min((int64_t)n, max((int64_t)0, (int64_t)(k0 - q.start) * a.group / a.key_tile)) : 0;
    return n;
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
template <bool KEYS>
__device__ __forceinline__ int shares_of(const Args& a, const Seq& q, int block) {
    const int n = KEYS ? q.kn : q.qn * a.group;
    if (block * FIXED >= n) return 0;
    if ((KEYS ? a.key_parts : a.parts) == 1) return 1;
    int first = 0;
    const int tiles = KEYS ? row_tiles(a, q, block * FIXED, first) : key_tiles(a, q, block * FIXED);
    return shares(tiles - first, KEYS ? a.key_parts : a.parts, KEYS ? a.key_part_tiles : a.part_tiles);
}
// a.listed (at most 64 sequences of at most 64 blocks): the grid has a workgroup for what there could be, and the first so many take
// what there is, found by adding it up a sequence to a lane.  Counted as the grid counts, what there is lay anywhere among it, and
// three or more long workgroups on one unit beside empty ones (8 sequences of 100 to 1023 tokens, 408 workgroups of 2048 with work to do: 26 to
// 40 tiles on the fullest units, 10 on average; forwards / queries' / keys' gradients in fp32 with heads of 80 128 / 173 / 293 us, 77 / 104 / 157
// added up).
template <bool KEYS>
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
    if (good)
        for (int b = 0; b < blocks; ++b) {
            const int c = shares_of<KEYS>(a, mine, b);
            if (c == 0) break;
            n += c;
        }
    const int front = sum_in_front(n, upto), s = __popcll(__ballot(upto <= (int)id));
    if (s >= a.seqs) return false;
    id -= __builtin_amdgcn_readlane(front, s);
    w.s = a.seq0 + s;
    sequence(a, w.s, q);
    const int own = ((KEYS ? q.kn : q.qn * a.group) + FIXED - 1) / FIXED, b = KEYS ? lane : own - 1 - lane;   // (most work first)
    const int in_front = sum_in_front(b >= 0 ? shares_of<KEYS>(a, q, b) : 0, upto), at = __popcll(__ballot(upto <= (int)id));
    w.block = KEYS ? at : own - 1 - at;
    w.part = (int)id - __builtin_amdgcn_readlane(in_front, at);
    return true;
}

// The same, as scalars: the compiler does not see that all lanes have found the same.
template <bool KEYS>
__device__ __forceinline__ bool find_work(const Args& a, Seq& q, Work& w) {
    if (!look_for_work<KEYS>(a, q, w)) return false;
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

// 32 passing rows (block b of the tile) times the fixed rows.
template <typename T, int DP, typename F>
__device__ __forceinline__ f32x16 dot(const unsigned char* tile, int b, const F& f, const Lanes<T, DP>& l) {
    using L = Tile<T, DP>;
    constexpr int N = F::READS ? 2 : L::NF <= 8 ? L::NF : L::NF / 2;
    const int at = anew<L::ROWB>(l.row);
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
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
                                     const Lanes<T, DP>& l) {
    using L = Tile<T, DP>;
    if constexpr (L::EB == 4 || F::READS || G::READS) {
        s = dot<T, DP>(tile, b, f, l);
        s2 = dot<T, DP>(tile2, b2, g, l);
    } else {
        constexpr int N = L::NF <= 4 ? L::NF : L::NF / 2;
        const int at = anew<L::ROWB>(l.row);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = s2[e] = 0.f;
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
// the accumulator's elements.
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

// ---- which tiles are seen: 64 of them at a time, a lane each, as masks ----------------------------------------------------
// (scalars: the compiler does not see that all lanes have the same, and would count and address tiles in vector registers)
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
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

// Checked arguments as the kernels take them, and the plan of a call; PS_OK or an error.
struct Plan {
    Args a;
    size_t bytes;                      // of workspace
};
int plan(const ps_attention_desc* d, const ps_attention_seqs* s, bool backward, void* workspace, Plan& p);
int check_strides(const ps_attention_desc* d, const ps_strides& s, const void* base, int64_t rows, int64_t heads, bool written);
int check_sequences(const Args& a, hipStream_t st);
void summarise_documents(const Args& a, hipStream_t st);
bool add_up(int32_t seqs, int64_t blocks, int32_t parts);

}  // namespace seqatt
