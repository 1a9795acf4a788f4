// Attention with capped scores, distance bias, document and prefix masks: the host's side of both directions, and forwards.
#include <math.h>
#include <string.h>

#include "seq_attention.h"

using namespace seqatt;
typedef __bf16 bf16;

namespace {

constexpr float SLACK = 8.f;           // powers of two that a score may exceed the exponent's reference by

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * LN2; }

// A lane's row: what it sees, and its running maximum, sum and weighted values.
template <typename T, int DP, int R>
struct Row {
    using L = Tile<T, DP, R>;
    int head, place, doc, end;         // keys in front of `end` are seen, if their documents are
    int64_t token;
    float slope, m = -INFINITY, l = 0.f;   // what goes with step()'s scores; the exponent's reference, in powers of two; this lane's share of the sum
    Fixed<T, DP> qf;
    f32x16 o[L::NA];
    const Lanes<T, DP> lanes;
    const int half;

    // row r of key head hk's queries; live: whether there is one
    __device__ __forceinline__ Row(const Args& a, const Seq& q, int hk, int r, bool live) : lanes(threadIdx.x & 63), half((threadIdx.x & 63) >> 5) {
        const int qi = (int)over_group(a, r);
        head = hk * a.group + r - qi * a.group;
        token = q.q0 + qi;
        place = q.start + qi;
        slope = a.slopes ? a.slopes[head] * a.slope_by : 0.f;
        doc = a.q_docs ? a.q_docs[token] : 0;
        end = seen_end(a, q, place);
        qf.load((const T*)a.q + token * a.qs.row + head * a.qs.head, live && doc >= 0, a.head_dim, half);
#pragma unroll
        for (int i = 0; i < L::NA; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    }

    // A tile of keys from k0 on and its values.  cut: some of the wavefront's rows see only the keys in front of their `end`; docs: documents
    // of its keys, null if the tile's and all rows' are one.
    __device__ __forceinline__ void step(const Args& a, const unsigned char* keys, const unsigned char* values, const int* docs, int k0, bool cut) {
        f32x16 sc[L::BLOCKS];
#pragma unroll
        for (int b = 0; b < L::BLOCKS; b += 2) {
            if constexpr (L::BLOCKS % 2 == 0)
                dots<T, DP>(keys, b, qf, sc[b], keys, b + 1, qf, sc[b + 1], lanes);
            else
                sc[b] = dot<T, DP>(keys, b, qf, lanes);
        }
        float c = a.scale * LOG2E;
        if (a.cap > 0.f) {
            const Cap cap = Cap::of<T>(a);
            auto bend = [&](auto far) {
#pragma unroll
                for (int b = 0; b < L::BLOCKS; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[b][e] = cap.score<T, far>(cap.bent<T, far>(sc[b][e]), 0.f);
            };
            if (Cap::far<T>(a))
                bend(std::true_type());
            else
                bend(std::false_type());
            c = 1.f;
        }
        if (a.slopes) {
            const float from = (float)(place - k0 - 4 * half);
#pragma unroll
            for (int b = 0; b < L::BLOCKS; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[b][e] = fmaf(-slope, fabsf(from - (float)(32 * b + row_of(e))), sc[b][e]);
        }
        if (cut) {
            const int left = end - k0 - 4 * half;
#pragma unroll
            for (int b = 0; b < L::BLOCKS; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[b][e] = left > 32 * b + row_of(e) ? sc[b][e] : -INFINITY;
        }
        if (docs) {
#pragma unroll
            for (int b = 0; b < L::BLOCKS; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int4 of = *(const int4*)&docs[32 * b + 8 * j + 4 * half];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[b][4 * j + i] = (&of.x)[i] == doc ? sc[b][4 * j + i] : -INFINITY;
                }
        }
        float mx = sc[0][0];
#pragma unroll
        for (int b = 0; b < L::BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[b][e]);
        const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1])) * c;
        // the reference follows the maximum lazily: it moves when a tile exceeds it by more than SLACK, so weights reach
        // 2^SLACK and the accumulators are rescaled a few times a row instead of at nearly every tile
        if (__any(mx > m + SLACK)) {
            const float next = mx > m + SLACK ? mx : m;
            const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
            m = next;
#pragma unroll
            for (int i = 0; i < L::NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
            l *= alpha;
        }
        const float ref = m == -INFINITY ? 0.f : m;                   // (a row that has seen nothing yet)
#pragma unroll
        for (int b = 0; b < L::BLOCKS; ++b) {
            Weights<T> w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    (&x.x)[i] = __builtin_amdgcn_exp2f(fmaf(sc[b][4 * j + i], c, -ref));
                    l += (&x.x)[i];
                }
                w.set(j, x);
            }
            weigh<T, DP>(values, b, w, o, lanes);
        }
    }

    // The halves of the wavefront put their sums together.  (Padding has seen the padding of cut tiles, zeros like itself: it sees nothing.)
    __device__ __forceinline__ void add_halves() {
        l += __shfl_xor(l, 32, 64);
        if (doc < 0) {
            l = 0.f;
            m = -INFINITY;
        }
    }
};

// A workgroup: FIXED rows of a key head's queries, against a share of the key tiles that any of them sees (one pass, running
// maximum and sum).  32 rows a wavefront, because a lane then has its row's maximum and sum to itself and its weights where the second product
// takes them; tiles of 64 keys (32 in fp32), two of them in LDS, for two or three workgroups a unit.  Bound by waits with few wavefronts
// there: no unit is full, and each wavefront waits for its own products, reads of LDS and barriers while one or two others have the SIMD.  With
// heads of 128 under a cap (16 prompts of 1500 to 2048 tokens with prefix, 16 heads on 4) 389 us, 0.60 PFLOP/s: vector units issue 46 %
// and matrix units are busy 26 % of the time, 1.7 wavefronts a SIMD wait 25 % of theirs; documents in two rows of 8192, 16 heads of 64: 87 us,
// 0.42 PFLOP/s, 40 %, 19 %, 2.1 wavefronts, 36 %.  A call of short prompts (64 of 4 to 512 tokens, 12 heads of 64: 33 us) waits 42 % of a
// wavefront's time, for its first tiles.  Three tiles in LDS, priorities around the matrix instructions and the sum of a row's weights by dot
// products made no difference (2 %).
template <typename T, int DP, bool PARTS>
__global__ __launch_bounds__(256, DP == 64 ? 3 : 2) void attend_kernel(Args a) {
    using L = Tile<T, DP>;
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][keys, values]
    __shared__ __align__(16) int s_doc[2][64];

    Seq q;
    Work w;
    if (!find_work<false>(a, q, w)) return;
    const int hk = w.hk, s = w.s, part = PARTS ? w.part : 0, rows = q.qn * a.group, r0 = w.block * FIXED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int tiles = key_tiles(a, q, r0);
    const int t0 = PARTS ? part * a.part_tiles : 0, t1 = PARTS ? min(tiles, t0 + a.part_tiles) : tiles;
    if (PARTS && t0 > 0 && t0 >= tiles) return;                           // (part 0 writes, keys or not)

    const int wr0 = r0 + 32 * wave;
    const bool live = wr0 + col < rows;
    Row<T, DP, L::ROWS> row(a, q, hk, min(wr0 + col, rows - 1), live);

    // what the workgroup's and the wavefront's rows see
    const int last = min(r0 + FIXED, rows) - 1;
    const int far = q.start + (int)over_group(a, last);                   // largest place
    const int wfar = q.start + (int)over_group(a, min(wr0 + 31, rows - 1)), wnear = q.start + (int)over_group(a, min(wr0, rows - 1));
    int dmin = 0, dmax = 0;                                               // documents of the workgroup's rows
    if (a.q_docs) {
        const int x = a.q_docs[q.q0 + (int)over_group(a, min(r0 + lane, last))], y = a.q_docs[q.q0 + (int)over_group(a, min(r0 + 64 + lane, last))];
        dmin = min(x, y);
        dmax = max(x, y);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            dmin = min(dmin, __shfl_xor(dmin, o, 64));
            dmax = max(dmax, __shfl_xor(dmax, o, 64));
        }
    }
    const int64_t kblock0 = doc_block0(q.k0, s);
    auto classify = [&](int t, bool& one, bool& pad) {
        const int k0 = t * L::ROWS;
        bool some = !a.causal || k0 <= far || k0 < q.prefix;
        one = !a.k_docs;
        if (a.k_docs && !a.k_blocks) {
            pad = true;
        } else if (a.k_docs && some) {
            const int2 m = a.k_blocks[kblock0 + k0 / DOC_BLOCK];
            some = dmax >= 0 && m.y >= max(dmin, 0) && m.x <= dmax;
            one = m.x == m.y && dmin == dmax && m.x == dmin;
            pad = m.x < 0;
        }
        return some;
    };
    auto is_cut = [&](int k0) { return k0 + L::ROWS > q.kn || (a.causal && k0 + L::ROWS - 1 > wnear && k0 + L::ROWS > q.prefix); };

    const T* kbase = (const T*)a.k + q.k0 * a.ks.row + hk * a.ks.head;
    const T* vbase = (const T*)a.v + q.k0 * a.vs.row + hk * a.vs.head;
    const Sender<T, DP, L::ROWS, true> keys(a.ks, 1, a.head_dim), values(a.vs, 1, a.head_dim);
    const bool regular = keys.regular && values.regular;
    auto request = [&](int t, bool padded, int buf) {
        const int k0 = t * L::ROWS;
        // (rows past the keys, and padding, are zeros: their weights are, and nothing is to come of them)
        if (k0 + L::ROWS <= q.kn && !padded && regular) {
            keys.whole(smem[buf][0], kbase + k0 * a.ks.row);
            values.whole(smem[buf][1], vbase + k0 * a.vs.row);
        } else {
            const uint64_t there = keys_there(a, q, k0, padded);
            keys.rows(smem[buf][0], a.head_dim, there, [&](int i) { return kbase + (k0 + i) * a.ks.row; });
            values.rows(smem[buf][1], a.head_dim, there, [&](int i) { return vbase + (k0 + i) * a.vs.row; });
        }
        if (a.k_docs && wave == 0) send_words(s_doc[buf], a.k_docs + q.k0 + min(k0 + lane, q.kn - 1));
    };

    Walk walk;
    int t = walk.next(t0, t1, classify), buf = 0;
    if (t < t1) request(t, walk.is_padded(t), 0);
    while (t < t1) {
        const bool one = walk.is_one(t);
        const int k0 = t * L::ROWS;
        t = walk.next(t + 1, t1, classify);
        vm_wait();
        __syncthreads();                                                  // the tile has landed, the one before it is no longer read
        if (t < t1) request(t, walk.is_padded(t), buf ^ 1);
        // (a wavefront whose rows all stand before the tile has nothing in it)
        if (wr0 < rows && !(a.causal && k0 > wfar && k0 >= q.prefix)) {
            row.step(a, smem[buf][0], smem[buf][1], one ? nullptr : s_doc[buf], k0, is_cut(k0));
        }
        buf ^= 1;
    }
    row.add_halves();
    __syncthreads();                                                      // (tiles are no longer read)
    if (wr0 >= rows) return;
    unsigned char* const mine = smem[0][0] + wave * PUT_BYTES;
    static_assert(sizeof(smem) >= 4 * PUT_BYTES, "rows on their way out");
    if (PARTS) {
        const int64_t at = ((int64_t)part * a.n_q + row.token) * a.heads + row.head;
        put_rows<float, DP>(mine, row.o, 1.f, a.head_dim, live ? a.part_o + at * a.head_dim : nullptr);
        if (live && half == 0) a.part_ml[at] = make_float2(row.m, row.l);
        return;
    }
    const float inv = row.l == 0.f ? 0.f : 1.f / row.l;
    put_rows<T, DP>(mine, row.o, inv, a.head_dim, live ? (T*)a.out_w + row.token * a.os.row + row.head * a.os.head : nullptr);
    if (sizeof(T) == 2 && a.rest_w)
        put_rows<T, DP, true>(mine, row.o, inv, a.head_dim, live ? (T*)a.rest_w + (row.token * a.heads + row.head) * a.head_dim : nullptr);
    if (a.lse_w && live && half == 0) a.lse_w[(int64_t)row.head * a.n_q + row.token] = lse_of(row.m, row.l);
}

// Few rows, at most 32 of a key head's queries: single tokens over their keys, where the time goes into reading keys and values.  The
// workgroup's wavefronts have the same rows and take tiles of 32 keys in turn, each with tiles of its own on their way through LDS, so
// none waits for another until their rows are put together at the end.  Bound by memory: 32 caches of 500 to 32768 keys, 8 heads of 128, 1.05 GB
// in 203 us, 5.2 TB/s (a copy reaches 5.1); one cache of 65521 keys, 4 heads, 134 MB in 27 us, 4.9 TB/s; 8 first rows over up to 512 keys
// 8.5 us, most of it the way to the first tile and out.  In fp32 a tile of 128 features leaves room for one a wavefront: the caches, 2.1 GB,
// 525 us, 4.0 TB/s; with heads of 64, two tiles a wavefront in one workgroup a unit, 1.05 GB at 4.1; 8 first rows 16 us.
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
};

template <typename T, int DP>
__global__ __launch_bounds__(256, (Few<T, DP>::WORKGROUPS)) void attend_few_kernel(Args a) {
    using F = Few<T, DP>;
    using L = typename F::L;
    constexpr int STAGES = F::STAGES;
    __shared__ __align__(1024) unsigned char smem[4][STAGES][2][L::BYTES];   // [wavefront][stage][keys, values]; at the end the rows' sums
    __shared__ __align__(16) int s_doc[4][STAGES][64];
    __shared__ float2 s_ml[4][32];
    static_assert(sizeof(smem) >= 4 * 32 * DP * sizeof(float), "the wavefronts' sums");

    unsigned id = blockIdx.x;
    const int hk = id % a.kv_heads;
    id /= a.kv_heads;
    const int part = id % a.parts, s = a.seq0 + (int)(id / a.parts);
    Seq q;
    if (!sequence(a, s, q)) {
        if (threadIdx.x == 0 && hk == 0 && part == 0) report_fault(a.status, PS_ST_BAD_LENGTH, s);
        return;
    }
    const int rows = q.qn * a.group;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    if (rows == 0) return;
    const int tiles = key_tiles(a, q, 0), t0 = part * a.part_tiles, t1 = min(tiles, t0 + a.part_tiles);
    if (t0 > 0 && t0 >= tiles) return;                                    // (part 0 writes, keys or not)

    const T* kbase = (const T*)a.k + q.k0 * a.ks.row + hk * a.ks.head;
    const T* vbase = (const T*)a.v + q.k0 * a.vs.row + hk * a.vs.head;
    const F few(a);
    const bool regular = a.ks.row < 1 << 20 && a.vs.row < 1 << 20;
    auto request = [&](int t, int stage) {
        const int k0 = t * 32;
        unsigned char *keys = smem[wave][stage][0], *values = smem[wave][stage][1];
        if (regular && k0 + 32 <= q.kn && !a.k_docs) {
            few.whole(keys, 0, kbase + k0 * a.ks.row);
            few.whole(values, 1, vbase + k0 * a.vs.row);
        } else {
            const uint64_t there = keys_there(a, q, k0, a.k_docs != nullptr);
            F::rows(keys, a.head_dim, there, [&](int i) { return kbase + (k0 + i) * a.ks.row; });
            F::rows(values, a.head_dim, there, [&](int i) { return vbase + (k0 + i) * a.vs.row; });
        }
        send_words(s_doc[wave][stage], a.k_docs ? (const void*)(a.k_docs + q.k0 + min(k0 + lane, q.kn - 1)) : (const void*)&zeros);
    };
    const int near = q.start, far = q.start + q.qn - 1;                   // places of the rows
    auto classify = [&](int t, bool&, bool&) {
        const int k0 = t * 32;
        return (t & 3) == wave && (!a.causal || k0 <= far || k0 < q.prefix);
    };

    Walk walk, ahead;                                                     // the tile to work on, the last one sent for
    int t = walk.next(t0, t1, classify), sent = ahead.next(t0, t1, classify), stage = 0, next_stage = 0;
    auto send_next = [&] {
        request(sent, next_stage);
        next_stage = next_stage + 1 < STAGES ? next_stage + 1 : 0;
        sent = ahead.next(sent + 1, t1, classify);
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i)
        if (sent < t1) send_next();
    Row<T, DP, 32> row(a, q, hk, min(col, rows - 1), col < rows);
    while (t < t1) {
        // (with a tile behind it every send of this one is WAIT sends old; the last ones wait for all)
        if (STAGES > 1 && sent < t1)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(F::WAIT) : "memory");
        else
            vm_wait();
        row.step(a, smem[wave][stage][0], smem[wave][stage][1], a.k_docs ? s_doc[wave][stage] : nullptr, t * 32,
                 t * 32 + 32 > q.kn || (a.causal && t * 32 + 31 > near && t * 32 + 32 > q.prefix));
        asm volatile("" ::: "memory");                                    // (its reads are over: their products are on their way)
        stage = stage + 1 < STAGES ? stage + 1 : 0;
        t = walk.next(t + 1, t1, classify);
        if (sent < t1) send_next();
    }
    row.add_halves();

    // the wavefronts' rows put together
    __syncthreads();
    float* sums = (float*)smem;                                           // [wavefront][row][DP]
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4*)(sums + (wave * 32 + col) * DP + 32 * i + 8 * g + 4 * half) =
                make_float4(row.o[i][4 * g], row.o[i][4 * g + 1], row.o[i][4 * g + 2], row.o[i][4 * g + 3]);
    if (half == 0) s_ml[wave][col] = make_float2(row.m, row.l);
    __syncthreads();
    const int fours = a.head_dim / 4;
    for (int i = threadIdx.x; i < rows * fours; i += 256) {
        const int r = i / fours, f = i % fours * 4;
        float m = s_ml[0][r].x, l = 0.f, by[4];
        for (int w = 1; w < 4; ++w) m = fmaxf(m, s_ml[w][r].x);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            by[w] = s_ml[w][r].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_ml[w][r].x - m);
            l = fmaf(s_ml[w][r].y, by[w], l);
            const float4 x = *(const float4*)(sums + (w * 32 + r) * DP + f);
            o = make_float4(fmaf(x.x, by[w], o.x), fmaf(x.y, by[w], o.y), fmaf(x.z, by[w], o.z), fmaf(x.w, by[w], o.w));
        }
        const int qi = (int)over_group(a, r), head = hk * a.group + r - qi * a.group;
        const int64_t token = q.q0 + qi, at = token * a.heads + head;
        if (a.parts > 1) {
            const int64_t mine = part * a.n_q * a.heads + at;
            *(float4*)(a.part_o + mine * a.head_dim + f) = o;
            if (f == 0) a.part_ml[mine] = make_float2(m, l);
            continue;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
        T* out = (T*)a.out_w + token * a.os.row + head * a.os.head + f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const T x = (T)v[j];
            out[j] = x;
            if (a.rest_w) ((bf16*)a.rest_w)[at * a.head_dim + f + j] = (bf16)(v[j] - (float)x);
        }
        if (f == 0 && a.lse_w) a.lse_w[(int64_t)head * a.n_q + token] = lse_of(m, l);
    }
}

// The parts of a row put together by a workgroup's four wavefronts, each a fourth of them; lane f has elements f and f + 64.
template <typename T>
__global__ __launch_bounds__(256) void join_few_kernel(Args a) {
    __shared__ float s_l[4], s_o[4][128];
    const int s = a.seq0 + (int)blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = blockIdx.x;
    Seq q;
    if (!sequence(a, s, q) || (int64_t)i >= (int64_t)q.qn * a.heads) return;
    const int64_t row = (int64_t)q.q0 * a.heads + i, token = q.q0 + i / a.heads;
    const int head = i % a.heads, block = (i / a.heads * a.group + head % a.group) / FIXED;
    const int parts = shares(key_tiles(a, q, block * FIXED), a.parts, a.part_tiles);
    const int64_t step = a.n_q * a.heads;
    float m = -INFINITY;
    for (int p = lane; p < parts; p += 64) m = fmaxf(m, a.part_ml[p * step + row].x);
    m = wave_max(m);
    float l = 0.f, x = 0.f, y = 0.f;
    const bool first = lane < a.head_dim, second = lane + 64 < a.head_dim;
#pragma unroll 4
    for (int p = wave; p < parts; p += 4) {
        const float2 ml = a.part_ml[p * step + row];
        const float* o = a.part_o + (p * step + row) * a.head_dim + lane;
        const float u = first ? o[0] : 0.f, v = second ? o[64] : 0.f;
        const float by = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
        l = fmaf(ml.y, by, l);
        x = fmaf(u, by, x);
        y = fmaf(v, by, y);
    }
    s_o[wave][lane] = x;
    s_o[wave][lane + 64] = y;
    if (lane == 0) s_l[wave] = l;
    __syncthreads();
    if (wave != 0) return;
    l = (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]);
    x = (s_o[0][lane] + s_o[1][lane]) + (s_o[2][lane] + s_o[3][lane]);
    y = (s_o[0][lane + 64] + s_o[1][lane + 64]) + (s_o[2][lane + 64] + s_o[3][lane + 64]);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = (T*)a.out_w + token * a.os.row + head * a.os.head;
    bf16* rest = (bf16*)a.rest_w + row * a.head_dim;
    auto put = [&](int e, float o) {
        const T t = (T)o;
        out[e] = t;
        if (a.rest_w) rest[e] = (bf16)(o - (float)t);
    };
    if (first) put(lane, x * inv);
    if (second) put(lane + 64, y * inv);
    if (a.lse_w && lane == 0) a.lse_w[(int64_t)head * a.n_q + token] = lse_of(m, l);
}

// The same where rows are many and parts few, a thread four neighbours of a row.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Args a) {
    const int s = a.seq0 + (int)blockIdx.y;
    Seq q;
    if (!sequence(a, s, q)) return;
    const int fours = a.head_dim / 4;
    const int64_t n = (int64_t)q.qn * a.heads * fours, step = a.n_q * a.heads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int mine = (int)(i / fours), f = (int)(i - (int64_t)mine * fours) * 4, qi = mine / a.heads, head = mine - qi * a.heads;
        const int64_t token = q.q0 + qi, row = token * a.heads + head;
        const int parts = shares(key_tiles(a, q, (qi * a.group + head % a.group) / FIXED * FIXED), a.parts, a.part_tiles);
        float m = -INFINITY, l = 0.f;
        for (int p = 0; p < parts; ++p) m = fmaxf(m, a.part_ml[p * step + row].x);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            const float2 ml = a.part_ml[p * step + row];
            const float4 x = *(const float4*)(a.part_o + (p * step + row) * a.head_dim + f);
            const float by = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
            l = fmaf(ml.y, by, l);
            o = make_float4(fmaf(x.x, by, o.x), fmaf(x.y, by, o.y), fmaf(x.z, by, o.z), fmaf(x.w, by, o.w));
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        T* const out = (T*)a.out_w + token * a.os.row + head * a.os.head + f;
        if constexpr (sizeof(T) == 2) {
            const uint2 x = make_uint2(cvt_pk_bf16(o.x, o.y), cvt_pk_bf16(o.z, o.w));
            *(uint2*)out = x;
            if (a.rest_w)
                *(uint2*)((bf16*)a.rest_w + row * a.head_dim + f) =
                    make_uint2(cvt_pk_bf16(o.x - __uint_as_float(x.x << 16), o.y - __uint_as_float(x.x & 0xffff0000u)),
                               cvt_pk_bf16(o.z - __uint_as_float(x.y << 16), o.w - __uint_as_float(x.y & 0xffff0000u)));
        } else {
            *(float4*)out = o;
        }
        if (a.lse_w && f == 0) a.lse_w[(int64_t)head * a.n_q + token] = lse_of(m, l);
    }
}

// Smallest and largest document of every DOC_BLOCK tokens, a wavefront each; padding counts as -1.
__global__ __launch_bounds__(256) void documents_kernel(Args a) {
    const int queries = blockIdx.z, s = a.seq0 + (int)blockIdx.y, lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    Seq q;
    if (!sequence(a, s, q)) return;
    const int n = queries ? q.qn : q.kn, first = queries ? q.q0 : q.k0;
    if (b * DOC_BLOCK >= n) return;
    const int32_t* docs = queries ? a.q_docs : a.k_docs;
    int lo = max(docs[first + min(b * DOC_BLOCK + lane, n - 1)], -1), hi = lo;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        lo = min(lo, __shfl_xor(lo, o, 64));
        hi = max(hi, __shfl_xor(hi, o, 64));
    }
    if (lane == 0) (queries ? a.q_blocks : a.k_blocks)[doc_block0(first, s) + b] = make_int2(lo, hi);
}

// Where no sequence may have rows, and no launch over rows finds the faulty ones.
__global__ __launch_bounds__(256) void check_kernel(Args a) {
    const int s = (int)(blockIdx.x * 256 + threadIdx.x);
    Seq q;
    if (s < a.n_seq && !sequence(a, s, q)) report_fault(a.status, PS_ST_BAD_LENGTH, s);
}

template <typename T, int DP>
void launch_attend(const Args& a, hipStream_t st) {
    const int64_t per_seq = (int64_t)a.kv_heads * a.row_blocks * a.parts;
    Args b = a;
    for (int32_t s0 = 0, n; s0 < a.n_seq; s0 += n) {
        const int64_t most = max((int64_t)1, (int64_t)(1 << 22) / per_seq);       // (a grid holds fewer than 2^32 threads)
        n = (int32_t)min((int64_t)(a.n_seq - s0), most);
        b.seq0 = s0;
        b.seqs = n;
        b.together = turns(per_seq, n);
        b.listed = add_up(n, a.row_blocks, a.parts);
        const dim3 grid((unsigned)(per_seq * n));
        if (a.few)
            hipLaunchKernelGGL((attend_few_kernel<T, DP>), grid, dim3(256), 0, st, b);
        else if (a.parts > 1)
            hipLaunchKernelGGL((attend_kernel<T, DP, true>), grid, dim3(256), 0, st, b);
        else
            hipLaunchKernelGGL((attend_kernel<T, DP, false>), grid, dim3(256), 0, st, b);
    }
    if (a.parts == 1) return;
    for (int32_t s0 = 0, n; s0 < a.n_seq; s0 += n) {
        n = min(a.n_seq - s0, 32768);
        b.seq0 = s0;
        // few rows have many parts and the chip to themselves; of many, threads have four elements each (25600 rows of 4 parts 9 us, a wavefront
        // a row 22, four wavefronts 53)
        const int64_t rows = (int64_t)a.max_q * a.heads;
        if (a.n_q * a.heads <= 4096)
            hipLaunchKernelGGL(join_few_kernel<T>, dim3((unsigned)rows, (unsigned)n), dim3(256), 0, st, b);
        else
            hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)min((rows * (a.head_dim / 4) + 255) / 256, (int64_t)4096), (unsigned)n), dim3(256), 0, st, b);
    }
}

// Rows and heads at multiples of 16 bytes.
bool good_strides(const ps_attention_desc* d, const ps_strides& s) {
    const int64_t align = d->dtype == 1 ? 8 : 4;
    return s.row >= 0 && s.head >= 0 && s.row % align == 0 && s.head % align == 0;
}

}  // namespace

namespace seqatt {

// Whether workgroups add up what work there is: where blocks are shared out, which leaves much of the grid without any.  Of whole blocks
// the empty ones do not matter (64 sequences of 4 to 512 tokens, forwards / keys' gradients 37 / 53 us either way).
bool add_up(int32_t seqs, int64_t blocks, int32_t parts) { return seqs <= 64 && blocks <= 64 && parts > 1; }

// A tensor that a call reads or writes.  Heads or rows of a written one may not fall on one another.
int check_strides(const ps_attention_desc* d, const ps_strides& s, const void* base, int64_t rows, int64_t heads, bool written) {
    if (!base || ((uintptr_t)base & 15) != 0 || !good_strides(d, s)) return PS_EINVAL;
    return written && !strides_apart(s, rows, heads, d->head_dim) ? PS_EINVAL : PS_OK;
}

int plan(const ps_attention_desc* d, const ps_attention_seqs* s, bool backward, void* workspace, Plan& p) {
    if (!d || d->n_seq < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0 || d->head_dim < 1 || d->max_q < 0 ||
        d->max_k < 0 || d->n_q < 0 || d->n_k < 0 || d->n_q > INT32_MAX || d->n_k > INT32_MAX || (d->dtype != 0 && d->dtype != 1) ||
        (d->causal != 0 && d->causal != 1))
        return PS_EINVAL;
    if (!(d->scale > 0.f) || !(d->softcap >= 0.f) || isinf(d->scale) || isinf(d->softcap)) return PS_EINVAL;
    if (d->head_dim > 128 || d->head_dim % 8 != 0) return PS_EUNSUPPORTED;
    const int64_t group = d->heads / d->kv_heads;
    if (max(min((int64_t)d->max_q, d->n_q), min((int64_t)d->max_k, d->n_k)) > 1 << 30) return PS_EUNSUPPORTED;   // (places stay in 32 bits)
    if (group > 32768 || (int64_t)d->max_q * group >= ((int64_t)1 << 31) / group) return PS_EUNSUPPORTED;
    if (d->heads > 65536) return PS_EUNSUPPORTED;
    Args& a = p.a;
    memset(&a, 0, sizeof(a));
    if (s) {
        if (!s->q_offsets || !s->k_offsets || !s->q_docs != !s->k_docs) return PS_EINVAL;
        a.q_offsets = s->q_offsets; a.k_offsets = s->k_offsets; a.k_lengths = s->k_lengths; a.q_start = s->q_start;
        a.prefix = s->prefix; a.q_docs = s->q_docs; a.k_docs = s->k_docs; a.slopes = s->slopes;
    }
    a.qs = d->q; a.ks = d->k; a.vs = d->v; a.os = d->out; a.gs = d->dout; a.dqs = d->dq; a.dks = d->dk; a.dvs = d->dv;
    a.n_q = d->n_q; a.n_k = d->n_k; a.n_seq = d->n_seq; a.heads = d->heads; a.kv_heads = d->kv_heads; a.head_dim = d->head_dim;
    a.group = (int32_t)group; a.max_q = (int32_t)min((int64_t)d->max_q, d->n_q); a.max_k = (int32_t)min((int64_t)d->max_k, d->n_k); a.causal = d->causal;
    a.scale = d->scale;
    a.cap = d->softcap < 0x1p100f ? d->softcap : 0.f;                     // (above, it bends no score by a place, and cap log2(e) is no float)
    a.slope_by = a.cap > 0.f ? LOG2E : 1.f / d->scale;
    a.cap_in = a.cap > 0.f ? d->scale / a.cap : 0.f;
    a.by_group = group > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint64_t)group + 1) : 0;
    a.row_blocks = (int32_t)(((int64_t)a.max_q * group + FIXED - 1) / FIXED);
    // Blocks that do not fill the chip, or of which the longest would be waited for: their tiles are shared out, so that there are
    // some 2048 shares of a length, of 256 keys (rows) or more each (fp32, one sequence of 3571, 12 heads of 80: 1024, 2048, 4096 shares 1766, 1602,
    // 1684 us a pass; bf16, 8192 tokens of 4 heads of 64: 430, 432, 620).  What blocks and tiles there are is estimated from the tensors'
    // rows: lengths stand on the device.
    a.tile = tile_rows(d->dtype == 1 ? 2 : 4);
    a.key_tile = key_tile_rows(d->dtype == 1 ? 2 : 4, padded(d->head_dim));
    auto share = [&](int64_t blocks_a_seq, int64_t tokens, int64_t tokens_a_block, int64_t passing, int64_t all_passing, int tile, int32_t& parts,
                     int32_t& part_tiles, int64_t chain) {
        const int tiles = (int)((passing + tile - 1) / tile);
        const int64_t all_tiles = all_passing / tile + a.n_seq;
        const int64_t blocks = a.kv_heads * min((int64_t)a.n_seq * blocks_a_seq, tokens / tokens_a_block + a.n_seq);
        parts = 1;
        part_tiles = tiles;
        const int least = blocks < 128 && passing > chain ? 64 : 256;
        if (blocks >= 512 || tiles < 2 * least / tile) return;
        const int64_t jobs = a.kv_heads * all_tiles * max((int64_t)1, blocks / max(1, a.n_seq * a.kv_heads));
        part_tiles = (int32_t)min((int64_t)tiles, max((int64_t)least / tile, jobs / 2048));
        // (what the shares leave to be added up stays within 256 MB)
        const int64_t most = max((int64_t)1, ((int64_t)64 << 20) / max((int64_t)1, tokens * a.kv_heads * a.head_dim));
        part_tiles = (int32_t)max((int64_t)part_tiles, (tiles + most - 1) / most);
        parts = (tiles + part_tiles - 1) / part_tiles;
    };
    const int64_t rows_a_seq = (int64_t)a.max_q * group;
    // Few rows: shares of 16 tiles or more (four a wavefront), so many that there are some 256 of up to 32 tiles, and of longer ones some
    // 1024, long sequences' and short ones' (one cache of 65521 keys, 4 heads of 128: 256 shares 28.5 us, 512 33.7).
    a.few = !backward && (int64_t)a.max_q * group <= 32;
    if (a.few) {
        a.tile = 32;
        const int64_t tiles = ((int64_t)a.max_k + 31) / 32, jobs = a.kv_heads * (d->n_k / 32 + d->n_seq);
        const int64_t most = max((int64_t)1, ((int64_t)64 << 20) / max((int64_t)1, d->n_q * d->heads * d->head_dim));
        a.part_tiles = (int32_t)max(max(min(max((int64_t)16, jobs / 256), (int64_t)32), jobs / 1024), (tiles + most - 1) / most);
        a.parts = (int32_t)max((int64_t)1, (tiles + a.part_tiles - 1) / a.part_tiles);
    } else {
        share(a.row_blocks, d->n_q * group, FIXED, a.max_k, d->n_k, a.tile, a.parts, a.part_tiles, INT32_MAX);
    }
    // Of few blocks of keys, shares of 64 rows: a block's chain of tiles, the rows of all its head's heads, is all that takes time.  The sum's launch
    // is worth it above 256 rows, 128 in fp32 (passes of 1 sequence of 191 tokens, 48 heads on 12, 61 -> 52 us; 14 of up to 70, 16 heads of 128 on
    // 4, 49 -> 43; fp32, 4 of 56, 4 heads on 1, 82 -> 56; 4 of 128 rows, 12 heads, would take 34 for 28).
    share((a.max_k + FIXED - 1) / FIXED, d->n_k, FIXED, rows_a_seq, d->n_q * group, a.key_tile, a.key_parts, a.key_part_tiles, d->dtype == 1 ? 256 : 128);
    // (a grid holds fewer than 2^32 threads)
    if ((int64_t)a.kv_heads * a.row_blocks * a.parts >= 1 << 24 || (int64_t)a.kv_heads * ((a.max_k + FIXED - 1) / FIXED) * a.key_parts >= 1 << 24)
        return PS_EUNSUPPORTED;
    size_t off = 0;
    uint8_t* base = (uint8_t*)workspace;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return (void*)(base + at);
    };
    // (a launch for the summaries, 4.7 us in each direction, takes longer than the few tiles of short sequences that they would rule out: 16
    // sequences of up to 64 tokens, the other three launches 53 us with them, 50 without)
    if (max(a.max_q, a.max_k) > 256) {
        a.q_blocks = (int2*)take(sizeof(int2) * (size_t)(d->n_q / DOC_BLOCK + d->n_seq + 1));
        a.k_blocks = (int2*)take(sizeof(int2) * (size_t)(d->n_k / DOC_BLOCK + d->n_seq + 1));
    }
    const size_t rows = (size_t)d->n_q * d->heads;
    if (a.parts > 1) {
        a.part_o = (float*)take(sizeof(float) * rows * d->head_dim * a.parts);
        if (!backward) a.part_ml = (float2*)take(sizeof(float2) * rows * a.parts);
    }
    if (backward) {
        a.row_lse = (float*)take(sizeof(float) * rows);
        a.row_delta = (float*)take(sizeof(float) * rows);
        if (a.key_parts > 1) {
            const size_t part = sizeof(float) * (size_t)d->n_k * d->kv_heads * d->head_dim * a.key_parts;
            a.part_dk = (float*)take(part);
            a.part_dv = (float*)take(part);
        }
    }
    p.bytes = off > 0 ? off : 256;     // (0 says that a call is refused)
    return PS_OK;
}

void summarise_documents(const Args& a, hipStream_t st) {
    if (!a.q_docs || !a.q_blocks) return;
    Args b = a;
    for (int32_t s0 = 0, n; s0 < a.n_seq; s0 += n) {
        n = min(a.n_seq - s0, 32768);
        b.seq0 = s0;
        const int blocks = (max(a.max_q, a.max_k) + DOC_BLOCK - 1) / DOC_BLOCK;
        if (blocks > 0)
            hipLaunchKernelGGL(documents_kernel, dim3((unsigned)((blocks + 3) / 4), (unsigned)n, 2), dim3(256), 0, st, b);
    }
}

int check_sequences(const Args& a, hipStream_t st) {
    if (!a.status || a.n_seq == 0) return PS_OK;
    (void)hipGetLastError();
    hipLaunchKernelGGL(check_kernel, dim3(((unsigned)a.n_seq + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

}  // namespace seqatt

extern "C" size_t ps_attention_workspace_bytes(const ps_attention_desc* desc, int backward) {
    Plan p, b;
    if (plan(desc, nullptr, false, nullptr, p) != PS_OK || plan(desc, nullptr, true, nullptr, b) != PS_OK) return 0;
    return backward && b.bytes > p.bytes ? b.bytes : p.bytes;
}

extern "C" int ps_attention_forward(const ps_attention_desc* desc, const ps_attention_seqs* seqs, const void* q, const void* k,
                                    const void* v, void* out, float* lse, void* out_rest, void* workspace, size_t workspace_bytes,
                                    ps_status* status, void* hip_stream) {
    Plan p;
    if (!seqs) return PS_EINVAL;
    const int code = plan(desc, seqs, false, workspace, p);
    if (code != PS_OK) return code;
    p.a.status = status;
    if (p.a.n_seq == 0 || p.a.max_q == 0) return check_sequences(p.a, (hipStream_t)hip_stream);
    if (check_strides(desc, desc->q, q, desc->n_q, desc->heads, false) ||
        check_strides(desc, desc->out, out, desc->n_q, desc->heads, true)) return PS_EINVAL;
    if (p.a.n_k > 0 && (check_strides(desc, desc->k, k, desc->n_k, desc->kv_heads, false) ||
                         check_strides(desc, desc->v, v, desc->n_k, desc->kv_heads, false)))
        return PS_EINVAL;
    if (((uintptr_t)out_rest & 15) != 0 || (out_rest && desc->dtype != 1) || (uintptr_t)lse % 4 != 0) return PS_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < p.bytes) return PS_EWORKSPACE;
    Args& a = p.a;
    a.q = q; a.k = k; a.v = v; a.out_w = out; a.lse_w = lse; a.rest_w = out_rest;
    hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();
    if (!a.few) summarise_documents(a, st);
    switch (padded(desc->head_dim)) {
        case 64: desc->dtype == 1 ? launch_attend<bf16, 64>(a, st) : launch_attend<float, 64>(a, st); break;
        case 96: desc->dtype == 1 ? launch_attend<bf16, 96>(a, st) : launch_attend<float, 96>(a, st); break;
        default: desc->dtype == 1 ? launch_attend<bf16, 128>(a, st) : launch_attend<float, 128>(a, st);
    }
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
