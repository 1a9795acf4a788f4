// Gradients of the attention of seq_attention_fwd.hip, in two launches: that of the queries (queries fixed, keys passing), which also
// leaves each row's dout . out, and those of keys and values (keys fixed, queries passing).  Scores are computed again in both;
// every gradient is then a sum in one wavefront's registers, in an order that the shapes fix.  Where blocks do not fill the chip
// their passing tiles are shared out, and a launch more adds up the shares, one after the other.
#include "seq_attention.h"

using namespace seqatt;
typedef __bf16 bf16;

namespace {

// The weights p and the gradients d of x = scale q . k (by_x() times d) of one block, from the products s = q . k and g = dout . v, with
// four neighbours to every j: lse(j) and delta(j), what their queries bring along; distance(j), how far they stand from their keys, times
// the slope; in_front(j, is) if the block is cut, which of the keys stand in front of their query's end; same(j, is) if it is of several
// documents, which are of their query's.  STEP fours at a time: what is the same for all of them is asked once a step, so four at a time
// make straight lines (two rows of 8192 tokens, queries' / keys' gradients 191 / 210 -> 160 / 181 us), and one keeps few registers waiting.
// rest: what the rounding of d to bf16 leaves.  Where a row's weight lies on few keys it does not average out, and what those keys have in
// common is multiplied by the sum of the roundings instead of the sum of d, which is zero.  So where weights are like that, in blocks that
// a mask cuts (rows see few keys) and under a cap (scores are large), a second product makes up for it: 16 x 2048 with prefix and cap,
// queries' / keys' gradients 499 / 860 -> 589 / 977 us, error against 64 bits 2.7e-3 -> 2.1e-3 of the norm (1.7e-3 is that of dq's and dk's
// own rounding; 2.3e-3 without cap, where a product more would cost 5 to 10 %).  (Documents in two rows of 8192, where blocks are cut: 130 / 146
// -> 144 / 160.)
template <typename T, int STEP, typename Lse, typename Delta, typename Distance, typename Front, typename Same>
__device__ __forceinline__ void gradients(const Args& a, const f32x16& s, const f32x16& g, Weights<T>& p, Weights<T>& d, Weights<T>& rest,
                                          bool cut, bool docs, Lse lse, Delta delta, Distance distance, Front in_front, Same same) {
    const Cap cap = Cap::of<T>(a);
    const float c1 = a.scale * LOG2E;
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += STEP) {
        float4 u[STEP], v[STEP];
#pragma unroll
        for (int k = 0; k < STEP; ++k) u[k] = lse(j0 + k);
        if (a.slopes) {
#pragma unroll
            for (int k = 0; k < STEP; ++k) {
                const float4 off = distance(j0 + k);
                u[k] = make_float4(u[k].x + off.x, u[k].y + off.y, u[k].z + off.z, u[k].w + off.w);
            }
        }
        if (a.cap > 0.f) {
            auto bend = [&](auto far) {
#pragma unroll
                for (int e = 0; e < 4 * STEP; ++e) {
                    const float b = cap.bent<T, far>(s[4 * j0 + e]);
                    float& w = (&u[e >> 2].x)[e & 3];
                    w = __builtin_amdgcn_exp2f(cap.score<T, far>(b, w));
                    (&v[e >> 2].x)[e & 3] = Cap::slope<T, far>(b) * w;
                }
            };
            if (Cap::far<T>(a))
                bend(std::true_type());
            else
                bend(std::false_type());
        } else {
#pragma unroll
            for (int e = 0; e < 4 * STEP; ++e) {
                float& w = (&u[e >> 2].x)[e & 3];
                w = __builtin_amdgcn_exp2f(fmaf(s[4 * j0 + e], c1, -w));
                (&v[e >> 2].x)[e & 3] = w;
            }
        }
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            const float4 t = delta(j0 + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) (&v[k].x)[i] *= g[4 * (j0 + k) + i] - (&t.x)[i];
        }
        auto only = [&](auto seen) {
#pragma unroll
            for (int k = 0; k < STEP; ++k) {
                bool is[4];
                seen(j0 + k, is);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    (&u[k].x)[i] = is[i] ? (&u[k].x)[i] : 0.f;
                    (&v[k].x)[i] = is[i] ? (&v[k].x)[i] : 0.f;
                }
            }
        };
        if (cut) only(in_front);
        if (docs) only(same);
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            p.set(j0 + k, u[k]);
            d.set(j0 + k, v[k]);
        }
        if constexpr (sizeof(T) == 2)
            if (cut || docs || a.cap > 0.f) {
#pragma unroll
                for (int k = 0; k < STEP; ++k) {
                    const float4 r = d.get(j0 + k);
                    rest.set(j0 + k, make_float4(v[k].x - r.x, v[k].y - r.y, v[k].z - r.z, v[k].w - r.w));
                }
            }
    }
}

template <typename T>
__device__ __forceinline__ float by_x(const Args& a) { return a.cap > 0.f && sizeof(T) == 2 ? 4.f * a.scale : a.scale; }

// Keys fixed: dk and dv of FIXED keys of a key head, from the rows of all its heads.  Four products a tile (a fifth for the rest), and twice the
// accumulators of the queries' launch, which leaves two workgroups a unit (one in fp32 above 64 features).  Bound by waits, as forwards: 16 x 2048
// with prefix and cap, heads of 128, 978 us, 0.48 PFLOP/s, vector units issuing 31 % and matrix units busy 24 % of the time, 1.3 wavefronts a
// SIMD at barriers and waits 36 % of theirs; documents in two rows of 8192, heads of 64: 166 us, 0.44 PFLOP/s, 33 %, 22 %, 1.6 wavefronts, 40 %.
// Where the heads of a key head are no divisor of a tile's rows, addresses are worked out a row at a time, which costs some 15 % (8 causal sequences
// of 1500 to 2048, 4 key heads of 64, this launch with 2, 3, 4, 5 heads to each: 119, 182, 198, 282 us).
template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 64 || sizeof(T) == 2 ? 2 : 1) void key_gradients_kernel(Args a) {
    using L = Tile<T, DP, key_tile_rows(sizeof(T), DP)>;
    // Two workgroups a unit need 256 registers a lane.  In bf16 the gradients of 32 keys by 128 features take half of them, so the values
    // wait in LDS (a quarter more reads there).
    constexpr bool IN_LDS = sizeof(T) == 2 && DP == 128;
    __shared__ __align__(1024) unsigned char s_values[IN_LDS ? 4 : 1][IN_LDS ? 32 * L::ROWB : 16];
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][queries, dout]
    __shared__ __align__(16) float s_lse[2][64], s_delta[2][64], s_slope[2][64], s_place[2][64];   // (places from k0 on)
    __shared__ __align__(16) int s_doc[2][64];

    Seq q;
    Work w;
    if (!find_work<true>(a, q, w)) return;                                // (faulty sequences: reported by the queries' launch)
    const int hk = w.hk, s = w.s, part = w.part, k0 = w.block * FIXED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int rows = q.qn * a.group;
    int first_tile;
    const int tiles = row_tiles(a, q, k0, first_tile);
    const int t0 = first_tile + part * a.key_part_tiles, t1 = min(tiles, t0 + a.key_part_tiles);
    if (part > 0 && t0 >= tiles) return;                                  // (part 0 writes, rows or not)

    // this lane's key
    const int wk0 = k0 + 32 * wave, key = wk0 + col;
    const bool live = key < q.kn;
    const int64_t token = q.k0 + min(key, q.kn - 1);
    const int doc = a.k_docs ? a.k_docs[token] : 0;
    const bool there = live && doc >= 0;
    const Lanes<T, DP> lanes(lane);
    Fixed<T, DP> kf, v;
    kf.load((const T*)a.k + token * a.ks.row + hk * a.ks.head, there, a.head_dim, half);
    v.load((const T*)a.v + token * a.vs.row + hk * a.vs.head, there, a.head_dim, half);
    auto keep = [&] {
        if constexpr (IN_LDS)
            return FixedInLds<T, DP>(s_values[wave], v, lanes);
        else
            return v;
    };
    const auto vf = keep();

    const float keyf = (float)(32 * wave + col), seen_from = !a.causal || key < q.prefix ? -INFINITY : keyf;   // places from k0 on
    const int last = min(k0 + FIXED, q.kn) - 1, wlast = min(wk0 + 31, q.kn - 1);
    int dmin = 0, dmax = 0;
    if (a.k_docs) {
        const int x = a.k_docs[q.k0 + min(k0 + lane, last)], y = a.k_docs[q.k0 + min(k0 + 64 + lane, last)];
        dmin = min(x, y);
        dmax = max(x, y);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            dmin = min(dmin, __shfl_xor(dmin, o, 64));
            dmax = max(dmax, __shfl_xor(dmax, o, 64));
        }
    }
    const int64_t qblock0 = doc_block0(q.q0, s);
    auto classify = [&](int t, bool& one, bool& pad) {
        const int first = (int)over_group(a, t * L::ROWS), end = (int)over_group(a, min(t * L::ROWS + L::ROWS, rows) - 1);
        bool some = !a.causal || k0 <= q.start + end || k0 < q.prefix;
        one = !a.q_docs;
        if (a.q_docs && !a.q_blocks) {
            pad = true;
        } else if (a.q_docs && some) {
            const int2 m = a.q_blocks[qblock0 + first / DOC_BLOCK], n = a.q_blocks[qblock0 + end / DOC_BLOCK];
            const int lo = min(m.x, n.x), hi = max(m.y, n.y);
            some = dmax >= 0 && hi >= max(dmin, 0) && lo <= dmax;
            one = lo == hi && dmin == dmax && lo == dmin;
            pad = lo < 0;
        }
        return some;
    };

    const Sender<T, DP, L::ROWS> queries(a.qs, a.group, a.head_dim), gradients_out(a.gs, a.group, a.head_dim);
    const bool regular = queries.regular && gradients_out.regular;
    const T *qbase = (const T*)a.q + q.q0 * a.qs.row + (int64_t)hk * a.group * a.qs.head, *gbase = (const T*)a.dout + q.q0 * a.gs.row + (int64_t)hk * a.group * a.gs.head;
    // What a tile's rows bring along, words that each of the wavefronts has one of: lse, dout . out, slope, document.
    const int steps = L::ROWS / a.group;                                  // tokens from tile to tile, if regular
    const int lane_token = (int)over_group(a, lane % L::ROWS), lane_head = hk * a.group + lane % L::ROWS - lane_token * a.group;
    float* const words = wave == 0 ? s_lse[0] : wave == 1 ? s_delta[0] : wave == 2 ? s_slope[0] : (float*)s_doc[0];
    const bool has_words = wave < 2 || (wave == 2 ? a.slopes != nullptr : a.q_docs != nullptr);
    const int word_step = wave == 2 ? 0 : steps;
    auto word = [&](int64_t token, int head) -> const void* {
        return wave < 2 ? (wave == 0 ? a.row_lse : a.row_delta) + head * a.n_q + token : wave == 2 ? (const void*)(a.slopes + head) : (const void*)(a.q_docs + token);
    };
    // What a lane needs for that only once a tile, the offsets of its chunks and its first word's address, waits in LDS where registers
    // are short: spilled to memory it would be read behind the tile just sent for, and waited for with it.
    constexpr int PER = L::PER_THREAD;
    struct Needs {
        unsigned q[PER], g[PER];
        const int32_t* word;
    } needs;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        needs.q[j] = queries.off[j];
        needs.g[j] = gradients_out.off[j];
    }
    needs.word = (const int32_t*)word(q.q0 + lane_token, lane_head);
    __shared__ Needs s_needs[IN_LDS ? 256 : 1];
    if (IN_LDS) s_needs[threadIdx.x] = needs;
    auto fetch = [&]() -> Needs { return IN_LDS ? s_needs[threadIdx.x] : needs; };
    auto request = [&](int t, bool padded, int buf) {
        const int r0 = t * L::ROWS;
        if (regular && r0 + L::ROWS <= rows && !padded) {
            const int64_t token = t * steps;
            const Needs mine = fetch();
            Sender<T, DP, L::ROWS>::whole(smem[buf][0], qbase + token * a.qs.row, mine.q);
            Sender<T, DP, L::ROWS>::whole(smem[buf][1], gbase + token * a.gs.row, mine.g);
            if (has_words) send_words(words + 64 * buf, mine.word + (int64_t)t * word_step);
            if (wave == 0) s_place[buf][lane] = (float)(q.start - k0 + (int)token + (int)over_group(a, lane % L::ROWS));
            return;
        }
        // (padding and rows past the end are zeros that see nothing)
        auto row = [&](const T* base, const ps_strides& st, int i) -> const T* {
            const int qi = (int)over_group(a, min(r0 + i, rows - 1)), head = r0 + i - qi * a.group;
            return base + qi * st.row + head * st.head;
        };
        const int r = min(r0 + lane, rows - 1), qi = (int)over_group(a, r), of = padded ? a.q_docs[q.q0 + qi] : 0;
        const uint64_t there = __ballot(r0 + lane < rows && of >= 0);
        Sender<T, DP, L::ROWS>::rows(smem[buf][0], a.head_dim, there, [&](int i) { return row(qbase, a.qs, i); });
        Sender<T, DP, L::ROWS>::rows(smem[buf][1], a.head_dim, there, [&](int i) { return row(gbase, a.gs, i); });
        const void* none = wave == 0 ? (const void*)&infinity_word : wave == 3 ? (const void*)&minus_one : (const void*)&zeros;
        if (has_words) send_words(words + 64 * buf, r0 + lane < rows ? word(q.q0 + qi, hk * a.group + r - qi * a.group) : none);
        if (wave == 0) s_place[buf][lane] = (float)(q.start - k0 + qi);
    };

    f32x16 dk[L::NA], dv[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[i][e] = dv[i][e] = 0.f;

    Walk walk;
    int t = walk.next(t0, t1, classify), buf = 0;
    if (t < t1) request(t, walk.is_padded(t), 0);
    while (t < t1) {
        const bool docs = !walk.is_one(t), cut = a.causal && wlast > q.start + (int)over_group(a, t * L::ROWS) && wlast >= q.prefix;
        const int far = q.start + (int)over_group(a, min(t * L::ROWS + L::ROWS, rows) - 1);
        t = walk.next(t + 1, t1, classify);
        vm_wait();
        __syncthreads();                                                  // the tile has landed, the one before it is no longer read
        if (t < t1) request(t, walk.is_padded(t), buf ^ 1);
        if (wk0 < q.kn && !(a.causal && wk0 > far && wk0 >= q.prefix)) {
#pragma unroll 1
            for (int b = 0; b < L::BLOCKS; ++b) {                         // (one after the other: registers)
                f32x16 sc, g;
                dots<T, DP>(smem[buf][0], b, kf, sc, smem[buf][1], b, vf, g, lanes);
                Weights<T> p, d, rest;
                auto at = [&](int j) { return 32 * b + 8 * j + 4 * half; };
                gradients<T, (DP > 64 ? 1 : 4)>(a, sc, g, p, d, rest, cut, docs, [&](int j) { return *(const float4*)&s_lse[buf][at(j)]; },
                             [&](int j) { return *(const float4*)&s_delta[buf][at(j)]; },
                             [&](int j) {
                                 const float4 by = *(const float4*)&s_slope[buf][at(j)], place = *(const float4*)&s_place[buf][at(j)];
                                 return make_float4(by.x * LOG2E * fabsf(place.x - keyf), by.y * LOG2E * fabsf(place.y - keyf),
                                                    by.z * LOG2E * fabsf(place.z - keyf), by.w * LOG2E * fabsf(place.w - keyf));
                             },
                             [&](int j, bool(&is)[4]) {
                                 const float4 place = *(const float4*)&s_place[buf][at(j)];
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = seen_from <= (&place.x)[i];
                             },
                             // (padding: rows' weights are 0 by their lse, keys' because no row is of their documents)
                             [&](int j, bool(&is)[4]) {
                                 const int4 of = *(const int4*)&s_doc[buf][at(j)];
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = (&of.x)[i] == doc;
                             });
                weigh<T, DP>(smem[buf][1], b, p, dv, lanes);
                weigh<T, DP>(smem[buf][0], b, d, dk, lanes);
                if (sizeof(T) == 2 && (cut || docs || a.cap > 0.f)) weigh<T, DP>(smem[buf][0], b, rest, dk, lanes);
            }
        }
        buf ^= 1;
    }
    __syncthreads();                                                      // (tiles are no longer read)
    if (wk0 >= q.kn) return;
    unsigned char* const mine = smem[0][0] + wave * PUT_BYTES;
    static_assert(sizeof(smem) >= 4 * PUT_BYTES, "rows on their way out");
    const int own = wk0 + (anew<256>((int)threadIdx.x) & 31);              // (the key, worked out again)
    const bool is = own < q.kn;
    const int64_t to = q.k0 + own;
    if (a.key_parts > 1) {
        const int64_t at = (((int64_t)part * a.n_k + to) * a.kv_heads + hk) * a.head_dim;
        put_rows<float, DP>(mine, dk, 1.f, a.head_dim, is ? a.part_dk + at : nullptr);
        put_rows<float, DP>(mine, dv, 1.f, a.head_dim, is ? a.part_dv + at : nullptr);
        return;
    }
    put_rows<T, DP>(mine, dk, by_x<T>(a), a.head_dim, is ? (T*)a.dk + to * a.dks.row + hk * a.dks.head : nullptr);
    put_rows<T, DP>(mine, dv, 1.f, a.head_dim, is ? (T*)a.dv + to * a.dvs.row + hk * a.dvs.head : nullptr);
}

// Queries fixed: dq of FIXED rows of a key head's queries.  Three products a tile (a fourth for the rest).  Bound by waits too: 16 x 2048 with
// prefix and cap, heads of 128, 586 us, 0.59 PFLOP/s, vector units issuing 48 % and matrix units busy 34 % of the time, 1.7 wavefronts a SIMD
// waiting 22 % of theirs; documents in two rows of 8192, heads of 64: 147 us, 0.37 PFLOP/s, 33 %, 19 %, 1.5 wavefronts, 40 %.
template <typename T, int DP>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP > 64 ? 1 : 2) void query_gradients_kernel(Args a) {
    using L = Tile<T, DP>;
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][keys, values]
    __shared__ __align__(16) int s_doc[2][64];

    Seq q;
    Work w;
    if (!find_work<false>(a, q, w)) return;
    const int hk = w.hk, s = w.s, part = w.part, rows = q.qn * a.group, r0 = w.block * FIXED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int tiles = key_tiles(a, q, r0);
    const int t0 = part * a.part_tiles, t1 = min(tiles, t0 + a.part_tiles);
    if (t0 > 0 && t0 >= tiles) return;                                    // (part 0 writes, keys or not)

    const int wr0 = r0 + 32 * wave, r = min(wr0 + col, rows - 1);
    const bool live = wr0 + col < rows;
    const int qi = (int)over_group(a, r), head = hk * a.group + r - qi * a.group;
    const int64_t token = q.q0 + qi;
    const int place = q.start + qi;
    const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.f;
    const int doc = a.q_docs ? a.q_docs[token] : 0;
    const bool there = live && doc >= 0;
    Fixed<T, DP> qf, gf;
    qf.load((const T*)a.q + token * a.qs.row + head * a.qs.head, there, a.head_dim, half);
    gf.load((const T*)a.dout + token * a.gs.row + head * a.gs.head, there, a.head_dim, half);
    const Lanes<T, DP> lanes(lane);
    // what the row brings along, for this launch and the keys'
    float lse, delta;
    {
        Fixed<T, DP> of;
        of.load((const T*)a.out + token * a.os.row + head * a.os.head, there, a.head_dim, half);
        delta = gf.share(of);
        if (sizeof(T) == 2 && a.rest) {
            of.load((const T*)a.rest + (token * a.heads + head) * a.head_dim, there, a.head_dim, half);
            delta += gf.share(of);
        }
        const int64_t at = (int64_t)head * a.n_q + token;
        const float mine = there ? a.lse[at] : -INFINITY;
        lse = mine == -INFINITY ? INFINITY : mine * LOG2E;
        delta += __shfl_xor(delta, 32, 64);
        if (live && half == 0 && part == 0) {
            a.row_lse[at] = lse;
            a.row_delta[at] = delta;
        }
    }

    // keys in front of `end` are seen, if their documents are
    const int end = seen_end(a, q, place);
    const int last = min(r0 + FIXED, rows) - 1;
    const int far = q.start + (int)over_group(a, last);
    const int wfar = q.start + (int)over_group(a, min(wr0 + 31, rows - 1)), wnear = q.start + (int)over_group(a, min(wr0, rows - 1));
    int dmin = 0, dmax = 0;
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

    const T* kbase = (const T*)a.k + q.k0 * a.ks.row + hk * a.ks.head;
    const T* vbase = (const T*)a.v + q.k0 * a.vs.row + hk * a.vs.head;
    const Sender<T, DP, L::ROWS, true> keys(a.ks, 1, a.head_dim), values(a.vs, 1, a.head_dim);
    const bool regular = keys.regular && values.regular;
    auto request = [&](int t, bool padded, int buf) {
        const int k0 = t * L::ROWS;
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

    f32x16 dq[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[i][e] = 0.f;

    Walk walk;
    int t = walk.next(t0, t1, classify), buf = 0;
    if (t < t1) request(t, walk.is_padded(t), 0);
    while (t < t1) {
        const bool docs = !walk.is_one(t);
        const int k0 = t * L::ROWS;
        const bool cut = k0 + L::ROWS > q.kn || (a.causal && k0 + L::ROWS - 1 > wnear && k0 + L::ROWS > q.prefix);
        const float from = (float)(place - k0 - 4 * half);
        t = walk.next(t + 1, t1, classify);
        vm_wait();
        __syncthreads();                                                  // the tile has landed, the one before it is no longer read
        if (t < t1) request(t, walk.is_padded(t), buf ^ 1);
        if (wr0 < rows && !(a.causal && k0 > wfar && k0 >= q.prefix)) {
#pragma unroll 1
            for (int b = 0; b < L::BLOCKS; ++b) {                         // (one after the other: registers)
                f32x16 sc, g;
                dots<T, DP>(smem[buf][0], b, qf, sc, smem[buf][1], b, gf, g, lanes);
                Weights<T> p, d, rest;
                auto at = [&](int j) { return 32 * b + 8 * j + 4 * half; };
                const int left = end - k0 - 32 * b - 4 * half;
                const float off = from - (float)(32 * b);
                gradients<T, 4>(a, sc, g, p, d, rest, cut, docs, [&](int) { return make_float4(lse, lse, lse, lse); },
                             [&](int) { return make_float4(delta, delta, delta, delta); },
                             [&](int j) {
                                 return make_float4(slope * fabsf(off - (float)(8 * j)), slope * fabsf(off - (float)(8 * j + 1)),
                                                    slope * fabsf(off - (float)(8 * j + 2)), slope * fabsf(off - (float)(8 * j + 3)));
                             },
                             [&](int j, bool(&is)[4]) {
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = left > 8 * j + i;
                             },
                             // (padding is zeros on both sides, and its weights are 0 by its lse)
                             [&](int j, bool(&is)[4]) {
                                 const int4 of = *(const int4*)&s_doc[buf][at(j)];
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = (&of.x)[i] == doc;
                             });
                weigh<T, DP>(smem[buf][0], b, d, dq, lanes);
                if (sizeof(T) == 2 && (cut || docs || a.cap > 0.f)) weigh<T, DP>(smem[buf][0], b, rest, dq, lanes);
            }
        }
        buf ^= 1;
    }
    __syncthreads();                                                      // (tiles are no longer read)
    if (wr0 >= rows) return;
    unsigned char* const mine = smem[0][0] + wave * PUT_BYTES;
    static_assert(sizeof(smem) >= 4 * PUT_BYTES, "rows on their way out");
    if (a.parts > 1)
        put_rows<float, DP>(mine, dq, 1.f, a.head_dim,
                            live ? a.part_o + (((int64_t)part * a.n_q + token) * a.heads + head) * a.head_dim : nullptr);
    else
        put_rows<T, DP>(mine, dq, by_x<T>(a), a.head_dim, live ? (T*)a.dq + token * a.dqs.row + head * a.dqs.head : nullptr);
}

// A gradient's shares added up, a thread four neighbours: those of queries (z = 0), keys (1) and values (2).  3365 tokens, 8 heads of 80 on 4,
// up to 4 shares: 61 MB in 18 us.
template <typename T>
__global__ __launch_bounds__(256) void add_kernel(Args a, int z0) {
    const int z = z0 + (int)blockIdx.z, s = a.seq0 + (int)blockIdx.y;
    Seq q;
    if (!sequence(a, s, q)) return;
    const int heads = z == 0 ? a.heads : a.kv_heads, of = z == 0 ? a.parts : a.key_parts, each = z == 0 ? a.part_tiles : a.key_part_tiles;
    const ps_strides to = z == 0 ? a.dqs : z == 1 ? a.dks : a.dvs;
    // (calls of few blocks: all of a tensor's rows are counted in 32 bits)
    const int fours = a.head_dim / 4, n = (z == 0 ? q.qn : q.kn) * heads * fours, token0 = z == 0 ? q.q0 : q.k0;
    const int64_t step = (z == 0 ? a.n_q : a.n_k) * heads * fours;
    const float4* part = (const float4*)(z == 0 ? a.part_o : z == 1 ? a.part_dk : a.part_dv) + (int64_t)token0 * heads * fours;
    T* out = (T*)(z == 0 ? a.dq : z == 1 ? a.dk : a.dv);
    const float by = z == 2 ? 1.f : by_x<T>(a);
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const int row = i / fours, mine = row / heads, head = row % heads;
        int first = 0;
        const int tiles = z == 0 ? key_tiles(a, q, (mine * a.group + head % a.group) / FIXED * FIXED) : row_tiles(a, q, mine / FIXED * FIXED, first);
        const int parts = shares(tiles - first, of, each);
        float4 sum = part[i];
#pragma unroll 4
        for (int p = 1; p < parts; ++p) {
            const float4 v = part[p * step + i];
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        T* at = out + (token0 + mine) * to.row + head * to.head + i % fours * 4;
        if constexpr (sizeof(T) == 2)
            *(uint2*)at = make_uint2(cvt_pk_bf16(sum.x * by, sum.y * by), cvt_pk_bf16(sum.z * by, sum.w * by));
        else
            *(float4*)at = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
    }
}

template <typename T, int DP>
void launch(const Args& a, hipStream_t st) {
    Args b = a;
    auto in_turn = [&](int64_t per_seq, int64_t most_seqs, auto launch_one) {
        if (per_seq == 0) return;
        const int64_t most = min(most_seqs, max((int64_t)1, (int64_t)(1 << 22) / per_seq));   // (a grid holds fewer than 2^32 threads)
        for (int32_t s0 = 0, n; s0 < a.n_seq; s0 += n) {
            n = (int32_t)min((int64_t)(a.n_seq - s0), most);
            b.seq0 = s0;
            b.seqs = n;
            b.together = turns(per_seq, n);
            launch_one((unsigned)n);
        }
    };
    const int64_t row_jobs = (int64_t)a.kv_heads * a.row_blocks * a.parts;
    const int64_t key_blocks = (a.max_k + FIXED - 1) / FIXED, key_jobs = a.kv_heads * key_blocks * a.key_parts;
    in_turn(row_jobs, a.n_seq, [&](unsigned n) {
        b.listed = add_up(n, a.row_blocks, a.parts);
        hipLaunchKernelGGL((query_gradients_kernel<T, DP>), dim3((unsigned)row_jobs * n), dim3(256), 0, st, b);
    });
    in_turn(key_jobs, a.n_seq, [&](unsigned n) {
        b.listed = add_up(n, key_blocks, a.key_parts);
        hipLaunchKernelGGL((key_gradients_kernel<T, DP>), dim3((unsigned)key_jobs * n), dim3(256), 0, st, b);
    });
    const int z0 = a.parts > 1 ? 0 : 1, z1 = a.key_parts > 1 ? 3 : 1;
    if (z0 == z1) return;
    const int64_t most = max(z0 == 0 ? (int64_t)a.max_q * a.heads : 0, z1 == 3 ? (int64_t)a.max_k * a.kv_heads : 0) * a.head_dim / 4;
    const unsigned blocks = (unsigned)min((most + 255) / 256, (int64_t)4096);
    in_turn(blocks, 32768, [&](unsigned n) {
        hipLaunchKernelGGL(add_kernel<T>, dim3(blocks, n, (unsigned)(z1 - z0)), dim3(256), 0, st, b, z0);
    });
}

}  // namespace

extern "C" int ps_attention_backward(const ps_attention_desc* desc, const ps_attention_seqs* seqs, const void* q, const void* k,
                                     const void* v, const void* out, const float* lse, const void* out_rest, const void* dout, void* dq,
                                     void* dk, void* dv, void* workspace, size_t workspace_bytes, ps_status* status, void* hip_stream) {
    Plan p;
    if (!seqs) return PS_EINVAL;
    const int code = plan(desc, seqs, true, workspace, p);
    if (code != PS_OK) return code;
    p.a.status = status;
    if (p.a.n_seq == 0 || (p.a.n_q == 0 && p.a.n_k == 0)) return check_sequences(p.a, (hipStream_t)hip_stream);
    const ps_attention_desc* d = desc;
    if (p.a.n_q > 0 && (check_strides(d, d->q, q, d->n_q, d->heads, false) || check_strides(d, d->out, out, d->n_q, d->heads, false) || !lse ||
                        check_strides(d, d->dout, dout, d->n_q, d->heads, false) || check_strides(d, d->dq, dq, d->n_q, d->heads, true)))
        return PS_EINVAL;
    if (p.a.n_k > 0 && (check_strides(d, d->k, k, d->n_k, d->kv_heads, false) || check_strides(d, d->v, v, d->n_k, d->kv_heads, false) ||
                        check_strides(d, d->dk, dk, d->n_k, d->kv_heads, true) || check_strides(d, d->dv, dv, d->n_k, d->kv_heads, true)))
        return PS_EINVAL;
    if (((uintptr_t)out_rest & 15) != 0 || (out_rest && d->dtype != 1) || (uintptr_t)lse % 4 != 0) return PS_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < p.bytes) return PS_EWORKSPACE;
    Args& a = p.a;
    a.q = q; a.k = k; a.v = v; a.out = out; a.lse = lse; a.rest = out_rest; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
    hipStream_t st = (hipStream_t)hip_stream;
    if (a.max_q == 0 && check_sequences(a, st) != PS_OK) return PS_EHIP;   // (else the queries' launch finds them)
    (void)hipGetLastError();
    summarise_documents(a, st);
    switch (padded(desc->head_dim)) {
        case 64: desc->dtype == 1 ? launch<bf16, 64>(a, st) : launch<float, 64>(a, st); break;
        case 96: desc->dtype == 1 ? launch<bf16, 96>(a, st) : launch<float, 96>(a, st); break;
        default: desc->dtype == 1 ? launch<bf16, 128>(a, st) : launch<float, 128>(a, st);
    }
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
