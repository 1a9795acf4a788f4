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
// (LOCAL: blocks that are cut and have rows with no more than FEW keys in their windows, the first and the last ones of long windows among them.  Where a window leaves them more, its edges
// are no reason.)
// LOCAL: late and windowed(j, is), which keys are in the window, as with `cut`.  BIASED: uneven, whether the learned bias differs within the block, and
// bias(j), in powers of two, if it does; summed, whether the gradients of the scores themselves are wanted (that of x has the cap's slope too): where
// has the words of their buckets' sums, to which `run` adds them, or, of an even block, they are added to `even`.
struct Nothing {
    __device__ __forceinline__ float4 operator()(int) const { return make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void operator()(int, bool (&)[4]) const {}
};
// A lane's gradients of scores on their way to the sums of buckets, in LDS, a lane's own.  Keys come by in order, so a bucket's come one after the other, and go
// to LDS when the next one's turn has come: an addition there takes 160 cycles of a wavefront's 64 lanes (64 sequences of up to 512 tokens, every
// value added by itself: 202 us; this way 98, and 76 with the longest sequences first and blocks' sums added up four columns at a time; without the bias's gradient 51.  The two values of a
// read, an addition and a write in place of an addition: no less).
struct Run {
    int word;                          // where the bucket's sums of a wavefront's lanes (or rows) start
    float sum;
    // own: a lane has a sum of its own; else a row's two lanes share one, and come one after the other so that the order is fixed (told apart twice: the
    // compiler would make one addition of the two)
    __device__ __forceinline__ void flush(float* sums, bool own) const {
        if (own) {
            __hip_atomic_fetch_add(sums + word, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            return;
        }
        if (!(anew<256>((int)threadIdx.x) & 32)) __hip_atomic_fetch_add(sums + word, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        if (anew<256>((int)threadIdx.x) & 32) __hip_atomic_fetch_add(sums + word, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    __device__ __forceinline__ void add(float* sums, bool own, int to, float e) {
        const bool next = to != word;
        if (next) flush(sums, own);
        sum = (next ? 0.f : sum) + e;
        word = to;
    }
};
// The words of a block's distances, in LDS: a sum's in the low half, and whether the next three distances have the same.
struct Words {
    const int* at;
    __device__ __forceinline__ int first(int j) const { return at[8 * j]; }
    __device__ __forceinline__ unsigned low(int j, int i) const { return *(const unsigned short*)(at + 8 * j + i); }
};
template <typename T, int STEP, bool LOCAL, bool BIASED, typename Lse, typename Delta, typename Distance, typename Front, typename Same, typename Windowed, typename Bias,
          typename Where>
__device__ __forceinline__ void gradients(const Args& a, const f32x16& s, const f32x16& g, Weights<T>& p, Weights<T>& d, Weights<T>& rest,
                                          bool cut, bool docs, bool late, bool left_over, bool uneven, bool summed, Lse lse, Delta delta, Distance distance, Front in_front,
                                          Same same, Windowed windowed, Bias bias, Where where, float* sums, bool own, Run& run, float& even) {
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
        if (BIASED && uneven && a.cap > 0.f) {                            // (else the products have started from it)
#pragma unroll
            for (int k = 0; k < STEP; ++k) {
                const float4 off = bias(j0 + k);
                u[k] = make_float4(u[k].x - off.x, u[k].y - off.y, u[k].z - off.z, u[k].w - off.w);
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
        if (LOCAL && late) only(windowed);
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            p.set(j0 + k, u[k]);
            d.set(j0 + k, v[k]);
        }
        if constexpr (sizeof(T) == 2)
            if (left_over) {
#pragma unroll
                for (int k = 0; k < STEP; ++k) {
                    const float4 r = d.get(j0 + k);
                    rest.set(j0 + k, make_float4(v[k].x - r.x, v[k].y - r.y, v[k].z - r.z, v[k].w - r.w));
                }
            }
        if constexpr (BIASED && !std::is_same<Where, Nothing>::value)
            if (summed) {
                // (all words first: one that is read behind an addition waits for it)
                int to[STEP];
                bool wide = true;                                         // fours of the same bucket
                if (uneven) {
#pragma unroll
                    for (int k = 0; k < STEP; ++k) to[k] = where.first(j0 + k);
#pragma unroll
                    for (int k = 0; k < STEP; ++k) wide = wide && to[k] >> 16;
                    wide = __all(wide);
                }
                // (without a cap they are d.  Under one they are made of p, of pairs that have some: a hidden one's dout . v may pass all numbers)
#pragma unroll
                for (int k = 0; k < STEP; ++k) {
                    if (a.cap == 0.f) {
                        u[k] = v[k];
                        continue;
                    }
                    const float4 t = delta(j0 + k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float& e = (&u[k].x)[i];
                        e = e == 0.f ? 0.f : e * (g[4 * (j0 + k) + i] - (&t.x)[i]);
                    }
                }
                if (!uneven || wide) {
#pragma unroll
                    for (int k = 0; k < STEP; ++k) {
                        const float all = (u[k].x + u[k].y) + (u[k].z + u[k].w);
                        if (uneven)
                            run.add(sums, own, to[k] & 0xffff, all);
                        else
                            even += all;
                    }
                } else {
                    unsigned each[STEP][4];
#pragma unroll
                    for (int k = 0; k < STEP; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) each[k][i] = i == 0 ? to[k] & 0xffff : where.low(j0 + k, i);
                    reads_first();
#pragma unroll
                    for (int k = 0; k < STEP; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) run.add(sums, own, (int)each[k][i], (&u[k].x)[i]);
                }
            }
    }
}

// Tiles of 32 rows that may see some of the 32 first keys from k0 on: from `first` on, in front of the returned one.
__device__ __forceinline__ int first_keys_rows(const Args& a, const Seq& q, int k0, int& first) {
    const int n = (q.qn * a.group + 31) / 32;
    first = a.causal && k0 >= q.prefix ? (int)min((int64_t)n, max((int64_t)0, (int64_t)(k0 - q.start) * a.group / 32)) : 0;
    return n;
}

template <typename T>
__device__ __forceinline__ float by_x(const Args& a) { return a.cap > 0.f && sizeof(T) == 2 ? 4.f * a.scale : a.scale; }

// Keys fixed: dk and dv of FIXED keys of a key head, from the rows of all its heads.  Four products a tile (a fifth for the rest), and twice the
// accumulators of the queries' launch, which leaves two workgroups a unit (one in fp32 above 64 features).  Bound by waits, as forwards: 16 x 2048
// with prefix and cap, heads of 128, 978 us, 0.48 PFLOP/s, vector units issuing 31 % and matrix units busy 24 % of the time, 1.3 wavefronts a
// SIMD at barriers and waits 36 % of theirs; documents in two rows of 8192, heads of 64: 166 us, 0.44 PFLOP/s, 33 %, 22 %, 1.6 wavefronts, 40 %.
// Where the heads of a key head are no divisor of a tile's rows, addresses are worked out a row at a time, which costs some 15 % (8 causal sequences
// of 1500 to 2048, 4 key heads of 64, this launch with 2, 3, 4, 5 heads to each: 119, 182, 198, 282 us).
template <typename T, int DP, bool LOCAL, bool BIASED>
__global__ __launch_bounds__(256, DP == 64 || sizeof(T) == 2 ? 2 : 1) void key_gradients_kernel(Args a) {
    using L = Tile<T, DP, key_tile_rows(sizeof(T), DP)>;
    // Two workgroups a unit need 256 registers a lane.  In bf16 the gradients of 32 keys by 128 features take half of them, so the values
    // wait in LDS (a quarter more reads there).
    // (LOCAL: above 64 features, there is more to keep)
    constexpr bool IN_LDS = sizeof(T) == 2 && DP > (LOCAL ? 64 : 96), NEEDS_IN_LDS = sizeof(T) == 2 && DP == 128;
    __shared__ __align__(1024) unsigned char s_values[IN_LDS ? 4 : 1][IN_LDS ? 32 * L::ROWB : 16];
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][queries, dout]
    __shared__ __align__(16) float s_lse[2][64], s_delta[2][64], s_slope[2][64], s_place[2][64];   // (places from k0 on)
    __shared__ __align__(16) int s_doc[2][64];
    __shared__ __align__(16) int s_at[LOCAL ? 2 : 1][LOCAL ? 64 : 4], s_bias_at[BIASED ? 2 : 1][BIASED ? 64 : 4];   // rows' places from k0 on; their words of the bias
    extern __shared__ __align__(16) float s_bias[];                       // [buffer][a.bias_words]

    Seq q;
    Work w;
    if (!find_work<true, LOCAL>(a, q, w)) return;                                // (faulty sequences: reported by the queries' launch)
    const int hk = w.hk, s = w.s, part = w.part, k0 = w.block * FIXED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int rows = q.qn * a.group;
    int first_tile;
    const int tiles = row_tiles<LOCAL>(a, q, k0, first_tile);
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

    const float own_keyf = (float)(32 * wave + col), own_seen_from = !a.causal || key < q.prefix ? -INFINITY : own_keyf;   // places from k0 on
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
        bool some = LOCAL || !a.causal || k0 <= q.start + end || k0 < q.prefix;
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
    __shared__ Needs s_needs[NEEDS_IN_LDS ? 256 : 1];
    if (NEEDS_IN_LDS) s_needs[threadIdx.x] = needs;
    auto fetch = [&]() -> Needs { return NEEDS_IN_LDS ? s_needs[threadIdx.x] : needs; };
    // A learned bias: a lane's row's words for the keys from k0 on, if its token is the qi-th and the tile's last row's the last-th.
    auto places = [&](int buf, int qi, int head, int last) {
        if (!LOCAL) return;
        if (wave == 0) {
            s_at[buf][lane] = q.start - k0 + qi;
            s_place[buf][lane] = (float)(q.start - k0 + qi);
        }
        if (BIASED) {
            const ArgsAgain w = again();
            const int place = Learned::place(q.start + qi), far = Learned::place(q.start + last), words = buf * w->bias_words;
            if (wave == 0) s_bias_at[buf][lane] = words + (head - hk * w->group) * w->bias_width + far - place;
            Learned::send(hk, k0 - far, s_bias + words);
        }
    };
    auto request = [&](int t, bool padded, int buf) {
        const int r0 = t * L::ROWS;
        if (regular && r0 + L::ROWS <= rows && !padded) {
            const int64_t token = t * steps;
            const Needs mine = fetch();
            Sender<T, DP, L::ROWS>::whole(smem[buf][0], qbase + token * a.qs.row, mine.q);
            Sender<T, DP, L::ROWS>::whole(smem[buf][1], gbase + token * a.gs.row, mine.g);
            if (has_words) send_words(words + 64 * buf, mine.word + (int64_t)t * word_step);
            if (!LOCAL && wave == 0) s_place[buf][lane] = (float)(q.start - k0 + (int)token + (int)over_group(a, lane % L::ROWS));
            if (LOCAL) {                                                  // (a lane's row worked out again: registers)
                const int own = (anew<256>((int)threadIdx.x) & 63) % L::ROWS, of = (int)over_group(a, own);
                places(buf, (int)token + of, hk * a.group + own - of * a.group, (int)token + (L::ROWS - 1) / a.group);
            }
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
        if (!LOCAL && wave == 0) s_place[buf][lane] = (float)(q.start - k0 + qi);
        // (of 64 lanes only those of the tile's rows have words in it)
        const int of_tile = min(r0 + lane % L::ROWS, rows - 1), token = (int)over_group(a, of_tile);
        places(buf, token, hk * a.group + of_tile - token * a.group, (int)over_group(a, min(r0 + L::ROWS, rows) - 1));
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
        // whether some of the wavefront's keys are not in some rows' windows, and none in any's (64 bits: a window may end beyond 32)
        bool late = false, none = false, few = true;
        if (LOCAL) {
            const ArgsAgain w = again();
            const int64_t left = w->left, right = w->right;
            const int near = q.start + (int)over_group(a, t * L::ROWS);
            late = near + right < wlast || far - left > wk0;
            none = far + right < wk0 || near - left > wlast;
            few = few_in_window(*w, q, near, far);
        }
        const bool left_over = docs || a.cap > 0.f || ((cut || late) && few);
        t = walk.next(t + 1, t1, classify);
        vm_wait();
        __syncthreads();                                                  // the tile has landed, the one before it is no longer read
        if (t < t1) request(t, walk.is_padded(t), buf ^ 1);
        if (wk0 < q.kn && !(a.causal && wk0 > far && wk0 >= q.prefix) && !none) {
#pragma unroll 1
            for (int b = 0; b < L::BLOCKS; ++b) {                         // (one after the other: registers)
                f32x16 sc, g;
                float even = 0.f;
                Run run = {};
                auto at = [&](int j) { return 32 * b + 8 * j + 4 * half; };
                if constexpr (BIASED) {
                    f32x16 start = no_start();
                    if (a.cap == 0.f) {
                        const float* own = s_bias + 32 * wave + (anew<256>((int)threadIdx.x) & 31);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int4 of = *(const int4*)&s_bias_at[buf][at(j)];
#pragma unroll
                            for (int i = 0; i < 4; ++i) start[4 * j + i] = own[(&of.x)[i]];
                        }
                    }
                    dots<T, DP>(smem[buf][0], b, kf, sc, smem[buf][1], b, vf, g, lanes, start);
                } else {
                    dots<T, DP>(smem[buf][0], b, kf, sc, smem[buf][1], b, vf, g, lanes);
                }
                Weights<T> p, d, rest;
                gradients<T, (DP > 64 ? 1 : 4), LOCAL, BIASED>(a, sc, g, p, d, rest, cut, docs, late, left_over, true, false, [&](int j) { return *(const float4*)&s_lse[buf][at(j)]; },
                             [&](int j) { return *(const float4*)&s_delta[buf][at(j)]; },
                             [&](int j) {
                                 const float4 by = *(const float4*)&s_slope[buf][at(j)], place = *(const float4*)&s_place[buf][at(j)];
                                 const float keyf = LOCAL ? (float)(32 * wave + (anew<256>((int)threadIdx.x) & 31)) : own_keyf;
                                 return make_float4(by.x * LOG2E * fabsf(place.x - keyf), by.y * LOG2E * fabsf(place.y - keyf),
                                                    by.z * LOG2E * fabsf(place.z - keyf), by.w * LOG2E * fabsf(place.w - keyf));
                             },
                             [&](int j, bool(&is)[4]) {
                                 const float4 place = *(const float4*)&s_place[buf][at(j)];
                                 float seen_from = own_seen_from;
                                 if (LOCAL) {                             // (worked out again: registers)
                                     const int own = 32 * wave + (anew<256>((int)threadIdx.x) & 31);
                                     seen_from = k0 + own < q.prefix ? -INFINITY : (float)own;
                                 }
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = seen_from <= (&place.x)[i];
                             },
                             // (padding: rows' weights are 0 by their lse, keys' because no row is of their documents)
                             [&](int j, bool(&is)[4]) {
                                 const int4 of = *(const int4*)&s_doc[buf][at(j)];
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = (&of.x)[i] == doc;
                             },
                             [&](int j, bool(&is)[4]) {
                                 // (worked out again: few tiles are cut by a window.  Distances are 33 bits at most, a window without end 31)
                                 const int own = 32 * wave + (anew<256>((int)threadIdx.x) & 31);
                                 const int4 place = *(const int4*)&s_at[buf][at(j)];
#pragma unroll
                                 for (int i = 0; i < 4; ++i) {
                                     const int off = (&place.x)[i] - own;   // (a row's place less the key's)
                                     is[i] = off <= a.left && off >= -a.right;
                                 }
                             },
                             [&](int j) {
                                 const int4 of = *(const int4*)&s_bias_at[buf][at(j)];
                                 const float* own = s_bias + 32 * wave + (anew<256>((int)threadIdx.x) & 31);
                                 return make_float4(own[of.x], own[of.y], own[of.z], own[of.w]);
                             },
                             Nothing(), nullptr, true, run, even);
                weigh<T, DP>(smem[buf][1], b, p, dv, lanes);
                weigh<T, DP>(smem[buf][0], b, d, dk, lanes);
                if (sizeof(T) == 2 && left_over) weigh<T, DP>(smem[buf][0], b, rest, dk, lanes);
            }
        }
        buf ^= 1;
    }
    __syncthreads();                                                      // (tiles are no longer read)
    if (wk0 >= q.kn) return;
    unsigned char* const mine = smem[0][0] + wave * PUT_BYTES;
    static_assert(sizeof(smem) >= 4 * PUT_BYTES, "rows on their way out");
    const int own = wk0 + (anew<256>((int)threadIdx.x) & 31);              // (the key, worked out again)
    const bool is = own < q.kn && !(LOCAL && own < again()->sinks);              // (the first keys' gradients have a launch of their own)
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
template <typename T, int DP, bool LOCAL, bool BIASED>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP > 64 ? 1 : 2) void query_gradients_kernel(Args a) {
    using L = Tile<T, DP, query_tile_rows(sizeof(T), DP, BIASED)>;
    // BIASED: [buffer][a.bias_words], then, if its gradient is wanted, [buffer][bias_width, in whole wavefronts] words of buckets' sums, and
    // [wavefront][buckets, and one for distances without][lane, or row] sums
    extern __shared__ __align__(16) float s_bias[];
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][keys, values]
    __shared__ __align__(16) int s_doc[2][64];

    Seq q;
    Work w;
    if (!find_work<false, LOCAL>(a, q, w)) return;
    const int hk = w.hk, s = w.s, part = w.part, rows = q.qn * a.group, r0 = w.block * FIXED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const Span span = key_tiles<LOCAL>(a, q, r0);
    const int tiles = span.tiles;
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
    const int end = seen_to<LOCAL>(a, q, place);
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
        const int k0 = span.at<LOCAL>(t) * L::ROWS;
        bool some = LOCAL || !a.causal || k0 <= far || k0 < q.prefix;
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
    const int wend = LOCAL ? seen_to<LOCAL>(a, q, wnear) : 0, wbegin = LOCAL ? window_begin(a, wfar) : 0;   // the first to end, the last to begin
    const int wend_far = LOCAL ? seen_to<LOCAL>(a, q, wfar) : 0, wbegin_near = LOCAL ? window_begin(a, wnear) : 0;
    // keys that some of the workgroup's rows have nearer than `reach`
    const int wide_from = BIASED ? Learned::place(q.start + (int)over_group(a, r0)) - a.reach + 1 : 0, wide_to = BIASED ? (int)min((int64_t)far + a.reach, (int64_t)INT32_MAX) : 0;
    const int bias_place = Learned::place(far), bias_from = BIASED ? (head - hk * a.group) * a.bias_width + bias_place - Learned::place(place) : 0;
    const int widths = (a.bias_width + 63) & ~63, columns = a.sum_columns, sums_a_wave = (a.n_buckets + 1) * columns;
    int* const s_bucket = (int*)(s_bias + 2 * a.bias_words);
    float* const s_sums = (float*)(s_bucket + 2 * widths);
    const bool summed = BIASED && a.bias_parts != nullptr;
    // What is further than `reach` in front of the row, or behind it, has one bias: a lane's own two, in LDS, as is what few tiles ask for (registers).
    enum Own { FRONT, BEHIND, SLOPE, DOC, END, OWN };
    __shared__ float s_own[BIASED ? OWN : 1][BIASED ? 256 : 1];
    auto kept = [&](Own which) { return s_own[which][anew<256>((int)threadIdx.x)]; };
    if (BIASED) {
        const float* const ends = a.table + (int64_t)head * (2 * a.reach + 1);
        const float in_powers = a.cap > 0.f ? 1.f : a.scale * LOG2E;
        s_own[FRONT][threadIdx.x] = ends[0] * in_powers;
        s_own[BEHIND][threadIdx.x] = ends[2 * a.reach] * in_powers;
        s_own[SLOPE][threadIdx.x] = slope;
        s_own[DOC][threadIdx.x] = __int_as_float(doc);
        s_own[END][threadIdx.x] = __int_as_float(end);
    }
    const int wnear_place = Learned::place(wnear), wfar_place = (int)min((int64_t)wfar, (int64_t)INT32_MAX - a.reach);   // (a key is below 2^30)
    if (summed)
        for (int i = threadIdx.x; i < sums_a_wave; i += 256) ((float4*)s_sums)[i] = make_float4(0.f, 0.f, 0.f, 0.f);   // (the first tile's barrier is behind this)
    auto request = [&](int t, bool padded, int buf) {
        const int k0 = span.at<LOCAL>(t) * L::ROWS;
        if (k0 + L::ROWS <= q.kn && !padded && regular) {
            keys.whole(smem[buf][0], kbase + k0 * a.ks.row);
            values.whole(smem[buf][1], vbase + k0 * a.vs.row);
        } else {
            const uint64_t there = keys_there(a, q, k0, padded);
            keys.rows(smem[buf][0], a.head_dim, there, [&](int i) { return kbase + (k0 + i) * a.ks.row; });
            values.rows(smem[buf][1], a.head_dim, there, [&](int i) { return vbase + (k0 + i) * a.vs.row; });
        }
        if (a.k_docs && wave == 0) send_words(s_doc[buf], a.k_docs + q.k0 + min(k0 + lane, q.kn - 1));
        if (BIASED && scalar(k0 + L::ROWS > wide_from && k0 < wide_to)) {
            Learned::send(hk, k0 - bias_place, s_bias + buf * a.bias_words);
            if (summed) Learned::send_buckets(k0 - bias_place, s_bucket + buf * widths);
        }
    };

    f32x16 dq[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[i][e] = 0.f;

    Run run = {a.n_buckets * columns, 0.f};
    Walk walk;
    int t = walk.next(t0, t1, classify), buf = 0;
    if (t < t1) request(t, walk.is_padded(t), 0);
    while (t < t1) {
        const bool docs = !walk.is_one(t);
        const int k0 = span.at<LOCAL>(t) * L::ROWS;
        const bool cut = LOCAL ? k0 + L::ROWS > wend : k0 + L::ROWS > q.kn || (a.causal && k0 + L::ROWS - 1 > wnear && k0 + L::ROWS > q.prefix);
        const bool late = LOCAL && k0 < wbegin && k0 + L::ROWS > a.sinks;
        const bool left_over = docs || a.cap > 0.f || ((cut || late) && (!LOCAL || few_in_window(a, q, wnear, wfar)));
        const bool none = LOCAL ? k0 >= wend_far || (k0 + L::ROWS <= wbegin_near && k0 >= a.sinks) : a.causal && k0 > wfar && k0 >= q.prefix;
        const float from = (float)(place - k0 - 4 * half);
        t = walk.next(t + 1, t1, classify);
        vm_wait();
        __syncthreads();                                                  // the tile has landed, the one before it is no longer read
        if (t < t1) request(t, walk.is_padded(t), buf ^ 1);
        if (wr0 < rows && !none) {
#pragma unroll 1
            for (int b = 0; b < L::BLOCKS; ++b) {                         // (one after the other: registers)
                f32x16 sc, g;
                // a block whose distances all are `reach` and more on one side has one bias, which goes with lse
                const int kb = k0 + 32 * b;
                const bool front = BIASED && kb + 31 <= wnear_place - a.reach, uneven = BIASED && !front && kb < wfar_place + a.reach;
                if constexpr (BIASED)
                    dots<T, DP>(smem[buf][0], b, qf, sc, smem[buf][1], b, gf, g, lanes,
                                Learned::start(uneven && a.cap == 0.f, half, [&](int i) { return s_bias[buf * a.bias_words + bias_from + 32 * b + i]; }));
                else
                    dots<T, DP>(smem[buf][0], b, qf, sc, smem[buf][1], b, gf, g, lanes);
                Weights<T> p, d, rest;
                auto at = [&](int j) { return 32 * b + 8 * j + 4 * half; };
                const int own_left = BIASED ? 0 : end - k0 - 32 * b - 4 * half;
                const float own_off = from - (float)(32 * b);
                // keys behind the first ones that are in front of the window (late tiles alone: the places are near enough to the window's length)
                const unsigned hidden = LOCAL ? max((int)((unsigned)place - (unsigned)a.left - (unsigned)a.sinks), 0) : 0;
                const float mine = BIASED && !uneven ? lse - kept(front ? FRONT : BEHIND) : lse;
                float even = 0.f;
                gradients<T, (BIASED && DP > 96 ? 1 : 4), LOCAL, BIASED>(a, sc, g, p, d, rest, cut, docs, late, left_over, uneven, summed, [&](int) { return make_float4(mine, mine, mine, mine); },
                             [&](int) { return make_float4(delta, delta, delta, delta); },
                             [&](int j) {
                                 const float off = BIASED ? (float)(place - kb - 4 * half) : own_off, by = BIASED ? kept(SLOPE) : slope;
                                 return make_float4(by * fabsf(off - (float)(8 * j)), by * fabsf(off - (float)(8 * j + 1)),
                                                    by * fabsf(off - (float)(8 * j + 2)), by * fabsf(off - (float)(8 * j + 3)));
                             },
                             [&](int j, bool(&is)[4]) {
                                 const int left = BIASED ? __float_as_int(kept(END)) - kb - 4 * half : own_left;
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = left > 8 * j + i;
                             },
                             // (padding is zeros on both sides, and its weights are 0 by its lse)
                             [&](int j, bool(&is)[4]) {
                                 const int4 of = *(const int4*)&s_doc[buf][at(j)];
                                 const int own = BIASED ? __float_as_int(kept(DOC)) : doc;
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = (&of.x)[i] == own;
                             },
                             [&](int j, bool(&is)[4]) {
#pragma unroll
                                 for (int i = 0; i < 4; ++i) is[i] = (unsigned)(k0 + at(j) + i - a.sinks) >= hidden;
                             },
                             [&](int j) {
                                 const float* own = s_bias + buf * a.bias_words + bias_from + at(j);
                                 return make_float4(own[0], own[1], own[2], own[3]);
                             },
                             Words{s_bucket + buf * widths + bias_place - Learned::place(place) + at(0)},
                             s_sums + wave * sums_a_wave + (anew<256>((int)threadIdx.x) & (columns - 1)), columns == 64, run, even);
                if (summed && !uneven)
                    run.add(s_sums + wave * sums_a_wave + (anew<256>((int)threadIdx.x) & (columns - 1)), columns == 64, a.bucket_words[front ? 0 : 2 * a.reach] & 0xffff, even);
                weigh<T, DP>(smem[buf][0], b, d, dq, lanes);
                if (sizeof(T) == 2 && left_over) weigh<T, DP>(smem[buf][0], b, rest, dq, lanes);
            }
        }
        buf ^= 1;
    }
    __syncthreads();                                                      // (tiles are no longer read, and the sums are there)
    if (summed) {
        run.flush(s_sums + wave * sums_a_wave + (lane & (columns - 1)), columns == 64);
        __syncthreads();
        // A bucket's sums of a head's lanes added up by `slices` neighbouring threads, a share of the rows each, which start at other rows from bucket to
        // bucket (all buckets have a row's sums in one bank).  Row r0 + x has head x % group less r0's.
        float* const to = a.bias_parts + ((int64_t)part * a.bias_blocks + (int64_t)q.q0 * a.group / FIXED + s + w.block) * a.n_buckets * a.heads;
        if ((a.group & (a.group - 1)) == 0) {
            // (heads that share keys by ones, twos, fours ..: a row's head goes by its column.  Eight neighbouring threads have a bucket, four columns of all
            // wavefronts each)
            const int c = threadIdx.x & 7;
            for (int b = threadIdx.x >> 3; b < a.n_buckets; b += 32) {
                float4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = i < 4 || columns == 64 ? *(const float4*)(s_sums + (i & 3) * sums_a_wave + b * columns + 32 * (i >> 2) + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int n = 4; n > 0; n /= 2)
#pragma unroll
                    for (int i = 0; i < n; ++i) v[i] = make_float4(v[i].x + v[i + n].x, v[i].y + v[i + n].y, v[i].z + v[i + n].z, v[i].w + v[i + n].w);
                float4 sum = v[0];
                for (int o = 4; 4 * o >= a.group && o > 0; o /= 2)
                    sum = make_float4(sum.x + __shfl_xor(sum.x, o, 64), sum.y + __shfl_xor(sum.y, o, 64), sum.z + __shfl_xor(sum.z, o, 64), sum.w + __shfl_xor(sum.w, o, 64));
                if (a.group <= 2) sum = make_float4(sum.x + sum.z, sum.y + sum.w, 0.f, 0.f);
                if (a.group == 1) sum.x += sum.y;
                float* const mine = to + b * a.heads + hk * a.group + 4 * c;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (4 * c + i < a.group) mine[i] = (&sum.x)[i];
            }
        } else {
            const int outs = a.n_buckets * a.group, most = min(256 / outs, 32), slices = most < 1 ? 1 : 1 << (31 - __builtin_clz(most)), slice = threadIdx.x & (slices - 1);
            for (int first = 0; first < outs; first += 256 / slices) {
                const int i = first + (int)threadIdx.x / slices, b = i / a.group, h = i - b * a.group;
                const int x0 = (h + a.group - r0 % a.group) % a.group, n = (FIXED - x0 + a.group - 1) / a.group, turns = (FIXED / a.group + slices) / slices;
                float sum = 0.f;
                if (i < outs)
                    for (int k = 0; k < turns; ++k) {
                        const int m = slice + slices * ((k + i) % turns), x = x0 + m * a.group;
                        if (m >= n) continue;
                        const float* of = s_sums + (x >> 5) * sums_a_wave + b * columns + (x & 31);
                        sum += columns == 64 ? of[0] + of[32] : of[0];
                    }
                for (int o = 1; o < slices; o *= 2) sum += __shfl_xor(sum, o, 64);
                if (i < outs && slice == 0) to[b * a.heads + hk * a.group + h] = sum;
            }
        }
    }
    if (wr0 >= rows) return;
    unsigned char* const mine = smem[0][0] + wave * PUT_BYTES;
    static_assert(sizeof(smem) >= 4 * PUT_BYTES, "rows on their way out");
    int64_t to_token = token;
    int to_head = head;
    if (BIASED) {                                                         // (worked out again: registers)
        const int own = min(wr0 + (anew<256>((int)threadIdx.x) & 31), rows - 1), of = (int)over_group(a, own);
        to_token = q.q0 + of;
        to_head = hk * a.group + own - of * a.group;
    }
    if (a.parts > 1)
        put_rows<float, DP>(mine, dq, 1.f, a.head_dim,
                            live ? a.part_o + (((int64_t)part * a.n_q + to_token) * a.heads + to_head) * a.head_dim : nullptr);
    else
        put_rows<T, DP>(mine, dq, by_x<T>(a), a.head_dim, live ? (T*)a.dq + to_token * a.dqs.row + to_head * a.dqs.head : nullptr);
}

// The first keys, which rows see wherever they stand: dk and dv of 32 of them and of a share of the rows that may see them, whose tiles the workgroup's wavefronts
// take in turn, each with tiles of its own on their way through LDS; what they have is put together at the end.
// (Rows that have few keys in their windows, see gradients().)
template <typename T, int DP, bool BIASED>
__global__ __launch_bounds__(256, 1) void first_keys_kernel(Args a) {
    using F = Few<T, DP>;
    using L = typename F::L;
    constexpr int STAGES = F::STAGES;
    enum Word { LSE, DELTA, SLOPE, FRONT, DOC, PLACE, TABLE, WORDS };
    __shared__ __align__(1024) unsigned char smem[4][STAGES][2][L::BYTES];   // [wavefront][stage][queries, dout]; at the end the wavefronts' sums
    __shared__ __align__(16) float s_word[4][STAGES][WORDS][64];          // what rows bring along; PLACE and TABLE are integers
    static_assert(sizeof(smem) >= 4 * 2 * 32 * DP * sizeof(float), "the wavefronts' sums");

    unsigned id = blockIdx.x;
    const int hk = id % a.kv_heads;
    id /= a.kv_heads;
    const int part = id % a.sink_parts;
    id /= a.sink_parts;
    const int k0 = (int)(id % a.sink_blocks) * 32, s = a.seq0 + (int)(id / a.sink_blocks);
    Seq q;
    if (!sequence(a, s, q) || k0 >= min(q.kn, a.sinks)) return;           // (faulty sequences: reported by the queries' launch)
    const int rows = q.qn * a.group;
    int first;
    const int tiles = first_keys_rows(a, q, k0, first), t0 = first + part * a.sink_part_tiles, t1 = min(tiles, t0 + a.sink_part_tiles);
    if (part > 0 && t0 >= tiles) return;                                  // (part 0 writes, rows or not)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;

    const int key = k0 + col, keys = min(q.kn, a.sinks);
    const int64_t token = q.k0 + min(key, q.kn - 1);
    const int doc = a.k_docs ? a.k_docs[token] : 0;
    const bool there = key < q.kn && doc >= 0;
    const Lanes<T, DP> lanes(lane);
    Fixed<T, DP> kf, vf;
    kf.load((const T*)a.k + token * a.ks.row + hk * a.ks.head, there, a.head_dim, half);
    vf.load((const T*)a.v + token * a.vs.row + hk * a.vs.head, there, a.head_dim, half);

    auto request = [&](int t, int stage) {
        const int r0 = t * 32, r = min(r0 + col, rows - 1), qi = (int)over_group(a, r), head = hk * a.group + r - qi * a.group;
        const int64_t row = q.q0 + qi;
        const bool is = r0 + col < rows && (!a.q_docs || a.q_docs[row] >= 0);   // (padding and rows past the end are zeros that see nothing)
        const uint64_t live = __ballot(is);
        auto from = [&](const void* base, const ps_strides& st, int i) -> const T* {
            const int x = min(r0 + i, rows - 1), token = (int)over_group(a, x);
            return (const T*)base + (q.q0 + token) * st.row + (hk * a.group + x - token * a.group) * st.head;
        };
        F::rows(smem[wave][stage][0], a.head_dim, live, [&](int i) { return from(a.q, a.qs, i); });
        F::rows(smem[wave][stage][1], a.head_dim, live, [&](int i) { return from(a.dout, a.gs, i); });
        float(*const to)[64] = s_word[wave][stage];
        const int64_t at = head * a.n_q + row;
        send_words(to[LSE], is ? (const void*)(a.row_lse + at) : (const void*)&infinity_word);
        send_words(to[DELTA], is ? (const void*)(a.row_delta + at) : (const void*)&zeros);
        if (a.slopes) send_words(to[SLOPE], a.slopes + head);
        if (a.q_docs) send_words(to[DOC], is ? (const void*)(a.q_docs + row) : (const void*)&minus_one);
        if (BIASED) send_words(to[FRONT], a.table + (int64_t)head * (2 * a.reach + 1));
        to[PLACE][lane] = __int_as_float(q.start + qi);
        if (BIASED) to[TABLE][lane] = __int_as_float(head * (2 * a.reach + 1) + a.reach);
    };

    f32x16 dk[L::NA], dv[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[i][e] = dv[i][e] = 0.f;
    const float in_powers = a.cap > 0.f ? 1.f : a.scale * LOG2E;
    int sent = t0 + wave, stage = 0, next_stage = 0;
    auto send_next = [&] {
        request(sent, next_stage);
        next_stage = next_stage + 1 < STAGES ? next_stage + 1 : 0;
        sent += 4;
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (sent < t1) send_next();
    for (int t = t0 + wave; t < t1; t += 4) {
        // (with two stages the next tile is sent for behind this one, which has landed by then)
        vm_wait();
        if (sent < t1) send_next();
        if (STAGES == 1) vm_wait();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const unsigned char *queries = smem[wave][stage][0], *douts = smem[wave][stage][1];
        const float(*const word)[64] = s_word[wave][stage];
        auto at = [&](int j) { return 8 * j + 4 * half; };
        const int near = q.start + (int)over_group(a, t * 32);
        const bool cut = a.causal && k0 + 31 > near && k0 + 31 >= q.prefix;
        const bool left_over = a.q_docs || a.cap > 0.f || cut || few_in_window(a, q, near, q.start + (int)over_group(a, min(t * 32 + 31, rows - 1)));
        const bool uneven = BIASED && (int64_t)near - a.reach < k0 + 31;  // (else all stand `reach` and more behind the keys)
        auto bias = [&](int j) {
            const int4 place = *(const int4*)&word[PLACE][at(j)], of = *(const int4*)&word[TABLE][at(j)];
            float4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) (&v.x)[i] = a.table[(&of.x)[i] + max(-a.reach, min(key - Learned::place((&place.x)[i]), a.reach))];
            return v;
        };
        f32x16 sc, g;
        f32x16 start = no_start();
        if (BIASED && uneven && a.cap == 0.f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 v = bias(j);
#pragma unroll
                for (int i = 0; i < 4; ++i) start[4 * j + i] = (&v.x)[i];
            }
        }
        dots<T, DP>(queries, 0, kf, sc, douts, 0, vf, g, lanes, start);
        Weights<T> p, d, rest;
        Run run = {};
        float even = 0.f;
        gradients<T, 4, true, BIASED>(a, sc, g, p, d, rest, cut, a.q_docs != nullptr, false, left_over, uneven, false,
                     [&](int j) {
                         float4 v = *(const float4*)&word[LSE][at(j)];
                         if (BIASED && !uneven) {
                             const float4 off = *(const float4*)&word[FRONT][at(j)];
                             v = make_float4(fmaf(-off.x, in_powers, v.x), fmaf(-off.y, in_powers, v.y), fmaf(-off.z, in_powers, v.z), fmaf(-off.w, in_powers, v.w));
                         }
                         return v;
                     },
                     [&](int j) { return *(const float4*)&word[DELTA][at(j)]; },
                     [&](int j) {
                         const float4 by = *(const float4*)&word[SLOPE][at(j)];
                         const int4 place = *(const int4*)&word[PLACE][at(j)];
                         return make_float4(by.x * LOG2E * fabsf((float)place.x - (float)key), by.y * LOG2E * fabsf((float)place.y - (float)key),
                                            by.z * LOG2E * fabsf((float)place.z - (float)key), by.w * LOG2E * fabsf((float)place.w - (float)key));
                     },
                     [&](int j, bool(&is)[4]) {
                         const int4 place = *(const int4*)&word[PLACE][at(j)];
#pragma unroll
                         for (int i = 0; i < 4; ++i) is[i] = key <= (&place.x)[i] || key < q.prefix;
                     },
                     [&](int j, bool(&is)[4]) {
                         const int4 of = *(const int4*)&word[DOC][at(j)];
#pragma unroll
                         for (int i = 0; i < 4; ++i) is[i] = (&of.x)[i] == doc;
                     },
                     Nothing(), bias, Nothing(), nullptr, true, run, even);
        weigh<T, DP>(douts, 0, p, dv, lanes);
        weigh<T, DP>(queries, 0, d, dk, lanes);
        if (sizeof(T) == 2 && left_over) weigh<T, DP>(queries, 0, rest, dk, lanes);
        asm volatile("" ::: "memory");
        stage = stage + 1 < STAGES ? stage + 1 : 0;
    }

    __syncthreads();
    float* const sums = (float*)smem;                                     // [wavefront][dk, dv][key][DP]
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int f = 32 * i + 8 * g + 4 * half;
            *(float4*)(sums + ((wave * 2 + 0) * 32 + col) * DP + f) = make_float4(dk[i][4 * g], dk[i][4 * g + 1], dk[i][4 * g + 2], dk[i][4 * g + 3]);
            *(float4*)(sums + ((wave * 2 + 1) * 32 + col) * DP + f) = make_float4(dv[i][4 * g], dv[i][4 * g + 1], dv[i][4 * g + 2], dv[i][4 * g + 3]);
        }
    __syncthreads();
    const int fours = a.head_dim / 4;
    for (int i = threadIdx.x; i < 2 * 32 * fours; i += 256) {
        const int z = i / (32 * fours), r = i / fours - z * 32, f = i % fours * 4;
        if (k0 + r >= keys) continue;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float4 x = *(const float4*)(sums + ((w * 2 + z) * 32 + r) * DP + f);
            v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
        }
        if (a.sink_parts > 1) {
            *(float4*)((z == 0 ? a.sink_dk : a.sink_dv) + ((((int64_t)part * a.n_seq + s) * a.sink_blocks * 32 + k0 + r) * a.kv_heads + hk) * a.head_dim + f) = v;
            continue;
        }
        const ps_strides to = z == 0 ? a.dks : a.dvs;
        const float by = z == 0 ? by_x<T>(a) : 1.f;
        T* const out = (T*)(z == 0 ? a.dk : a.dv) + (int64_t)(q.k0 + k0 + r) * to.row + hk * to.head + f;
        if constexpr (sizeof(T) == 2)
            *(uint2*)out = make_uint2(cvt_pk_bf16(v.x * by, v.y * by), cvt_pk_bf16(v.z * by, v.w * by));
        else
            *(float4*)out = make_float4(v.x * by, v.y * by, v.z * by, v.w * by);
    }
}

// A gradient's shares added up, a thread four neighbours: those of queries (z = 0), keys (1) and values (2).  3365 tokens, 8 heads of 80 on 4,
// up to 4 shares: 61 MB in 18 us.
template <typename T, bool LOCAL>
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
        if (LOCAL && z > 0 && mine < a.sinks) continue;                   // (added up apart)
        int first = 0;
        const int tiles = z == 0 ? key_tiles<LOCAL>(a, q, (mine * a.group + head % a.group) / FIXED * FIXED).tiles : row_tiles<LOCAL>(a, q, mine / FIXED * FIXED, first);
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

// The same of the first keys' gradients, dk (z = 0) and dv (1), whose shares are many and values few: 16 threads to four neighbours, every sixteenth share
// each (16384 rows in 256 shares 26 -> 5.5 us).
template <typename T>
__global__ __launch_bounds__(256) void add_sinks_kernel(Args a) {
    __shared__ float4 s_sum[16][16];
    const int z = blockIdx.z, s = a.seq0 + (int)blockIdx.y, lane = threadIdx.x & 15, turn = threadIdx.x >> 4;
    Seq q;
    if (!sequence(a, s, q)) return;
    const int fours = a.head_dim / 4, a_key = a.kv_heads * fours, keys = a.sink_blocks * 32;
    const int64_t n = (int64_t)min(q.kn, a.sinks) * a_key, step = (int64_t)a.n_seq * keys * a_key;
    const float4* part = (const float4*)(z == 0 ? a.sink_dk : a.sink_dv) + (int64_t)s * keys * a_key;
    const ps_strides to = z == 0 ? a.dks : a.dvs;
    T* out = (T*)(z == 0 ? a.dk : a.dv);
    const float by = z == 1 ? 1.f : by_x<T>(a);
    for (int64_t i0 = (int64_t)blockIdx.x * 16; i0 < n; i0 += (int64_t)gridDim.x * 16) {
        const int64_t i = i0 + lane;
        const int key = (int)(i / a_key), in_key = (int)(i - (int64_t)key * a_key), head = in_key / fours;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n) {
            int first;
            const int tiles = first_keys_rows(a, q, key / 32 * 32, first), parts = shares(tiles - first, a.sink_parts, a.sink_part_tiles);
#pragma unroll 4
            for (int p = turn; p < parts; p += 16) {
                const float4 v = part[p * step + i];
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
        }
        s_sum[turn][lane] = sum;
        __syncthreads();
        if (turn == 0 && i < n) {
#pragma unroll
            for (int t = 1; t < 16; ++t) {
                const float4 v = s_sum[t][lane];
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            T* at = out + (int64_t)(q.k0 + key) * to.row + head * to.head + (in_key - head * fours) * 4;
            if constexpr (sizeof(T) == 2)
                *(uint2*)at = make_uint2(cvt_pk_bf16(sum.x * by, sum.y * by), cvt_pk_bf16(sum.z * by, sum.w * by));
            else
                *(float4*)at = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
        }
        __syncthreads();
    }
}

// A learned bias's gradient from the sums of blocks of rows (zeros for blocks that there are not): 64 values a workgroup, `each` blocks, the sixteen
// wavefronts taking turns; then, where those are not all, what they made of it in the same way.
__global__ __launch_bounds__(1024) void add_bias_kernel(const float* from, int64_t blocks, int64_t each, int n, float* to) {
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
    const int64_t b0 = blockIdx.y * each, b1 = min(blocks, b0 + each);
    float sum = 0.f;
    if (i < n) {
#pragma unroll 8
        for (int64_t b = b0 + wave; b < b1; b += 16) sum += from[b * n + i];
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || i >= n) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += s_sum[w][lane];
    to[(int64_t)blockIdx.y * n + i] = sum;
}
void add_bias(const Args& a, float* dbias, hipStream_t st) {
    const int n = a.n_buckets * a.heads;
    const int64_t blocks = a.parts * a.bias_blocks, each = blocks > 256 ? 128 + blocks / 32768 : 256, chunks = (blocks + each - 1) / each;
    const unsigned across = (unsigned)((n + 63) / 64);
    float* const between = chunks > 1 ? a.bias_parts + blocks * n : dbias;
    hipLaunchKernelGGL(add_bias_kernel, dim3(across, (unsigned)(chunks > 1 ? chunks : 1)), dim3(1024), 0, st, a.bias_parts, blocks, each, n, between);
    if (chunks > 1) hipLaunchKernelGGL(add_bias_kernel, dim3(across), dim3(1024), 0, st, between, chunks, chunks, n, dbias);
}

template <typename T, int DP, bool LOCAL, bool BIASED>
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
    const unsigned tile_lds = BIASED ? 2 * a.bias_words * sizeof(float) : 0;
    // (up to 52 KB, with the tiles 113: a launch gets 160 without a word)
    const unsigned sums_lds = a.bias_parts ? (2 * ((a.bias_width + 63) & ~63) + 4 * (a.n_buckets + 1) * a.sum_columns) * sizeof(float) : 0;
    in_turn(row_jobs, a.n_seq, [&](unsigned n) {
        b.listed = add_up(a, n, a.row_blocks, a.parts);
        hipLaunchKernelGGL((query_gradients_kernel<T, DP, LOCAL, BIASED>), dim3((unsigned)row_jobs * n), dim3(256), tile_lds + sums_lds, st, b);
    });
    in_turn(key_jobs, a.n_seq, [&](unsigned n) {
        b.listed = add_up(a, n, key_blocks, a.key_parts);
        if (BIASED) set_width(b, FIXED + (a.key_tile - 1) / a.group + 2);
        hipLaunchKernelGGL((key_gradients_kernel<T, DP, LOCAL, BIASED>), dim3((unsigned)key_jobs * n), dim3(256), BIASED ? 2 * b.bias_words * sizeof(float) : 0, st, b);
    });
    if constexpr (LOCAL) {
        if (a.sink_blocks > 0) {
            const int64_t jobs = (int64_t)a.kv_heads * a.sink_blocks * a.sink_parts;
            in_turn(jobs, a.n_seq, [&](unsigned n) {
                hipLaunchKernelGGL((first_keys_kernel<T, DP, BIASED>), dim3((unsigned)jobs * n), dim3(256), 0, st, b);
            });
        }
        if (a.sink_parts > 1) {
            const unsigned blocks = (unsigned)min(((int64_t)a.sinks * a.kv_heads * a.head_dim / 4 + 15) / 16, (int64_t)4096);
            in_turn(blocks, 32768, [&](unsigned n) { hipLaunchKernelGGL(add_sinks_kernel<T>, dim3(blocks, n, 2), dim3(256), 0, st, b); });
        }
    }
    const int z0 = a.parts > 1 ? 0 : 1, z1 = a.key_parts > 1 ? 3 : 1;
    if (z0 == z1) return;
    const int64_t most = max(z0 == 0 ? (int64_t)a.max_q * a.heads : 0, z1 == 3 ? (int64_t)a.max_k * a.kv_heads : 0) * a.head_dim / 4;
    const unsigned blocks = (unsigned)min((most + 255) / 256, (int64_t)4096);
    in_turn(blocks, 32768, [&](unsigned n) {
        hipLaunchKernelGGL((add_kernel<T, LOCAL>), dim3(blocks, n, (unsigned)(z1 - z0)), dim3(256), 0, st, b, z0);
    });
}

}  // namespace

namespace {

template <bool LOCAL>
int backward(const ps_attention_desc* desc, const ps_attention_seqs* seqs, const ps_attention_local* local, const void* q, const void* k, const void* v,
             const void* out, const float* lse, const void* out_rest, const void* dout, void* dq, void* dk, void* dv, float* dbias, void* workspace,
             size_t workspace_bytes, ps_status* status, void* hip_stream) {
    Plan p;
    if (!seqs || (LOCAL && !local)) return PS_EINVAL;
    const int code = plan(desc, seqs, local, true, workspace, p, sees_ahead(desc, seqs));
    if (code != PS_OK) return code;
    p.a.status = status;
    if (dbias && (p.a.n_buckets == 0 || (uintptr_t)dbias % 4 != 0)) return PS_EINVAL;
    if (!dbias) p.a.bias_parts = nullptr;
    if (p.a.n_seq == 0 || (p.a.n_q == 0 && p.a.n_k == 0)) {
        if (dbias) {                       // (a sum over no blocks)
            (void)hipGetLastError();
            p.a.bias_blocks = 0;
            add_bias(p.a, dbias, (hipStream_t)hip_stream);
            if (hipGetLastError() != hipSuccess) return PS_EHIP;
        }
        return check_sequences(p.a, (hipStream_t)hip_stream);
    }
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
    if (LOCAL) make_table(a, local, a.slope_by, st);                           // (and clears the sums of blocks)
    auto of_type = [&](auto biased) {
        constexpr bool B = decltype(biased)::value;
        switch (padded(desc->head_dim)) {
            case 64: desc->dtype == 1 ? launch<bf16, 64, LOCAL, B>(a, st) : launch<float, 64, LOCAL, B>(a, st); break;
            case 96: desc->dtype == 1 ? launch<bf16, 96, LOCAL, B>(a, st) : launch<float, 96, LOCAL, B>(a, st); break;
            default: desc->dtype == 1 ? launch<bf16, 128, LOCAL, B>(a, st) : launch<float, 128, LOCAL, B>(a, st);
        }
    };
    if constexpr (LOCAL) {
        if (a.table) {
            of_type(std::true_type());
            if (dbias) add_bias(a, dbias, st);
            return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
        }
    }
    of_type(std::false_type());
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

}  // namespace

extern "C" int ps_attention_backward(const ps_attention_desc* desc, const ps_attention_seqs* seqs, const void* q, const void* k,
                                     const void* v, const void* out, const float* lse, const void* out_rest, const void* dout, void* dq,
                                     void* dk, void* dv, void* workspace, size_t workspace_bytes, ps_status* status, void* hip_stream) {
    return backward<false>(desc, seqs, nullptr, q, k, v, out, lse, out_rest, dout, dq, dk, dv, nullptr, workspace, workspace_bytes, status, hip_stream);
}

extern "C" int ps_local_attention_backward(const ps_attention_desc* desc, const ps_attention_seqs* seqs, const ps_attention_local* local, const void* q,
                                           const void* k, const void* v, const void* out, const float* lse, const void* out_rest, const void* dout,
                                           void* dq, void* dk, void* dv, float* dbias, void* workspace, size_t workspace_bytes, ps_status* status,
                                           void* hip_stream) {
    return backward<true>(desc, seqs, local, q, k, v, out, lse, out_rest, dout, dq, dk, dv, dbias, workspace, workspace_bytes, status, hip_stream);
}
