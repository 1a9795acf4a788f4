// Gradients of the attention of seq_attention_fwd.hip, in three launches: what a row brings along (its lse and dout . out), the
// gradients of keys and values (keys fixed, queries passing), that of the queries (queries fixed, keys passing).  Scores are computed
// again in both of the latter; every gradient is then a sum in one wavefront's registers, in an order that the shapes fix, and
// nothing is added up in memory.
#include "seq_attention.h"

using namespace seqatt;
typedef __bf16 bf16;

namespace {

// stats[head][token]: 16 lanes a row, 8 elements a lane.
template <typename T>
__global__ __launch_bounds__(256) void stats_kernel(Args a) {
    const int e = (threadIdx.x & 15) * 8;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < a.n_q * a.heads; first += (int64_t)gridDim.x * 16) {
        const int64_t row = first + (threadIdx.x >> 4);
        const bool live = row < a.n_q * a.heads;
        const int64_t token = live ? row / a.heads : 0;
        const int head = live ? (int)(row - token * a.heads) : 0;
        float sum = 0.f;
        if (live && e < a.head_dim) {
            const T *o = (const T*)a.out + token * a.os.row + head * a.os.head + e, *g = (const T*)a.dout + token * a.gs.row + head * a.gs.head + e;
            T x[8], y[8];
#pragma unroll
            for (int i = 0; i < (int)sizeof(x) / 16; ++i) {
                ((uint4*)x)[i] = ((const uint4*)o)[i];
                ((uint4*)y)[i] = ((const uint4*)g)[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf((float)x[i], (float)y[i], sum);
            if (sizeof(T) == 2 && a.rest) {
                *(uint4*)x = *(const uint4*)((const bf16*)a.rest + row * a.head_dim + e);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf((float)x[i], (float)y[i], sum);
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        if (live && e == 0) {
            const float lse = a.lse[(int64_t)head * a.n_q + token];
            a.stats[(int64_t)head * a.n_q + token] = make_float2(lse == -INFINITY ? INFINITY : lse * LOG2E, sum);
        }
    }
}

// The weights and the gradients of x = scale q . k of one block, from the products s = q . k and g = dout . v.
// row(e, lse, delta, slope_times_distance, seen): what element e's query and key are to one another.
template <typename T, typename Row>
__device__ __forceinline__ void gradients(const Args& a, const f32x16& s, const f32x16& g, float (&p)[16], float (&d)[16], Row row) {
    const float c1 = a.scale * LOG2E, inner = a.cap > 0.f ? a.scale / a.cap : 0.f, outer = a.cap * LOG2E;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float lse, delta, off;
        const bool seen = row(e, lse, delta, off);
        float y, slope = 1.f;
        if (a.cap > 0.f) {
            const float u = bend<T>(s[e] * inner);
            slope = fmaf(-u, u, 1.f);
            y = fmaf(u, outer, -(lse + off));
        } else {
            y = fmaf(s[e], c1, -(lse + off));
        }
        const float w = __builtin_amdgcn_exp2f(y);
        p[e] = seen ? w : 0.f;
        d[e] = seen ? w * (g[e] - delta) * slope : 0.f;
    }
}

// Keys fixed: dk and dv of FIXED keys of a key head, from the rows of all its heads.
template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 64 ? 2 : 1) void key_gradients_kernel(Args a) {
    using L = Tile<T, DP>;
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][queries, dout]
    __shared__ __align__(16) float s_lse[2][L::ROWS], s_delta[2][L::ROWS], s_slope[2][L::ROWS];
    __shared__ __align__(16) int s_place[2][L::ROWS], s_doc[2][L::ROWS];

    const int key_blocks = (a.max_k + FIXED - 1) / FIXED;
    unsigned id = blockIdx.x;
    const int hk = id % a.kv_heads;
    id /= a.kv_heads;
    const int kb = (int)(id % key_blocks), s = a.seq0 + (int)(id / key_blocks);   // (causal: the keys that most rows see first)
    Seq q;
    if (!sequence(a, s, q)) return;                                       // (reported by the queries' launch)
    const int k0 = kb * FIXED;
    if (k0 >= q.kn) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int rows = q.qn * a.group, tiles = (rows + L::ROWS - 1) / L::ROWS;

    // this lane's key
    const int wk0 = k0 + 32 * wave, key = wk0 + col;
    const bool live = key < q.kn;
    const int64_t token = q.k0 + min(key, q.kn - 1);
    const int doc = a.k_docs ? (live && a.k_docs[token] >= 0 ? a.k_docs[token] : -2) : 0;
    const bool there = live && (!a.k_docs || doc >= 0);
    Fixed<T, DP> kf, vf;
    kf.load((const T*)a.k + token * a.ks.row + hk * a.ks.head, there, a.head_dim, half);
    vf.load((const T*)a.v + token * a.vs.row + hk * a.vs.head, there, a.head_dim, half);
    const Lanes<T, DP> lanes(lane);

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
    auto classify = [&](int t, bool& all) {
        const int first = (int)over_group(a, t * L::ROWS), end = (int)over_group(a, min(t * L::ROWS + L::ROWS, rows) - 1);
        bool some = true;
        all = true;
        if (a.causal) {
            some = k0 <= q.start + end || k0 < q.prefix;
            all = wlast <= q.start + first || wlast < q.prefix;
        }
        if (a.q_docs && some) {
            const int2 m = a.q_blocks[qblock0 + first / DOC_BLOCK], n = a.q_blocks[qblock0 + end / DOC_BLOCK];
            const int lo = min(m.x, n.x), hi = max(m.y, n.y);
            some = dmax >= 0 && hi >= max(dmin, 0) && lo <= dmax;
            all = all && lo == hi && dmin == dmax && lo == dmin;
        }
        return some;
    };

    Coming<T, DP> cq, cg;
    float2 cstats = make_float2(INFINITY, 0.f);
    float cslope = 0.f;
    int cplace = 0, cdoc = -1;
    auto request = [&](int t) {
        const int r0 = t * L::ROWS;
        // (a row's token and head; padding and rows past the end are zeros)
        auto find = [&](int i, int64_t& tok, int& head) {
            const int r = r0 + i;
            if (r >= rows) return false;
            const int qi = (int)over_group(a, r);
            head = hk * a.group + r - qi * a.group;
            tok = q.q0 + qi;
            return !a.q_docs || a.q_docs[tok] >= 0;
        };
        cq.load(a.head_dim, [&](int i) {
            int64_t tok;
            int head;
            return find(i, tok, head) ? (const T*)a.q + tok * a.qs.row + head * a.qs.head : nullptr;
        });
        cg.load(a.head_dim, [&](int i) {
            int64_t tok;
            int head;
            return find(i, tok, head) ? (const T*)a.dout + tok * a.gs.row + head * a.gs.head : nullptr;
        });
        if (threadIdx.x < L::ROWS) {
            int64_t tok;
            int head;
            const bool is = find(threadIdx.x, tok, head);
            cstats = is ? a.stats[head * a.n_q + tok] : make_float2(INFINITY, 0.f);
            cslope = is && a.slopes ? a.slopes[head] * LOG2E : 0.f;
            cplace = is ? q.start + (int)(tok - q.q0) : 0;
            cdoc = a.q_docs ? (is ? a.q_docs[tok] : -1) : 0;
        }
    };
    auto arrive = [&](int buf) {
        cq.store(smem[buf][0]);
        cg.store(smem[buf][1]);
        if (threadIdx.x < L::ROWS) {
            s_lse[buf][threadIdx.x] = cstats.x;
            s_delta[buf][threadIdx.x] = cstats.y;
            s_slope[buf][threadIdx.x] = cslope;
            s_place[buf][threadIdx.x] = cplace;
            s_doc[buf][threadIdx.x] = cdoc;
        }
    };

    f32x16 dk[L::NA], dv[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[i][e] = dv[i][e] = 0.f;

    Walk walk;
    int t = walk.next(0, tiles, classify), buf = 0;
    if (t < tiles) {
        request(t);
        arrive(0);
        __syncthreads();
    }
    while (t < tiles) {
        const bool whole = walk.is_whole(t);
        const int far = q.start + (int)over_group(a, min(t * L::ROWS + L::ROWS, rows) - 1);
        t = walk.next(t + 1, tiles, classify);
        if (t < tiles) request(t);
        if (wk0 < q.kn && !(a.causal && wk0 > far && wk0 >= q.prefix)) {
#pragma unroll
            for (int b = 0; b < L::BLOCKS; ++b) {
                const f32x16 sc = dot<T, DP>(smem[buf][0], b, kf, lanes), g = dot<T, DP>(smem[buf][1], b, vf, lanes);
                float p[16], d[16];
                gradients<T>(a, sc, g, p, d, [&](int e, float& lse, float& delta, float& off) {
                    const int i = 32 * b + row_of(e) + 4 * half;
                    lse = s_lse[buf][i];
                    delta = s_delta[buf][i];
                    off = a.slopes ? s_slope[buf][i] * fabsf((float)(s_place[buf][i] - key)) : 0.f;
                    if (whole) return true;
                    bool seen = !a.causal || key <= s_place[buf][i] || key < q.prefix;
                    if (a.q_docs) seen = seen && s_doc[buf][i] == doc;
                    return seen;
                });
                weigh<T, DP>(smem[buf][1], b, p, dv, lanes);
                weigh<T, DP>(smem[buf][0], b, d, dk, lanes);
                if (sizeof(T) == 2 && !whole) {
                    keep_rest(d);
                    weigh<T, DP>(smem[buf][0], b, d, dk, lanes);
                }
            }
        }
        if (t < tiles) arrive(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }
    if (!live) return;
    put_row<T, DP>((T*)a.dk + token * a.dks.row + hk * a.dks.head, dk, a.scale, a.head_dim, half);
    put_row<T, DP>((T*)a.dv + token * a.dvs.row + hk * a.dvs.head, dv, 1.f, a.head_dim, half);
}

// Queries fixed: dq of FIXED rows of a key head's queries.
template <typename T, int DP>
__global__ __launch_bounds__(256, 2) void query_gradients_kernel(Args a) {
    using L = Tile<T, DP>;
    __shared__ __align__(1024) unsigned char smem[2][2][L::BYTES];        // [buffer][keys, values]
    __shared__ __align__(16) int s_doc[2][L::ROWS];

    unsigned id = blockIdx.x;
    const int hk = id % a.kv_heads;
    id /= a.kv_heads;
    const int rb = a.row_blocks - 1 - (int)(id % a.row_blocks), s = a.seq0 + (int)(id / a.row_blocks);
    Seq q;
    if (!sequence(a, s, q)) {
        if (threadIdx.x == 0 && hk == 0 && rb == 0) report_fault(a.status, PS_ST_BAD_LENGTH, s);
        return;
    }
    const int rows = q.qn * a.group, r0 = rb * FIXED;
    if (r0 >= rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int tiles = (q.kn + L::ROWS - 1) / L::ROWS;

    const int wr0 = r0 + 32 * wave, r = min(wr0 + col, rows - 1);
    const bool live = wr0 + col < rows;
    const int qi = (int)over_group(a, r), head = hk * a.group + r - qi * a.group;
    const int64_t token = q.q0 + qi;
    const int place = q.start + qi;
    const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.f;
    const int doc = a.q_docs && live ? max(a.q_docs[token], -1) : -1;
    const bool there = live && (!a.q_docs || doc >= 0);
    Fixed<T, DP> qf, gf;
    qf.load((const T*)a.q + token * a.qs.row + head * a.qs.head, there, a.head_dim, half);
    gf.load((const T*)a.dout + token * a.gs.row + head * a.gs.head, there, a.head_dim, half);
    const float2 st = there ? a.stats[(int64_t)head * a.n_q + token] : make_float2(INFINITY, 0.f);
    const Lanes<T, DP> lanes(lane);

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
    auto classify = [&](int t, bool& all) {
        const int k0 = t * L::ROWS;
        bool some = true;
        all = k0 + L::ROWS <= q.kn;
        if (a.causal) {
            some = k0 <= far || k0 < q.prefix;
            all = all && (k0 + L::ROWS - 1 <= wnear || k0 + L::ROWS <= q.prefix);
        }
        if (a.k_docs && some) {
            const int2 m = a.k_blocks[kblock0 + k0 / DOC_BLOCK];
            some = dmax >= 0 && m.y >= max(dmin, 0) && m.x <= dmax;
            all = all && m.x == m.y && dmin == dmax && m.x == dmin;
        }
        return some;
    };

    const T* kbase = (const T*)a.k + q.k0 * a.ks.row + hk * a.ks.head;
    const T* vbase = (const T*)a.v + q.k0 * a.vs.row + hk * a.vs.head;
    Coming<T, DP> ck, cv;
    int cdoc = 0;
    auto request = [&](int t) {
        const int k0 = t * L::ROWS;
        auto is = [&](int i) { return k0 + i < q.kn && (!a.k_docs || a.k_docs[q.k0 + k0 + i] >= 0); };
        ck.load(a.head_dim, [&](int i) { return is(i) ? kbase + (int64_t)(k0 + i) * a.ks.row : nullptr; });
        cv.load(a.head_dim, [&](int i) { return is(i) ? vbase + (int64_t)(k0 + i) * a.vs.row : nullptr; });
        if (a.k_docs && threadIdx.x < L::ROWS)
            cdoc = k0 + (int)threadIdx.x < q.kn ? a.k_docs[q.k0 + k0 + threadIdx.x] : -2;
    };
    auto arrive = [&](int buf) {
        ck.store(smem[buf][0]);
        cv.store(smem[buf][1]);
        if (a.k_docs && threadIdx.x < L::ROWS) s_doc[buf][threadIdx.x] = cdoc < 0 ? -2 : cdoc;
    };

    f32x16 dq[L::NA];
#pragma unroll
    for (int i = 0; i < L::NA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[i][e] = 0.f;

    Walk walk;
    int t = walk.next(0, tiles, classify), buf = 0;
    if (t < tiles) {
        request(t);
        arrive(0);
        __syncthreads();
    }
    while (t < tiles) {
        const bool whole = walk.is_whole(t);
        const int k0 = t * L::ROWS;
        t = walk.next(t + 1, tiles, classify);
        if (t < tiles) request(t);
        if (wr0 < rows && !(a.causal && k0 > wfar && k0 >= q.prefix)) {
#pragma unroll
            for (int b = 0; b < L::BLOCKS; ++b) {
                const f32x16 sc = dot<T, DP>(smem[buf][0], b, qf, lanes), g = dot<T, DP>(smem[buf][1], b, gf, lanes);
                float p[16], d[16];
                gradients<T>(a, sc, g, p, d, [&](int e, float& lse, float& delta, float& off) {
                    const int i = 32 * b + row_of(e) + 4 * half, key = k0 + i;
                    lse = st.x;
                    delta = st.y;
                    off = a.slopes ? slope * fabsf((float)(place - key)) : 0.f;
                    if (whole) return true;
                    bool seen = key < q.kn && (!a.causal || key <= place || key < q.prefix);
                    if (a.k_docs) seen = seen && s_doc[buf][i] == doc;
                    return seen;
                });
                weigh<T, DP>(smem[buf][0], b, d, dq, lanes);
                if (sizeof(T) == 2 && !whole) {
                    keep_rest(d);
                    weigh<T, DP>(smem[buf][0], b, d, dq, lanes);
                }
            }
        }
        if (t < tiles) arrive(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }
    if (live) put_row<T, DP>((T*)a.dq + token * a.dqs.row + head * a.dqs.head, dq, a.scale, a.head_dim, half);
}

template <typename T, int DP>
void launch(const Args& a, hipStream_t st) {
    const int64_t rows = a.n_q * a.heads;
    // (a grid holds fewer than 2^32 threads: rows are taken in turn by what workgroups there are)
    if (rows > 0) hipLaunchKernelGGL(stats_kernel<T>, dim3((unsigned)min((rows + 15) / 16, (int64_t)1 << 22)), dim3(256), 0, st, a);
    Args b = a;
    auto in_parts = [&](int64_t per_seq, auto launch_one) {
        if (per_seq == 0) return;
        const int64_t most = max((int64_t)1, (int64_t)(1 << 22) / per_seq);
        for (int32_t s0 = 0, n; s0 < a.n_seq; s0 += n) {
            n = (int32_t)min((int64_t)(a.n_seq - s0), most);
            b.seq0 = s0;
            launch_one(dim3((unsigned)(per_seq * n)));
        }
    };
    in_parts((int64_t)a.kv_heads * ((a.max_k + FIXED - 1) / FIXED), [&](dim3 grid) {
        hipLaunchKernelGGL((key_gradients_kernel<T, DP>), grid, dim3(256), 0, st, b);
    });
    in_parts((int64_t)a.kv_heads * a.row_blocks, [&](dim3 grid) {
        hipLaunchKernelGGL((query_gradients_kernel<T, DP>), grid, dim3(256), 0, st, b);
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
    if (p.a.n_seq == 0 || (p.a.n_q == 0 && p.a.n_k == 0)) return PS_OK;
    const ps_attention_desc* d = desc;
    if (p.a.n_q > 0 && (check_strides(d, d->q, q, false, d->heads) || check_strides(d, d->out, out, false, d->heads) || !lse ||
                        check_strides(d, d->dout, dout, false, d->heads) || check_strides(d, d->dq, dq, true, d->heads)))
        return PS_EINVAL;
    if (p.a.n_k > 0 && (check_strides(d, d->k, k, false, d->kv_heads) || check_strides(d, d->v, v, false, d->kv_heads) ||
                        check_strides(d, d->dk, dk, true, d->kv_heads) || check_strides(d, d->dv, dv, true, d->kv_heads)))
        return PS_EINVAL;
    if (((uintptr_t)out_rest & 15) != 0 || (out_rest && d->dtype != 1) || (uintptr_t)lse % 4 != 0) return PS_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < p.bytes) return PS_EWORKSPACE;
    Args& a = p.a;
    a.q = q; a.k = k; a.v = v; a.out = out; a.lse = lse; a.rest = out_rest; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv; a.status = status;
    hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();
    summarise_documents(a, st);
    if (desc->dtype == 1)
        desc->head_dim <= 64 ? launch<bf16, 64>(a, st) : launch<bf16, 128>(a, st);
    else
        desc->head_dim <= 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
