// Norms of queries and keys, a head of a row at a time, with the rotation to their positions in the same pass, and the gradients.
//     r = 1 / sqrt(mean x^2 + eps),  u = r x,  out = turn(u w);   g = turn back(dout),  dw = sum g u,  dx = r (g w - u mean(g w u)).
// A head stays in the registers of a few neighbouring lanes, which have all they need of it to themselves but two sums: those of x^2 and,
// backwards, of g w x, which do not wait for one another.  So every tensor is read once and written once, and memory bounds the call.
#include <math.h>

#include "internal.h"
#include "rotary.h"

typedef __bf16 bf16;

namespace {

struct NormArgs {
    const void *x[2], *weight[2], *dout[2];
    void* out[2];                      // out, or dx
    ps_strides xs[2], gs[2], os[2];
    float* partial;                    // backwards, [workgroups][2][head_dim]: sums of the weights' gradients
    const int32_t* positions;
    const float* frequencies;
    int64_t n_rows;
    int32_t heads[2], head_dim, n_pairs, interleaved;
    int32_t rows, heads_each;          // rows of a tile, heads of a workgroup
    int32_t lanes, units;              // lanes to a head (a power of two), units of a head
    float magnitude, eps;
};

constexpr int TABLE = 256;             // pairs of a tile's rows, at most
constexpr int MOST_BLOCKS = 1024;      // workgroups along the rows, backwards

// A head is cut into units of two pieces of VEC elements: pieces that turn with one another (halves; single elements, interleaved), or that
// turn within themselves or not at all.  A lane has PER units, the same of every head.
template <typename T, int VEC, int PER, bool BACK>
__global__ __launch_bounds__(256) void norm_rotary_kernel(NormArgs a) {
    struct Piece { T v[VEC]; };        // (moved whole at any address)
    constexpr int BATCH = BACK ? 1 : 2;   // heads of a lane on their way together
    __shared__ float2 table[TABLE];
    __shared__ float s_sum[BACK ? 256 * 2 * VEC * PER : 1];

    const int n = a.n_pairs, lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = 256 / a.lanes;
    const bool together = !a.interleaved || VEC == 1;                     // a turning unit's pieces turn with one another
    const int turning = together ? n / VEC : 0, apart = a.interleaved ? 1 : n, step = a.interleaved ? 2 : VEC;
    int e[PER][2], at[PER][2];         // a piece's first element, -1: none; its first pair, -1: does not turn
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int u = lane + k * a.lanes;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (u < turning) {
                e[k][i] = u * step + i * apart;
                at[k][i] = u * VEC;
            } else {
                e[k][i] = (together ? 2 * n : 0) + (2 * (u - turning) + i) * VEC;
                at[k][i] = e[k][i] < 2 * n ? e[k][i] / 2 : -1;
                if (e[k][i] >= a.head_dim) e[k][i] = -1;
            }
        }
    }
    float acc[2][PER][2][VEC];
    if (BACK) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) acc[t][k][i][j] = 0.f;
    }

    // a unit's elements turned, or turned back
    auto turn = [&](float (&v)[2][VEC], int k, const float2* cs, float sign) {
        const int u = lane + k * a.lanes;
        if (u < turning) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float2 w = cs[at[k][0] + j];
                const float p = v[0][j], q = v[1][j], s = w.y * sign;
                v[0][j] = fmaf(-q, s, p * w.x);
                v[1][j] = fmaf(q, w.x, p * s);
            }
            return;
        }
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (at[k][i] >= 0) {
#pragma unroll
                    for (int j = 0; j < VEC; j += 2) {
                        const float2 w = cs[at[k][i] + j / 2];
                        const float p = v[i][j], q = v[i][j + 1], s = w.y * sign;
                        v[i][j] = fmaf(-q, s, p * w.x);
                        v[i][j + 1] = fmaf(q, w.x, p * s);
                    }
                }
        }
    };
    auto over_lanes = [&](float v) {
        for (int o = 1; o < a.lanes; o *= 2) v += __shfl_xor(v, o, 64);
        return v;
    };

    for (int64_t tile = blockIdx.x; tile * a.rows < a.n_rows; tile += gridDim.x) {
        const int64_t row0 = tile * a.rows;
        const int rows = (int)min((int64_t)a.rows, a.n_rows - row0);
        __syncthreads();                                                  // (the tile before is done with the table)
        for (int i = threadIdx.x; i < rows * n; i += 256) {
            const float2 w = turn_of(a.positions[row0 + i / n], a.frequencies[i % n]);
            table[i] = make_float2(w.x * a.magnitude, w.y * a.magnitude);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int in_front = t == 0 ? 0 : a.heads[0], head0 = blockIdx.y * a.heads_each;
            const int h0 = max(head0 - in_front, 0), heads = min(head0 + a.heads_each - in_front, a.heads[t]) - h0;
            if (heads <= 0) continue;
            const T* weights = (const T*)a.weight[t];
            float w[PER][2][VEC];
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) w[k][i][j] = weights && e[k][i] >= 0 ? (float)weights[e[k][i] + j] : 1.f;
            for (int first = 0; first < rows * heads; first += groups * BATCH) {
                Piece x[BATCH][PER][2], g[BATCH][PER][2];
                int r[BATCH];
                T* to[BATCH];
                bool is[BATCH];
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    const unsigned i = first + b * groups + group;
                    is[b] = (int)i < rows * heads;
                    r[b] = is[b] ? i / (unsigned)heads : 0;
                    const int h = h0 + (is[b] ? (int)(i - r[b] * (unsigned)heads) : 0);
                    const int64_t row = row0 + r[b];
                    const T* from = (const T*)a.x[t] + row * a.xs[t].row + h * a.xs[t].head;
                    to[b] = (T*)a.out[t] + row * a.os[t].row + h * a.os[t].head;
                    const T* gradient = BACK ? (const T*)a.dout[t] + row * a.gs[t].row + h * a.gs[t].head : nullptr;
#pragma unroll
                    for (int k = 0; k < PER; ++k)
#pragma unroll
                        for (int i2 = 0; i2 < 2; ++i2) {
                            const bool there = is[b] && e[k][i2] >= 0;
#pragma unroll
                            for (int j = 0; j < VEC; ++j) x[b][k][i2].v[j] = g[b][k][i2].v[j] = (T)0.f;
                            if (there) {
                                x[b][k][i2] = *(const Piece*)(from + e[k][i2]);
                                if (BACK) g[b][k][i2] = *(const Piece*)(gradient + e[k][i2]);
                            }
                        }
                }
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    const float2* cs = table + r[b] * n;
                    float squares = 0.f, along = 0.f, gv[PER][2][VEC];
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        if (BACK) {
#pragma unroll
                            for (int i = 0; i < 2; ++i)
#pragma unroll
                                for (int j = 0; j < VEC; ++j) gv[k][i][j] = (float)g[b][k][i].v[j];
                            turn(gv[k], k, cs, -1.f);
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < VEC; ++j) {
                                const float v = (float)x[b][k][i].v[j];
                                squares = fmaf(v, v, squares);
                                if (BACK) along = fmaf(gv[k][i][j] * w[k][i][j], v, along);
                            }
                    }
                    squares = over_lanes(squares);
                    const float by = 1.f / sqrtf(squares / (float)a.head_dim + a.eps);
                    if (BACK) along = over_lanes(along) * by / (float)a.head_dim;
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        float v[2][VEC];
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < VEC; ++j) {
                                const float u = (float)x[b][k][i].v[j] * by;
                                if (BACK) {
                                    acc[t][k][i][j] = fmaf(gv[k][i][j], u, acc[t][k][i][j]);
                                    v[i][j] = by * fmaf(-u, along, gv[k][i][j] * w[k][i][j]);
                                } else {
                                    v[i][j] = u * w[k][i][j];
                                }
                            }
                        if (!BACK) turn(v, k, cs, 1.f);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (is[b] && e[k][i] >= 0) {
                                Piece o;
#pragma unroll
                                for (int j = 0; j < VEC; ++j) o.v[j] = (T)v[i][j];
                                *(Piece*)(to[b] + e[k][i]) = o;
                            }
                    }
                }
            }
        }
    }
    if constexpr (BACK) {
        // what the workgroup's lanes have of an element, added up in their order
        float* out = a.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.head_dim;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s_sum[((k * 2 + i) * VEC + j) * 256 + threadIdx.x] = acc[t][k][i][j];
            __syncthreads();
            if (a.heads[t] == 0) continue;
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        // the element's share of the first group that is this thread's turn
                        const int which = (k * 2 + i) * VEC + j;
                        if (which % groups != group || e[k][i] < 0) continue;
                        float sum = 0.f;
                        for (int m = 0; m < groups; ++m) sum += s_sum[which * 256 + m * a.lanes + lane];
                        out[t * a.head_dim + e[k][i] + j] = sum;
                    }
        }
    }
}

// The workgroups' sums added up: 8 columns a workgroup, 32 threads to each.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* partial, int parts, int head_dim, float* dweight, float* dweight2) {
    __shared__ float s[256];
    const int c = blockIdx.x * 8 + (threadIdx.x & 7);
    float sum = 0.f;
    if (c < 2 * head_dim) {
#pragma unroll 8
        for (int p = threadIdx.x >> 3; p < parts; p += 32) sum += partial[(int64_t)p * 2 * head_dim + c];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 8 || c >= 2 * head_dim) return;
    sum = 0.f;
    for (int i = 0; i < 32; ++i) sum += s[i * 8 + threadIdx.x];
    float* to = c < head_dim ? dweight : dweight2;
    if (to) to[c < head_dim ? c : c - head_dim] = sum;
}

// How a call is cut up.
struct Cut {
    int vec, per;
    int64_t tiles, blocks;             // tiles of rows; workgroups along them
    int shares;                        // of the heads
};

bool strides_ok(const ps_strides& s, bool written, int heads, int head_dim, int64_t rows) {
    return s.row >= 0 && s.head >= 0 && (!written || strides_apart(s, rows, heads, head_dim));
}

// Rows of a tile: a pair a thread for the table; heads are shared out where rows alone do not fill the chip.  (Nothing here goes by n_pairs
// that the workspace is sized by: it holds the most there can be.)
Cut cut(NormArgs& a, size_t es, bool back) {
    Cut c;
    const uintptr_t pieces = (uintptr_t)(a.head_dim | (a.interleaved ? 2 * a.n_pairs : a.n_pairs)) * es;
    c.vec = (int)((pieces % 16 == 0 ? 16 : pieces % 8 == 0 ? 8 : es) / es);
    const bool together = !a.interleaved || c.vec == 1;
    const int turning = together ? a.n_pairs / c.vec : 0, rest = (a.head_dim - (together ? 2 * a.n_pairs : 0)) / c.vec;
    a.units = turning + (rest + 1) / 2;
    a.lanes = 1;
    while (a.lanes < a.units && a.lanes < 64) a.lanes *= 2;
    c.per = a.units > 64 ? 4 : 1;
    const int all = a.heads[0] + a.heads[1];
    const int most = a.n_pairs > 0 ? TABLE / a.n_pairs : 8;
    a.rows = most < 8 ? most : 8;
    while (a.rows > 1 && (a.n_rows + a.rows - 1) / a.rows < 1024) a.rows /= 2;
    c.tiles = (a.n_rows + a.rows - 1) / a.rows;
    c.blocks = back && c.tiles > MOST_BLOCKS ? MOST_BLOCKS : c.tiles;
    const int shares = (int)(c.tiles >= 512 ? 1 : 512 / c.tiles < all ? 512 / c.tiles : all);
    a.heads_each = (all + shares - 1) / shares;
    c.shares = (all + a.heads_each - 1) / a.heads_each;
    return c;
}

template <typename T, bool BACK>
void launch(const NormArgs& a, const Cut& c, dim3 grid, hipStream_t st) {
    constexpr int W = 16 / sizeof(T);
    const dim3 threads(256);
    if (c.vec == W)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W, 1, BACK>), grid, threads, 0, st, a);
    else if (c.vec == W / 2 && c.per == 1)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W / 2, 1, BACK>), grid, threads, 0, st, a);
    else if (c.vec == W / 2)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W / 2, (sizeof(T) == 4 ? 4 : 1), BACK>), grid, threads, 0, st, a);
    else if (c.per == 1)
        hipLaunchKernelGGL((norm_rotary_kernel<T, 1, 1, BACK>), grid, threads, 0, st, a);
    else
        hipLaunchKernelGGL((norm_rotary_kernel<T, 1, 4, BACK>), grid, threads, 0, st, a);
}

// Arguments that both directions check.
int check(const ps_norm_rotary_desc* d, const void* x2) {
    if (!d || (d->dtype != 0 && d->dtype != 1) || d->head_dim < 1 || d->n_pairs < 0 || (int64_t)2 * d->n_pairs > d->head_dim || d->heads < 1 ||
        d->heads2 < 0 || d->n_rows < 0 || (d->interleaved & ~1) || (d->heads2 > 0) != (x2 != nullptr))
        return PS_EINVAL;
    if (!(d->eps > 0.f) || isinf(d->eps)) return PS_EINVAL;
    // (a workgroup counts the heads of its rows, 8 at most, in 32 bits)
    if (d->head_dim > 512 || ((int64_t)d->heads + d->heads2) * d->head_dim > 1 << 27 || d->n_rows > INT32_MAX) return PS_EUNSUPPORTED;
    return PS_OK;
}

bool same(const ps_strides& a, const ps_strides& b) { return a.row == b.row && a.head == b.head; }

template <bool BACK>
int enqueue(NormArgs& a, const ps_norm_rotary_desc* d, hipStream_t st, int64_t& parts) {
    const size_t es = d->dtype == 1 ? 2 : 4;
    const Cut c = cut(a, es, BACK);
    parts = c.blocks * c.shares;
    const int64_t per = 1 << 22;       // (a grid holds fewer than 2^32 threads)
    for (int64_t b0 = 0; b0 < c.blocks; b0 += per) {
        NormArgs b = a;
        const int64_t first = b0 * a.rows;
        if (!BACK) {
            for (int i = 0; i < 2; ++i) {
                if (!b.x[i]) continue;
                b.x[i] = (const char*)a.x[i] + (size_t)first * a.xs[i].row * es;
                b.out[i] = (char*)a.out[i] + (size_t)first * a.os[i].row * es;
            }
            if (a.positions) b.positions = a.positions + first;
            b.n_rows = a.n_rows - first;
        }
        const dim3 grid((unsigned)(c.blocks - b0 < per ? c.blocks - b0 : per), (unsigned)c.shares);
        if (!BACK) b.n_rows = b.n_rows < (int64_t)grid.x * a.rows ? b.n_rows : (int64_t)grid.x * a.rows;
        d->dtype == 1 ? launch<bf16, BACK>(b, c, grid, st) : launch<float, BACK>(b, c, grid, st);
    }
    return PS_OK;
}

}  // namespace

extern "C" int ps_norm_rotary_forward(const ps_norm_rotary_desc* d, const void* x, const void* weight, void* out, const void* x2,
                                      const void* weight2, void* out2, const int32_t* positions, const float* frequencies, void* hip_stream) {
    const int code = check(d, x2);
    if (code != PS_OK) return code;
    if (!x2 != !out2 || (!x2 && weight2) || !strides_ok(d->x, false, d->heads, d->head_dim, d->n_rows) || !strides_ok(d->out, true, d->heads, d->head_dim, d->n_rows) ||
        (x2 && (!strides_ok(d->x2, false, d->heads2, d->head_dim, d->n_rows) || !strides_ok(d->out2, true, d->heads2, d->head_dim, d->n_rows))))
        return PS_EINVAL;
    if (d->n_rows == 0) return PS_OK;
    if (!x || !out || (d->n_pairs > 0 && (!positions || !frequencies))) return PS_EINVAL;
    const size_t es = d->dtype == 1 ? 2 : 4;
    if (((uintptr_t)x | (uintptr_t)out | (uintptr_t)x2 | (uintptr_t)out2 | (uintptr_t)weight | (uintptr_t)weight2) % es != 0) return PS_EINVAL;
    if ((x == out && !same(d->x, d->out)) || (x2 && x2 == out2 && !same(d->x2, d->out2))) return PS_EINVAL;
    NormArgs a = {{x, x2}, {weight, weight2}, {nullptr, nullptr}, {out, out2}, {d->x, d->x2}, {}, {d->out, d->out2}, nullptr, positions, frequencies,
                  d->n_rows, {d->heads, d->heads2}, d->head_dim, d->n_pairs, d->interleaved, 1, 1, 1, 1, d->magnitude, d->eps};
    (void)hipGetLastError();
    int64_t parts;
    enqueue<false>(a, d, (hipStream_t)hip_stream, parts);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

extern "C" size_t ps_norm_rotary_workspace_bytes(int64_t n_rows, int32_t heads, int32_t heads2, int32_t head_dim) {
    if (n_rows < 0 || n_rows > INT32_MAX || heads < 1 || heads2 < 0 || head_dim < 1 || head_dim > 512) return 0;
    // (workgroups along the rows times shares of the heads: at most the one or 512 of both)
    return align_up(sizeof(float) * 2 * (size_t)head_dim * MOST_BLOCKS, 256);
}

extern "C" int ps_norm_rotary_backward(const ps_norm_rotary_desc* d, const void* x, const void* weight, const void* dout, void* dx, float* dweight,
                                       const void* x2, const void* weight2, const void* dout2, void* dx2, float* dweight2, const int32_t* positions,
                                       const float* frequencies, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int code = check(d, x2);
    if (code != PS_OK) return code;
    if (!x2 != !dout2 || !x2 != !dx2 || (!x2 && (weight2 || dweight2))) return PS_EINVAL;
    for (int i = 0; i < (x2 ? 2 : 1); ++i) {
        const int heads = i == 0 ? d->heads : d->heads2;
        if (!strides_ok(i == 0 ? d->x : d->x2, false, heads, d->head_dim, d->n_rows) || !strides_ok(i == 0 ? d->dout : d->dout2, false, heads, d->head_dim, d->n_rows) ||
            !strides_ok(i == 0 ? d->dx : d->dx2, true, heads, d->head_dim, d->n_rows))
            return PS_EINVAL;
    }
    const size_t es = d->dtype == 1 ? 2 : 4;
    if (((uintptr_t)dweight | (uintptr_t)dweight2) % 4 != 0) return PS_EINVAL;
    if (d->n_rows > 0) {
        if (!x || !dout || !dx || (d->n_pairs > 0 && (!positions || !frequencies))) return PS_EINVAL;
        if (((uintptr_t)x | (uintptr_t)dout | (uintptr_t)dx | (uintptr_t)x2 | (uintptr_t)dout2 | (uintptr_t)dx2 | (uintptr_t)weight | (uintptr_t)weight2) % es != 0)
            return PS_EINVAL;
        if ((dx == x && !same(d->x, d->dx)) || (dx == dout && !same(d->dout, d->dx)) || (x2 && ((dx2 == x2 && !same(d->x2, d->dx2)) || (dx2 == dout2 && !same(d->dout2, d->dx2)))))
            return PS_EINVAL;
    }
    if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < ps_norm_rotary_workspace_bytes(d->n_rows, d->heads, d->heads2, d->head_dim)) return PS_EWORKSPACE;
    NormArgs a = {{x, x2}, {weight, weight2}, {dout, dout2}, {dx, dx2}, {d->x, d->x2}, {d->dout, d->dout2}, {d->dx, d->dx2}, (float*)workspace, positions,
                  frequencies, d->n_rows, {d->heads, d->heads2}, d->head_dim, d->n_pairs, d->interleaved, 1, 1, 1, 1, d->magnitude, d->eps};
    hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();
    int64_t parts = 0;
    if (d->n_rows > 0) enqueue<true>(a, d, st, parts);
    if (dweight || dweight2)
        hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((2 * d->head_dim + 7) / 8)), dim3(256), 0, st, (const float*)workspace, (int)parts,
                           d->head_dim, dweight, dweight2);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
