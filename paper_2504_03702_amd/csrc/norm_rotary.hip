// Norms of queries and keys, a head of a row at a time, with the rotation to their positions in the same pass, and the gradients.
//     r = 1 / sqrt(mean x^2 + eps),  u = r x,  out = turn(u w);   g = turn back(dout),  dw = sum g u,  dx = r (g w - u mean(g w u)).
// A head stays in the registers of a few neighbouring lanes, which have all they need of it to themselves but two sums: those of x^2 and,
// backwards, of g w x, which do not wait for one another.  So every tensor is read once and written once, and memory bounds the call.
// dw is a sum in fp32, of a lane's heads, lanes and workgroups in turn, of u that the hardware's root (one place off at most) has made: 2e-7 of its norm from 64 bits at 3333 and 32768 rows.
#include <float.h>
#include <math.h>

#include "internal.h"
#include "rotary.h"

typedef __bf16 bf16;

namespace {

struct NormArgs {
    const void *x[2], *weight[2], *dout[2];
    void* out[2];                      // out, or dx
    ps_strides xs[2], gs[2], os[2];
    float* partial[2];                 // backwards, [workgroups of a tensor][head_dim]: sums of the weight's gradient
    const int32_t* positions;
    const float* frequencies;
    int64_t n_rows;
    int32_t heads[2], head_dim, n_pairs, interleaved;
    int32_t rows, heads_each, shares[2];   // rows of a tile; heads of a workgroup, and workgroups of a tile for each tensor
    int32_t lanes, units;              // lanes to a head (a power of two), units of a head
    uint32_t by_pairs, by_heads;       // 2^32 / n_pairs + 1, 2^32 / heads_each + 1 (of 2 to 4096), for quotients
    float magnitude, eps;
};

constexpr int TABLE = 512;             // pairs of a tile's rows, at most
constexpr int MOST_BLOCKS = 1024;      // workgroups along the rows, backwards

// A head is cut into units of two pieces of VEC elements: pieces that turn with one another (halves; single elements, interleaved), or that
// turn within themselves or not at all.  A lane has PER units, the same of every head.  A workgroup has a tile's rows of some heads of one tensor; the first BATCH
// heads of its lanes are on their way while the table is made.  WHOLE: all lanes have all pieces, so nothing is asked of any (32768 rows of two tensors of 16
// heads of 64 in bf16, forwards 72 -> 51 us).
template <typename T, int VEC, int PER, bool BACK, bool WHOLE>
__global__ __launch_bounds__(256) void norm_rotary_kernel(NormArgs a) {
    struct Piece { T v[VEC]; };        // (moved whole at any address)
    constexpr int BATCH = PER > 1 || BACK ? 1 : 2;
    __shared__ float2 table[TABLE];
    __shared__ float s_sum[BACK ? 256 * 2 * VEC * PER : 1];

    const int second = blockIdx.y >= (unsigned)a.shares[0];
    const int n = a.n_pairs, lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = 256 / a.lanes;
    const int h0 = ((int)blockIdx.y - (second ? a.shares[0] : 0)) * a.heads_each, heads = min(a.heads_each, (second ? a.heads[1] : a.heads[0]) - h0);
    // (chosen, not indexed: the arguments would go to memory for it)
    const T *const from = (const T*)(second ? a.x[1] : a.x[0]), *const gradient = (const T*)(second ? a.dout[1] : a.dout[0]);
    const T* const weights = (const T*)(second ? a.weight[1] : a.weight[0]);
    T* const to = (T*)(second ? a.out[1] : a.out[0]);
    const int64_t x_row = second ? a.xs[1].row : a.xs[0].row, x_head = second ? a.xs[1].head : a.xs[0].head, o_row = second ? a.os[1].row : a.os[0].row,
                  o_head = second ? a.os[1].head : a.os[0].head, g_row = second ? a.gs[1].row : a.gs[0].row, g_head = second ? a.gs[1].head : a.gs[0].head;
    const float of_head = 1.f / (float)a.head_dim;
    const bool together = !a.interleaved || VEC == 1;                     // a turning unit's pieces turn with one another
    const int turning = together ? n / VEC : 0, apart = a.interleaved ? 1 : n, step = a.interleaved ? 2 : VEC;
    int e[PER][2], at[PER][2];         // a piece's first element, -1: none; its first pair, -1: does not turn
    float w[PER][2][VEC];
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
            Piece of;
            if (weights) of = *(const Piece*)(weights + max(e[k][i], 0));
#pragma unroll
            for (int j = 0; j < VEC; ++j) w[k][i][j] = weights ? (float)of.v[j] : 1.f;
        }
    }
    float acc[PER][2][VEC];
    if (BACK) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) acc[k][i][j] = 0.f;
    }

    // a unit's elements turned, or turned back
    auto turn = [&](float (&v)[2][VEC], int k, const float2* cs, float sign) {
        const int u = lane + k * a.lanes;
        if (u < turning) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float2 c = cs[at[k][0] + j];
                const float p = v[0][j], q = v[1][j], s = c.y * sign;
                v[0][j] = fmaf(-q, s, p * c.x);
                v[1][j] = fmaf(q, c.x, p * s);
            }
            return;
        }
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (at[k][i] >= 0) {
#pragma unroll
                    for (int j = 0; j < VEC; j += 2) {
                        const float2 c = cs[at[k][i] + j / 2];
                        const float p = v[i][j], q = v[i][j + 1], s = c.y * sign;
                        v[i][j] = fmaf(-q, s, p * c.x);
                        v[i][j + 1] = fmaf(q, c.x, p * s);
                    }
                }
        }
    };
    // (of neighbouring lanes, the same in all of them)
    auto over_lanes = [&](float v) {
        for (int o = 1; o < a.lanes; o *= 2) v += __shfl_xor(v, o, 64);
        return v;
    };

    Piece x[BATCH][PER][2], g[BATCH][PER][2];
    int r[BATCH], h[BATCH];            // row of the tile and head
    bool there[BATCH];
    int64_t row0 = 0;
    int rows = 0;
    auto fetch = [&](int first) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = first + b * groups + group;
            const bool is = i < rows * heads;
            const int mine = WHOLE && !is ? rows * heads - 1 : i;         // (the last head again, to no effect)
            const int quotient = heads == 1 ? mine : a.by_heads && heads == a.heads_each ? (int)__umulhi((unsigned)mine, a.by_heads) : mine / heads;
            there[b] = is;
            r[b] = WHOLE || is ? quotient : 0;
            h[b] = h0 + mine - quotient * heads;
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (!WHOLE) {
#pragma unroll
                        for (int v = 0; v < VEC; ++v) x[b][k][j].v[v] = g[b][k][j].v[v] = (T)0.f;
                        if (!is || e[k][j] < 0) continue;
                    }
                    x[b][k][j] = *(const Piece*)(from + (row0 + r[b]) * x_row + h[b] * x_head + e[k][j]);
                    if (BACK) g[b][k][j] = *(const Piece*)(gradient + (row0 + r[b]) * g_row + h[b] * g_head + e[k][j]);
                }
        }
    };
    auto work = [&] {
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
            if (BACK) along = over_lanes(along);
            const float by = __builtin_amdgcn_rsqf(fmaf(squares, of_head, a.eps)), mean = along * by * of_head;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                float v[2][VEC];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float u = (float)x[b][k][i].v[j] * by;
                        if (BACK) {
                            // (chosen, not multiplied by zero: a head that is there again may be overwritten by its own dx in the meantime)
                            const float with = fmaf(gv[k][i][j], u, acc[k][i][j]);
                            acc[k][i][j] = !WHOLE || there[b] ? with : acc[k][i][j];
                            v[i][j] = by * fmaf(-u, mean, gv[k][i][j] * w[k][i][j]);
                        } else {
                            v[i][j] = u * w[k][i][j];
                        }
                    }
                if (!BACK) turn(v, k, cs, 1.f);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (there[b] && (WHOLE || e[k][i] >= 0)) {
                        Piece o;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) o.v[j] = (T)v[i][j];
                        *(Piece*)(to + (row0 + r[b]) * o_row + h[b] * o_head + e[k][i]) = o;
                    }
            }
        }
    };

    for (int64_t tile = blockIdx.x; tile * a.rows < a.n_rows; tile += gridDim.x) {
        row0 = tile * a.rows;
        rows = (int)min((int64_t)a.rows, a.n_rows - row0);
        fetch(0);
        if (BACK) __syncthreads();                                        // (the tile before is done with the table)
        for (int i = threadIdx.x; i < rows * n; i += 256) {
            const int row = n == 1 ? i : (int)__umulhi((unsigned)i, a.by_pairs);
            const float2 c = turn_of(a.positions[row0 + row], a.frequencies[i - row * n]);
            table[i] = make_float2(c.x * a.magnitude, c.y * a.magnitude);
        }
        __syncthreads();
        work();
        for (int first = groups * BATCH; first < rows * heads; first += groups * BATCH) {
            fetch(first);
            work();
        }
    }
    if constexpr (BACK) {
        // what the workgroup's lanes have of an element, added up in their order
        float* out = (second ? a.partial[1] : a.partial[0]) + ((int64_t)blockIdx.x * (second ? a.shares[1] : a.shares[0]) + h0 / a.heads_each) * a.head_dim;
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s_sum[((k * 2 + i) * VEC + j) * 256 + threadIdx.x] = acc[k][i][j];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int which = (k * 2 + i) * VEC + j;              // (the groups take turns)
                    if (which % groups != group || e[k][i] < 0) continue;
                    float sum = 0.f;
                    for (int m = 0; m < groups; ++m) sum += s_sum[which * 256 + m * a.lanes + lane];
                    out[e[k][i] + j] = sum;
                }
    }
}

// The workgroups' sums added up, of both tensors: 8 columns a workgroup, 32 threads to each.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* partial, const float* partial2, int parts, int parts2, int head_dim, float* dweight, float* dweight2) {
    __shared__ float s[256];
    const int c = blockIdx.x * 8 + (threadIdx.x & 7), n = blockIdx.y ? parts2 : parts;
    const float* from = blockIdx.y ? partial2 : partial;
    float* to = blockIdx.y ? dweight2 : dweight;
    if (!to) return;
    float sum = 0.f;
    if (c < head_dim) {
#pragma unroll 16
        for (int p = threadIdx.x >> 3; p < n; p += 32) sum += from[(int64_t)p * head_dim + c];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 8 || c >= head_dim) return;
    sum = 0.f;
    for (int i = 0; i < 32; ++i) sum += s[i * 8 + threadIdx.x];
    to[c] = sum;
}

// How a call is cut up.
struct Cut {
    int vec, per;
    int64_t tiles, blocks;             // tiles of rows; workgroups along them
};

bool strides_ok(const ps_strides& s, bool written, int heads, int head_dim, int64_t rows) {
    return s.row >= 0 && s.head >= 0 && (!written || strides_apart(s, rows, heads, head_dim));
}

// Rows of a tile: a pair a thread for the table, two tiles to a unit or more (3333 rows of 12 fp32 heads of 80: in 1667 tiles forwards / backwards 13.5 / 15.4 us,
// in 834 10.3 / 14.3); heads are shared out where rows alone do not fill the chip.  (Nothing here goes by n_pairs
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
    const int all = a.heads[0] + a.heads[1], larger = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1];
    const int most = a.n_pairs > 0 ? TABLE / a.n_pairs : 16;
    a.rows = most < 16 ? most : 16;
    while (a.rows > 1 && (a.n_rows + a.rows - 1) / a.rows < 512) a.rows /= 2;
    c.tiles = (a.n_rows + a.rows - 1) / a.rows;
    c.blocks = back && c.tiles > MOST_BLOCKS ? MOST_BLOCKS : c.tiles;
    const int shares = (int)(c.tiles >= 512 ? 1 : 512 / c.tiles < all ? 512 / c.tiles : all);
    a.heads_each = (all + shares - 1) / shares < larger ? (all + shares - 1) / shares : larger;
    for (int i = 0; i < 2; ++i) a.shares[i] = (a.heads[i] + a.heads_each - 1) / a.heads_each;
    auto inverse = [](int x) { return x > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint64_t)x + 1) : 0u; };
    a.by_pairs = inverse(a.n_pairs);
    a.by_heads = a.heads_each <= 4096 ? inverse(a.heads_each) : 0;
    return c;
}

template <typename T, bool BACK>
void launch(const NormArgs& a, const Cut& c, dim3 grid, hipStream_t st) {
    constexpr int W = 16 / sizeof(T);
    const dim3 threads(256);
    if (c.vec == W && a.head_dim == 2 * W * a.lanes)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W, 1, BACK, true>), grid, threads, 0, st, a);
    else if (c.vec == W)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W, 1, BACK, false>), grid, threads, 0, st, a);
    else if (c.vec == W / 2 && c.per == 1)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W / 2, 1, BACK, false>), grid, threads, 0, st, a);
    else if (c.vec == W / 2)
        hipLaunchKernelGGL((norm_rotary_kernel<T, W / 2, (sizeof(T) == 4 ? 4 : 1), BACK, false>), grid, threads, 0, st, a);
    else if (c.per == 1)
        hipLaunchKernelGGL((norm_rotary_kernel<T, 1, 1, BACK, false>), grid, threads, 0, st, a);
    else
        hipLaunchKernelGGL((norm_rotary_kernel<T, 1, 4, BACK, false>), grid, threads, 0, st, a);
}

// Arguments that both directions check.
int check(const ps_norm_rotary_desc* d, const void* x2) {
    if (!d || (d->dtype != 0 && d->dtype != 1) || d->head_dim < 1 || d->n_pairs < 0 || (int64_t)2 * d->n_pairs > d->head_dim || d->heads < 1 ||
        d->heads2 < 0 || d->n_rows < 0 || (d->interleaved & ~1) || (d->heads2 > 0) != (x2 != nullptr))
        return PS_EINVAL;
    if (!(d->eps >= FLT_MIN) || isinf(d->eps)) return PS_EINVAL;          // (the root takes no smaller numbers, and a head may be zeros)
    // (a workgroup counts the heads of its rows, 16 at most, in 32 bits)
    if (d->head_dim > 512 || ((int64_t)d->heads + d->heads2) * d->head_dim > 1 << 26 || d->n_rows > INT32_MAX) return PS_EUNSUPPORTED;
    return PS_OK;
}

bool same(const ps_strides& a, const ps_strides& b) { return a.row == b.row && a.head == b.head; }

template <bool BACK>
int64_t enqueue(NormArgs& a, const ps_norm_rotary_desc* d, hipStream_t st) {
    const size_t es = d->dtype == 1 ? 2 : 4;
    const Cut c = cut(a, es, BACK);
    if (BACK) a.partial[1] = a.partial[0] + c.blocks * a.shares[0] * a.head_dim;
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
        const dim3 grid((unsigned)(c.blocks - b0 < per ? c.blocks - b0 : per), (unsigned)(a.shares[0] + a.shares[1]));
        if (!BACK) b.n_rows = b.n_rows < (int64_t)grid.x * a.rows ? b.n_rows : (int64_t)grid.x * a.rows;
        d->dtype == 1 ? launch<bf16, BACK>(b, c, grid, st) : launch<float, BACK>(b, c, grid, st);
    }
    return c.blocks;
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
    NormArgs a = {{x, x2}, {weight, weight2}, {nullptr, nullptr}, {out, out2}, {d->x, d->x2}, {}, {d->out, d->out2}, {}, positions, frequencies,
                  d->n_rows, {d->heads, d->heads2}, d->head_dim, d->n_pairs, d->interleaved, 1, 1, {}, 1, 1, 0, 0, d->magnitude, d->eps};
    (void)hipGetLastError();
    enqueue<false>(a, d, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

extern "C" size_t ps_norm_rotary_workspace_bytes(int64_t n_rows, int32_t heads, int32_t heads2, int32_t head_dim) {
    if (n_rows < 0 || n_rows > INT32_MAX || heads < 1 || heads2 < 0 || head_dim < 1 || head_dim > 512 || ((int64_t)heads + heads2) * head_dim > 1 << 26) return 0;
    // (workgroups along the rows times shares of the heads of both tensors: two of the one, or 512 and a tile's more)
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
    NormArgs a = {{x, x2}, {weight, weight2}, {dout, dout2}, {dx, dx2}, {d->x, d->x2}, {d->dout, d->dout2}, {d->dx, d->dx2}, {(float*)workspace, (float*)workspace}, positions,
                  frequencies, d->n_rows, {d->heads, d->heads2}, d->head_dim, d->n_pairs, d->interleaved, 1, 1, {}, 1, 1, 0, 0, d->magnitude, d->eps};
    hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();
    const int64_t blocks = d->n_rows > 0 ? enqueue<true>(a, d, st) : 0;
    if (dweight || dweight2)
        hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((d->head_dim + 7) / 8), x2 ? 2 : 1), dim3(256), 0, st, a.partial[0], a.partial[1],
                           (int)(blocks * a.shares[0]), (int)(blocks * a.shares[1]), d->head_dim, dweight, dweight2);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
