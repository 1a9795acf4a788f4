// Rotary positions.  A call reads and writes its tensors once and computes next to nothing, so memory bounds it: a workgroup takes a
// few rows, puts the cosines and sines of their pairs into LDS once, and streams all heads past them.  32768 rows of two tensors of 16 heads of
// 64 in bf16, 268 MB: 55 us, 4.9 TB/s (a copy reaches 5.1); 64 rows of 40 heads of 128: 3.4 us.
#include <math.h>

#include "internal.h"
#include "rotary.h"

typedef __bf16 bf16;

namespace {

struct RotaryArgs {
    const void* x[2];
    void* out[2];
    ps_strides xs[2], os[2];
    const int32_t* positions;
    const float* frequencies;
    int64_t n_rows;
    int32_t heads, heads2, head_dim, n_pairs, interleaved, rows, heads_each;   // rows, heads of a workgroup
    float magnitude, sign;
    int32_t in_place[2];
};

constexpr int TABLE = 2048;            // pairs of a workgroup's rows, at most

// VEC elements at a time; BATCH such units of a thread on their way together, the first of them while the table is made (8192 rows of 40 heads of
// 128, half of them turning, in bf16: one after the other behind the table 36 us, 2 30.5, 4 30; 16384 fp32 rows of 18 heads of 128 51, 50.5, 54).
template <typename T, int VEC>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
    __shared__ float2 table[TABLE];
    constexpr bool WIDE = VEC > 1;
    constexpr int BATCH = 2;
    struct Piece { T v[VEC]; };          // (moved whole at any address)
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = (int)min((int64_t)a.rows, a.n_rows - row0), n = a.n_pairs;
    const int head0 = blockIdx.y * a.heads_each, heads = min(a.heads_each, a.heads + a.heads2 - head0);
    // units of a head: its turning pairs (VEC of them in halves, VEC / 2 or one interleaved), then what is copied, VEC a unit
    const int turning = a.interleaved ? (WIDE ? 2 * n / VEC : n) : n / VEC, units = turning + (a.head_dim - 2 * n) / VEC, all = rows * heads * units;
    constexpr int COPIED = -1, NONE = -2;
    Piece p[BATCH], q[BATCH];
    T* out[BATCH];
    int at[BATCH];                     // in the table
    auto fetch = [&](int first) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const unsigned i = first + 256 * b, head = i / (unsigned)units, unit = i - head * units, r = head / (unsigned)heads;
            const int h = head0 + (int)(head - r * heads), second = h >= a.heads, hh = second ? h - a.heads : h;
            at[b] = NONE;
            if ((int)i >= all) continue;
            const int64_t row = row0 + r;
            const T* x = (const T*)a.x[second] + row * a.xs[second].row + hh * a.xs[second].head;
            out[b] = (T*)a.out[second] + row * a.os[second].row + hh * a.os[second].head;
            int e, other;
            if ((int)unit >= turning) {
                if (a.in_place[second]) continue;
                at[b] = COPIED;
                e = other = 2 * n + ((int)unit - turning) * VEC;
            } else if (!a.interleaved) {
                at[b] = r * n + unit * VEC;
                e = unit * VEC;
                other = n + e;
            } else {
                at[b] = r * n + unit * (WIDE ? VEC / 2 : 1);
                e = unit * (WIDE ? VEC : 2);
                other = WIDE ? e : e + 1;
            }
            out[b] += e;
            p[b] = *(const Piece*)(x + e);
            if (other != e) q[b] = *(const Piece*)(x + other);
        }
    };
    auto turn = [&] {
        const int apart = a.interleaved ? 1 : n;                          // the pair's other element (not WIDE interleaved)
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (at[b] == NONE) continue;
            const float2* cs = table + at[b];
            if (at[b] == COPIED) {
            } else if (WIDE && a.interleaved) {
                if constexpr (WIDE) {
#pragma unroll
                    for (int j = 0; j < VEC; j += 2) {
                        const float u = (float)p[b].v[j], v = (float)p[b].v[j + 1];
                        const float2 w = cs[j / 2];
                        p[b].v[j] = (T)fmaf(-v, w.y, u * w.x);
                        p[b].v[j + 1] = (T)fmaf(v, w.x, u * w.y);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float u = (float)p[b].v[j], v = (float)q[b].v[j];
                    const float2 w = cs[j];
                    p[b].v[j] = (T)fmaf(-v, w.y, u * w.x);
                    q[b].v[j] = (T)fmaf(v, w.x, u * w.y);
                }
                *(Piece*)(out[b] + apart) = q[b];
            }
            *(Piece*)out[b] = p[b];
        }
    };
    fetch(threadIdx.x);
    for (int i = threadIdx.x; i < rows * n; i += 256) {
        const float2 w = turn_of(a.positions[row0 + i / n], a.frequencies[i % n]);
        table[i] = make_float2(w.x * a.magnitude, w.y * a.magnitude * a.sign);
    }
    __syncthreads();
    turn();
    for (int i = threadIdx.x + 256 * BATCH; i - (int)threadIdx.x < all; i += 256 * BATCH) {
        fetch(i);
        turn();
    }
}

bool strides_ok(const ps_strides& s, bool written, int heads, int head_dim, int64_t rows) {
    return s.row >= 0 && s.head >= 0 && (!written || strides_apart(s, rows, heads, head_dim));
}

template <typename T>
void launch(const RotaryArgs& a, int bytes, dim3 grid, hipStream_t st) {
    constexpr int ES = sizeof(T);
    if (bytes == 16)
        hipLaunchKernelGGL((rotary_kernel<T, 16 / ES>), grid, dim3(256), 0, st, a);
    else if (bytes == 8)
        hipLaunchKernelGGL((rotary_kernel<T, 8 / ES>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((rotary_kernel<T, 1>), grid, dim3(256), 0, st, a);
}

}  // namespace

extern "C" int ps_rotary(const ps_rotary_desc* d, const void* x, void* out, const void* x2, void* out2, const int32_t* positions,
                         const float* frequencies, void* hip_stream) {
    if (!d || (d->dtype != 0 && d->dtype != 1) || d->head_dim < 1 || d->n_pairs < 0 || (int64_t)2 * d->n_pairs > d->head_dim ||
        d->heads < 1 || d->heads2 < 0 || d->n_rows < 0 || (d->interleaved & ~1) || (d->inverse & ~1) || !x2 != !out2 || (d->heads2 > 0) != (x2 != nullptr))
        return PS_EINVAL;
    // (a workgroup counts the elements of its rows, 8 at most, in 32 bits)
    if (d->head_dim > 4096 || ((int64_t)d->heads + d->heads2) * d->head_dim > 1 << 27 || d->n_rows > INT32_MAX) return PS_EUNSUPPORTED;
    if (!strides_ok(d->x, false, d->heads, d->head_dim, d->n_rows) || !strides_ok(d->out, true, d->heads, d->head_dim, d->n_rows) ||
        (x2 && (!strides_ok(d->x2, false, d->heads2, d->head_dim, d->n_rows) || !strides_ok(d->out2, true, d->heads2, d->head_dim, d->n_rows))))
        return PS_EINVAL;
    if (d->n_rows == 0) return PS_OK;
    if (!x || !out || (d->n_pairs > 0 && (!positions || !frequencies))) return PS_EINVAL;
    const size_t es = d->dtype == 1 ? 2 : 4;
    if (((uintptr_t)x | (uintptr_t)out | (uintptr_t)x2 | (uintptr_t)out2) % es != 0) return PS_EINVAL;
    RotaryArgs a = {{x, x2}, {out, out2}, {d->x, d->x2}, {d->out, d->out2}, positions, frequencies, d->n_rows, d->heads, d->heads2,
                    d->head_dim, d->n_pairs, d->interleaved, 1, 1, d->magnitude, d->inverse ? -1.f : 1.f, {x == out, x2 == out2}};
    if ((x == out && (d->x.row != d->out.row || d->x.head != d->out.head)) || (x2 && x2 == out2 && (d->x2.row != d->out2.row || d->x2.head != d->out2.head)))
        return PS_EINVAL;
    // 16 bytes at a time, or 8, where the pieces of a head allow it, at whatever addresses (8000 rows of 16 heads of 80, 40 of them in two halves,
    // bf16: 8 bytes 13 us, one element 32; 16384 rows of 16 heads of 64 that start an odd element apart 14, one element 35)
    const uintptr_t pieces = (uintptr_t)(d->head_dim | (d->interleaved ? 2 * d->n_pairs : d->n_pairs)) * es;
    const int bytes = pieces % 16 == 0 ? 16 : pieces % 8 == 0 ? 8 : 1;
    // Rows of a workgroup: a pair a thread for the table; heads are shared out where rows alone do not fill the chip.
    const int all = d->heads + d->heads2;
    const int64_t most = d->n_pairs > 0 ? (d->n_pairs >= 256 ? 1 : 256 / d->n_pairs) : 8;
    a.rows = (int32_t)(most < 8 ? most : 8);
    while (a.rows > 1 && (d->n_rows + a.rows - 1) / a.rows < 1024) a.rows /= 2;
    const int64_t blocks = (d->n_rows + a.rows - 1) / a.rows;
    const int shares = (int)(blocks >= 512 ? 1 : 512 / blocks < all ? 512 / blocks : all);
    a.heads_each = (all + shares - 1) / shares;
    (void)hipGetLastError();
    const int64_t per = 1 << 22;       // (a grid holds fewer than 2^32 threads)
    for (int64_t b0 = 0; b0 < blocks; b0 += per) {
        RotaryArgs b = a;
        const int64_t first = b0 * a.rows;
        for (int i = 0; i < 2; ++i) {
            if (!b.x[i]) continue;
            b.x[i] = (const char*)a.x[i] + (size_t)first * a.xs[i].row * es;
            b.out[i] = (char*)a.out[i] + (size_t)first * a.os[i].row * es;
        }
        if (positions) b.positions = positions + first;
        b.n_rows = d->n_rows - first;
        const dim3 grid((unsigned)(blocks - b0 < per ? blocks - b0 : per), (unsigned)((all + a.heads_each - 1) / a.heads_each));
        d->dtype == 1 ? launch<bf16>(b, bytes, grid, (hipStream_t)hip_stream) : launch<float>(b, bytes, grid, (hipStream_t)hip_stream);
    }
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

extern "C" int ps_rotary_frequencies(int32_t n, double base, int scaling, double factor, int32_t trained_len, double slow, double fast,
                                     float* f) {
    if (n < 1 || !f || !(base > 0) || isinf(base) || scaling < PS_ROTARY_PLAIN || scaling > PS_ROTARY_PARTS) return PS_EINVAL;
    if (scaling != PS_ROTARY_PLAIN && (!(factor > 0) || isinf(factor))) return PS_EINVAL;
    if (scaling == PS_ROTARY_BASE && n < 2) return PS_EINVAL;
    if (scaling == PS_ROTARY_PARTS && (trained_len < 1 || !(slow >= 0) || !(fast > slow))) return PS_EINVAL;
    if (scaling == PS_ROTARY_BASE) base *= pow(factor, (double)n / (n - 1));
    for (int32_t i = 0; i < n; ++i) {
        double w = pow(base, -(double)i / n);
        if (scaling == PS_ROTARY_LINEAR) w /= factor;
        if (scaling == PS_ROTARY_PARTS) {
            const double turns = trained_len * w * 0.15915494309189533577;
            const double kept = turns <= slow ? 0.0 : turns >= fast ? 1.0 : (turns - slow) / (fast - slow);
            w = w / factor * (1.0 - kept) + w * kept;
        }
        f[i] = (float)w;
    }
    return PS_OK;
}
