// Dropout with bias and residual, and its gradients.  The mask is drawn where it is used (Philox4x32-10, Salmon et al. 2011, "Parallel
// random numbers: as easy as 1, 2, 3"): one draw of 128 bits is 16 bits for each of the 8 neighbours that a thread holds.
#include <math.h>

#include "device_util.h"
#include "internal.h"

typedef __bf16 bf16;

namespace {

// The four words of the counter (group, row, offset) under the key `seed`.
__device__ __forceinline__ uint4 draw(uint32_t group, uint32_t row, uint64_t seed, uint64_t offset) {
    uint4 c = make_uint4(group, row, (uint32_t)offset, (uint32_t)(offset >> 32));
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}
__device__ __forceinline__ uint32_t piece(const uint4& u, int i) {
    const uint32_t w = i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w;
    return i & 1 ? w >> 16 : w & 0xffffu;
}

template <typename T>
struct alignas(16) Eight {
    T v[8];
    // n of them; the others are zero.  WIDE: always 8, at multiples of 16 bytes.  Else 8 go whole at whatever address they have (32768 x 767 of bf16,
    // forwards 83 us an element at a time, 31.5 so), and the last of a row one by one.  (On rows that are WIDE the other way takes 5 to 15 % more.)
    template <bool WIDE>
    __device__ __forceinline__ void load(const T* p, int n) {
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(v) / 16; ++i) ((uint4*)v)[i] = ((const uint4*)p)[i];
        } else if (n == 8) {
            __builtin_memcpy(v, p, sizeof(v));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0.f;
        }
    }
    template <bool WIDE>
    __device__ __forceinline__ void store(T* p, int n) const {
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(v) / 16; ++i) ((uint4*)p)[i] = ((const uint4*)v)[i];
        } else if (n == 8) {
            __builtin_memcpy(p, v, sizeof(v));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = v[i];
        }
    }
};

struct DropoutArgs {
    const void *x, *bias, *residual;
    void* out;
    const int64_t* rng;
    float* sums;                       // [row blocks][groups * 8]
    int64_t ld_x, ld_residual, ld_out, rows;
    int32_t cols, groups, row_step;    // groups of 8 columns; rows of a row block
    uint32_t lost;
    float by;
};

// out = residual + keep ? (x + bias) / (1 - p) : 0.  Each value passes once, so it is bound by bytes: 65536 x 1024 of bf16 with bias and residual
// (403 MB) take 78.5 us, 5.1 TB/s, what a copy reaches; the ten rounds of the draw for 8 values fit under it.  Sums in fp32, one rounding to T.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
    const uint64_t seed = (uint64_t)a.rng[0], offset = (uint64_t)a.rng[1];
    const int64_t all = a.rows * a.groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / a.groups;
        const int g = (int)(i - row * a.groups), col = 8 * g, n = min(8, a.cols - col);
        Eight<T> x, b, r;
        x.template load<WIDE>((const T*)a.x + row * a.ld_x + col, n);
        if (a.bias) b.template load<WIDE>((const T*)a.bias + col, n);
        if (a.residual) r.template load<WIDE>((const T*)a.residual + row * a.ld_residual + col, n);
        const uint4 u = draw((uint32_t)g, (uint32_t)row, seed, offset);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y = (float)x.v[j];
            if (a.bias) y += (float)b.v[j];
            y = piece(u, j) >= a.lost ? y * a.by : 0.f;
            if (a.residual) y += (float)r.v[j];
            x.v[j] = (T)y;
        }
        x.template store<WIDE>((T*)a.out + row * a.ld_out + col, n);
    }
}

// dx, and the sums of a row block's columns: 2^log groups of columns to a workgroup, the others of its threads share its rows.  32 groups
// where there are several row blocks, two where there is one: 128 threads then share its rows, a row in pieces of 32 or 64 bytes (577 rows of
// 128 in fp32 with 1, 2, 4, 8 groups: 4.5, 4.4, 5.5, 7.7 us).  Bound by bytes at many rows: 65536 x 1024 of bf16 at 5.5 TB/s of dout and dx.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void dropout_sums_kernel(DropoutArgs a, int log, float* dbias) {
    __shared__ float part[256][8];
    const uint64_t seed = (uint64_t)a.rng[0], offset = (uint64_t)a.rng[1];
    const int lanes = 256 >> log, g = blockIdx.x * (1 << log) + (threadIdx.x & ((1 << log) - 1)), lane = threadIdx.x >> log;
    const int64_t r0 = (int64_t)blockIdx.y * a.row_step, r1 = min(a.rows, r0 + a.row_step);
    const int col = 8 * g, n = min(8, a.cols - col);
    float s[8] = {};
    if (g < a.groups)
        for (int64_t row = r0 + lane; row < r1; row += lanes) {
            Eight<T> x;
            x.template load<WIDE>((const T*)a.x + row * a.ld_x + col, n);
            const uint4 u = draw((uint32_t)g, (uint32_t)row, seed, offset);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = piece(u, j) >= a.lost ? (float)x.v[j] * a.by : 0.f;
                s[j] += y;
                x.v[j] = (T)y;
            }
            x.template store<WIDE>((T*)a.out + row * a.ld_out + col, n);
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) part[threadIdx.x][j] = s[j];
    for (int half = lanes / 2; half > 0; half /= 2) {
        __syncthreads();
        if (lane < half)
#pragma unroll
            for (int j = 0; j < 8; ++j) part[threadIdx.x][j] += part[threadIdx.x + (half << log)][j];
    }
    if (lane == 0 && g < a.groups) {
        const bool last = gridDim.y == 1;                                 // one row block: these are the gradients
        float* to = last ? dbias + col : a.sums + ((int64_t)blockIdx.y * a.groups + g) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!last || j < n) to[j] = part[threadIdx.x][j];
    }
}

// 8 columns a workgroup, 32 shares of the 256 row blocks at most: eight loads of a thread, at once (32 columns and 8 shares 11.2 us of
// 1024 columns).
__global__ __launch_bounds__(256) void bias_kernel(const float* sums, int blocks, int stride, int cols, float* dbias) {
    __shared__ float part[32][8];
    const int c = blockIdx.x * 8 + (threadIdx.x & 7), share = threadIdx.x >> 3;
    float s = 0.f;
    if (c < cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = share + 32 * i;
            if (b < blocks) s += sums[(int64_t)b * stride + c];
        }
    }
    part[share][threadIdx.x & 7] = s;
    for (int half = 16; half > 0; half /= 2) {
        __syncthreads();
        if (share < half) part[share][threadIdx.x & 7] += part[share + half][threadIdx.x & 7];
    }
    if (share == 0 && c < cols) dbias[c] = part[0][threadIdx.x];
}

// Rows of a row block.  Up to 768 rows: one block, whose sums are the gradients, without a second launch (128 columns of fp32: 64 rows
// 5.2 -> 3.2 us, 577 rows 5.3 -> 4.4, 1024 would take 5.2 for 5.4; 2048 columns: 577 rows 6.8 -> 5.4, 2048 would take 14.7 for 10.2).
// Else 256 blocks at most, so that the second sum is short, of 32 rows at least.
constexpr int ONE_BLOCK = 768;
int32_t row_step(int64_t rows) {
    if (rows <= ONE_BLOCK) return rows < 1 ? 1 : (int32_t)rows;
    const int64_t step = (rows + 255) / 256;
    return (int32_t)(step < 32 ? 32 : step);
}

bool refused(int64_t rows, int32_t cols, float p, int32_t dtype, int& code) {
    code = PS_EINVAL;
    if (rows < 0 || cols < 0 || !(p >= 0.f && p <= 1.f) || (dtype != 0 && dtype != 1)) return true;
    code = PS_EUNSUPPORTED;
    if (rows > INT32_MAX || cols > (1 << 20)) return true;
    code = PS_OK;
    return false;
}

bool aligned(const void* p, int64_t ld, int32_t dtype) { return (uintptr_t)p % 16 == 0 && ld % (dtype == 1 ? 8 : 4) == 0; }

void set_rate(DropoutArgs& a, float p) {
    a.lost = (uint32_t)rintf(p * 65536.f);
    a.by = a.lost < 65536 ? 65536.f / (float)(65536 - a.lost) : 0.f;
}

template <typename T>
void launch(const DropoutArgs& a, bool wide, hipStream_t st) {
    const int64_t all = a.rows * a.groups, blocks = (all + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22));
    if (wide)
        hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, st, a);
}

template <typename T>
void launch_sums(const DropoutArgs& a, bool wide, float* dbias, hipStream_t st) {
    int log = 0;
    while ((1 << log) < a.groups && log < (a.row_step < a.rows ? 5 : 1)) ++log;
    const int blocks = (int)((a.rows + a.row_step - 1) / a.row_step);
    const dim3 grid((unsigned)((a.groups + (1 << log) - 1) >> log), (unsigned)blocks);
    if (wide)
        hipLaunchKernelGGL((dropout_sums_kernel<T, true>), grid, dim3(256), 0, st, a, log, dbias);
    else
        hipLaunchKernelGGL((dropout_sums_kernel<T, false>), grid, dim3(256), 0, st, a, log, dbias);
    if (blocks > 1)
        hipLaunchKernelGGL(bias_kernel, dim3((unsigned)((a.cols + 7) / 8)), dim3(256), 0, st, a.sums, blocks, a.groups * 8, a.cols, dbias);
}

}  // namespace

extern "C" int ps_dropout_forward(const void* x, int64_t ld_x, const void* bias, const void* residual, int64_t ld_residual,
                                  const int64_t* rng, float p, int32_t dtype, int64_t rows, int32_t cols, void* out, int64_t ld_out,
                                  void* hip_stream) {
    int code;
    if (refused(rows, cols, p, dtype, code)) return code;
    if (rows == 0 || cols == 0) return PS_OK;
    if (!x || !rng || !out || ld_x < cols || ld_out < cols || (residual && ld_residual < cols)) return PS_EINVAL;
    const uintptr_t es = dtype == 1 ? 2 : 4;
    if (((uintptr_t)x | (uintptr_t)out | (uintptr_t)bias | (uintptr_t)residual) % es != 0 || (uintptr_t)rng % 8 != 0) return PS_EINVAL;
    if ((out == x && ld_out != ld_x) || (out == residual && ld_out != ld_residual)) return PS_EINVAL;
    DropoutArgs a = {x, bias, residual, out, rng, nullptr, ld_x, ld_residual, ld_out, rows, cols, (cols + 7) / 8, 0, 0, 0.f};
    set_rate(a, p);
    const bool wide = cols % 8 == 0 && aligned(x, ld_x, dtype) && aligned(out, ld_out, dtype) && aligned(bias, 0, dtype) &&
                      (!residual || aligned(residual, ld_residual, dtype));
    (void)hipGetLastError();
    dtype == 1 ? launch<bf16>(a, wide, (hipStream_t)hip_stream) : launch<float>(a, wide, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}

extern "C" size_t ps_dropout_workspace_bytes(int64_t rows, int32_t cols) {
    int code;
    if (refused(rows, cols, 0.f, 0, code)) return 0;
    const int64_t blocks = rows == 0 ? 1 : (rows + row_step(rows) - 1) / row_step(rows);
    return align_up(sizeof(float) * (size_t)blocks * (size_t)((cols + 7) / 8 * 8), 256);
}

extern "C" int ps_dropout_backward(const void* dout, int64_t ld_dout, const int64_t* rng, float p, int32_t dtype, int64_t rows,
                                   int32_t cols, void* dx, int64_t ld_dx, float* dbias, void* workspace, size_t workspace_bytes,
                                   void* hip_stream) {
    int code;
    if (refused(rows, cols, p, dtype, code)) return code;
    if (cols == 0 || (rows == 0 && !dbias)) return PS_OK;
    if (rows > 0 && (!dout || !rng || !dx || ld_dout < cols || ld_dx < cols || (dx == dout && ld_dx != ld_dout))) return PS_EINVAL;
    const uintptr_t es = dtype == 1 ? 2 : 4;
    if (((uintptr_t)dout | (uintptr_t)dx) % es != 0 || (uintptr_t)rng % 8 != 0 || (uintptr_t)dbias % 4 != 0) return PS_EINVAL;
    if (dbias && (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < ps_dropout_workspace_bytes(rows, cols))) return PS_EWORKSPACE;
    hipStream_t st = (hipStream_t)hip_stream;
    DropoutArgs a = {dout, nullptr, nullptr, dx, rng, (float*)workspace, ld_dout, 0, ld_dx, rows, cols, (cols + 7) / 8, row_step(rows), 0, 0.f};
    set_rate(a, p);
    const bool wide = cols % 8 == 0 && aligned(dout, ld_dout, dtype) && aligned(dx, ld_dx, dtype);
    (void)hipGetLastError();
    if (!dbias)
        dtype == 1 ? launch<bf16>(a, wide, st) : launch<float>(a, wide, st);
    else if (rows == 0)
        hipLaunchKernelGGL(bias_kernel, dim3((unsigned)((cols + 7) / 8)), dim3(256), 0, st, a.sums, 0, 0, cols, dbias);
    else
        dtype == 1 ? launch_sums<bf16>(a, wide, dbias, st) : launch_sums<float>(a, wide, dbias, st);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_EHIP;
}
