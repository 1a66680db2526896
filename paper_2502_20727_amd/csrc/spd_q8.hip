// Rows to 8-bit integers, and the product of such rows with packed 8-bit weights, for gfx950.
#include <type_traits>

#include "spd_q8_internal.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------
// Rows to 8 bits.  One workgroup per row.
// ------------------------------------------------------------------------------------------
enum RowKind { ROW_NORM, ROW_PLAIN, ROW_SWIGLU };

struct RowArgs {
    const void *x, *add;
    const float *gain;
    void *sum;
    int8_t *codes;
    float *scales;
    int64_t ld_x, ld_add, ld_sum, ld_codes;
    int n;
    float eps;
};

template <class T, int KIND, bool ADD>
struct RowSource {
    const T *x, *add;
    const float *gain;
    int n;
    __device__ __forceinline__ float sum(int i) const {       // the norm's summand
        float s = (float)x[i];
        if constexpr (ADD) s += (float)add[i];
        return s;
    }
    __device__ __forceinline__ float value(int i) const {     // up to the norm's factor
        if constexpr (KIND == ROW_NORM) return sum(i) * gain[i];
        else if constexpr (KIND == ROW_PLAIN) return (float)x[i];
        else {
            const float g = (float)x[i], u = (float)x[n + i];
            return g / (1.f + __builtin_expf(-g)) * u;
        }
    }
};

template <class T, int KIND, bool ADD>
__global__ void __launch_bounds__(256) k_rows_q8(RowArgs A) {
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    RowSource<T, KIND, ADD> src;
    src.x = (const T *)A.x + row * A.ld_x;
    src.add = ADD ? (const T *)A.add + row * A.ld_add : nullptr;
    src.gain = A.gain;
    src.n = A.n;
    float ss = 0.f, most = 0.f;
    bool fine = true;
    for (int i = threadIdx.x; i < A.n; i += 256) {
        const float v = src.value(i);
        if constexpr (KIND == ROW_NORM) {
            const float s = src.sum(i);
            ss += s * s;
        }
        fine = fine && fabsf(v) <= 3.402823466e38f;
        most = fmaxf(most, fabsf(v));
    }
    if (!fine) most = __builtin_inff();
    __shared__ float sh[2][4];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        ss += __shfl_xor(ss, d, 64);
        most = fmaxf(most, __shfl_xor(most, d, 64));
    }
    if (lane == 0) {
        sh[0][wave] = ss;
        sh[1][wave] = most;
    }
    __syncthreads();
    ss = (sh[0][0] + sh[0][1]) + (sh[0][2] + sh[0][3]);
    most = fmaxf(fmaxf(sh[1][0], sh[1][1]), fmaxf(sh[1][2], sh[1][3]));
    const float factor = KIND == ROW_NORM ? 1.f / sqrtf(ss / (float)A.n + A.eps) : 1.f;
    const bool ok = most < __builtin_inff() && (KIND != ROW_NORM || (ss < __builtin_inff()));
    const float a = fmaxf(most * factor, 0x1p-90f), up = 127.f / a;
    if (threadIdx.x == 0) A.scales[row] = ok ? a / 127.f : __builtin_nanf("");
    int8_t *codes = A.codes + row * A.ld_codes;
    for (int i = threadIdx.x; i < A.n; i += 256) {
        const float c = rintf(src.value(i) * factor * up);
        codes[i] = ok ? (int8_t)(int)c : (int8_t)0;
        if constexpr (KIND == ROW_NORM)
            if (A.sum) ((T *)A.sum)[row * A.ld_sum + i] = (T)src.sum(i);
    }
}

template <class T>
hipError_t launch_rows(int kind, int rows, const RowArgs &A, hipStream_t s) {
    const dim3 grid(rows), block(256);
    if (kind == ROW_NORM) {
        if (A.add) hipLaunchKernelGGL((k_rows_q8<T, ROW_NORM, true>), grid, block, 0, s, A);
        else hipLaunchKernelGGL((k_rows_q8<T, ROW_NORM, false>), grid, block, 0, s, A);
    } else if (kind == ROW_PLAIN) hipLaunchKernelGGL((k_rows_q8<T, ROW_PLAIN, false>), grid, block, 0, s, A);
    else hipLaunchKernelGGL((k_rows_q8<T, ROW_SWIGLU, false>), grid, block, 0, s, A);
    return hipGetLastError();
}

int rows_impl(int kind, int32_t dtype, int32_t rows, const RowArgs &A, void *stream) {
    const int64_t width = kind == ROW_SWIGLU ? 2 * (int64_t)A.n : A.n;
    if (dtype != SPD_F32 && dtype != SPD_BF16 && dtype != SPD_F16) return SPD_EINVAL;
    if (rows < 0 || A.n < 0 || A.n > (1 << 30)) return SPD_EINVAL;
    if (!A.x || !A.codes || !A.scales || A.ld_x < width || A.ld_codes < A.n) return SPD_EINVAL;
    if ((kind == ROW_NORM && !A.gain) || (A.add && A.ld_add < A.n) || (A.sum && A.ld_sum < A.n)) return SPD_EINVAL;
    const uintptr_t es = dtype == SPD_F32 ? 4 : 2;
    if ((uintptr_t)A.x % es || (uintptr_t)A.add % es || (uintptr_t)A.sum % es || (uintptr_t)A.scales % 4 || (uintptr_t)A.gain % 4) return SPD_EINVAL;
    if ((A.sum == A.x && A.ld_sum != A.ld_x) || (A.sum && A.sum == A.add && A.ld_sum != A.ld_add)) return SPD_EINVAL;
    if (rows == 0 || A.n == 0) return SPD_OK;
    (void)hipGetLastError();
    hipStream_t s = (hipStream_t)stream;
    SPD_HIP(dtype == SPD_F32 ? launch_rows<float>(kind, rows, A, s)
                             : dtype == SPD_BF16 ? launch_rows<__bf16>(kind, rows, A, s) : launch_rows<_Float16>(kind, rows, A, s));
    return SPD_OK;
}

// ------------------------------------------------------------------------------------------
// Product.  Weights are the first MFMA operand, rows the second: a lane holds four consecutive output columns of one row.
// ------------------------------------------------------------------------------------------
struct Q8Args {
    const int8_t *codes;
    const float *scales;
    const char *packed;
    const void *add;
    void *out;
    int64_t ld_codes, ld_add, ld_out;
    int rows, K, N, KT, NT;
};

// (a place past the matrix: nothing)
template <class T>
__device__ __forceinline__ void q8_store(const Q8Args &A, int m, int n, i32x4 acc) {
    if (m >= A.rows || n >= A.N) return;
    const float sm = A.scales[m];
    const float *wsc = (const float *)A.packed;
    T *out = (T *)A.out + m * A.ld_out;
    const T *add = A.add ? (const T *)A.add + m * A.ld_add : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < A.N) {
            float v = (float)acc[i] * sm * wsc[n + i];
            if (add) v += (float)add[n + i];
            out[n + i] = (T)v;
        }
}

// one wave: 64 columns x 64 rows, operands straight from memory
template <class T>
__global__ void __launch_bounds__(256) k_q8_tile(Q8Args A) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nt0 = (blockIdx.x * 4 + wave) * 4, m0 = blockIdx.y * 64;
    if (nt0 >= A.NT) return;
    const int r = lane & 15, g = lane >> 4;
    const char *w[4];
    const int8_t *x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int nt = nt0 + i < A.NT ? nt0 + i : A.NT - 1, m = m0 + 16 * i + r;
        w[i] = A.packed + spd_q8_weights_at(A.N) + (size_t)nt * A.KT * 1024 + lane * 16;
        x[i] = A.codes + (int64_t)(m < A.rows ? m : A.rows - 1) * A.ld_codes;
    }
    i32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
    for (int kt = 0; kt < A.KT; ++kt) {
        const int k = kt * 64 + 16 * g < A.K ? kt * 64 + 16 * g : 0;      // past K: anything, the weights are zero there
        i32x4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = *(const i32x4 *)(w[i] + (size_t)kt * 1024);
            b[i] = *(const i32x4 *)(x[i] + k);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) q8_store<T>(A, m0 + 16 * j + r, (nt0 + i) * 16 + 4 * g, acc[i][j]);
}

template <class T>
hipError_t launch_product(const Q8Args &A, hipStream_t s) {
    hipLaunchKernelGGL((k_q8_tile<T>), dim3((A.NT + 15) / 16, (A.rows + 63) / 64), dim3(256), 0, s, A);
    return hipGetLastError();
}

}  // namespace

extern "C" {

int spd_q8_norm(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, const void *add, int64_t ld_add, const float *gain,
                float eps, void *sum, int64_t ld_sum, int8_t *codes, int64_t ld_codes, float *scales, void *stream) {
    if (!(eps >= 0.f)) return SPD_EINVAL;
    return rows_impl(ROW_NORM, dtype, rows, RowArgs{x, add, gain, sum, codes, scales, ld_x, ld_add, ld_sum, ld_codes, n, eps}, stream);
}

int spd_q8_rows(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, int8_t *codes, int64_t ld_codes, float *scales,
                void *stream) {
    return rows_impl(ROW_PLAIN, dtype, rows, RowArgs{x, nullptr, nullptr, nullptr, codes, scales, ld_x, 0, 0, ld_codes, n, 0.f}, stream);
}

int spd_q8_swiglu(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, int8_t *codes, int64_t ld_codes, float *scales,
                  void *stream) {
    return rows_impl(ROW_SWIGLU, dtype, rows, RowArgs{x, nullptr, nullptr, nullptr, codes, scales, ld_x, 0, 0, ld_codes, n, 0.f}, stream);
}

size_t spd_q8_matmul_workspace(int32_t rows, int32_t K, int32_t N) {
    (void)rows;
    (void)K;
    (void)N;
    return 0;
}

int spd_q8_matmul(int32_t rows, int32_t K, int32_t N, const int8_t *codes, int64_t ld_codes, const float *scales, const void *packed,
                  int32_t out_dtype, const void *add, int64_t ld_add, void *out, int64_t ld_out, void *workspace, void *stream) {
    if (rows < 0 || !spd_q8_weight_bytes(K, N)) return SPD_EINVAL;
    if (out_dtype != SPD_F32 && out_dtype != SPD_BF16 && out_dtype != SPD_F16) return SPD_EINVAL;
    if (!codes || !scales || !packed || !out || ((uintptr_t)codes & 15) || ((uintptr_t)packed & 255) || ((uintptr_t)scales & 3)) return SPD_EINVAL;
    if (ld_codes % 16 || ld_codes < (K + 15) / 16 * 16 || ld_out < N || (add && ld_add < N)) return SPD_EINVAL;
    const uintptr_t es = out_dtype == SPD_F32 ? 4 : 2;
    if ((uintptr_t)out % es || (uintptr_t)add % es) return SPD_EINVAL;
    if (add == out && ld_add != ld_out) return SPD_EINVAL;
    if (spd_q8_matmul_workspace(rows, K, N) && (!workspace || ((uintptr_t)workspace & 255))) return SPD_EINVAL;
    if (rows == 0) return SPD_OK;
    (void)hipGetLastError();
    const Q8Args A{codes, scales, (const char *)packed, add, out, ld_codes, ld_add, ld_out, rows, K, N, spd_q8_ktiles(K), spd_q8_ntiles(N)};
    hipStream_t s = (hipStream_t)stream;
    SPD_HIP(out_dtype == SPD_F32 ? launch_product<float>(A, s) : out_dtype == SPD_BF16 ? launch_product<__bf16>(A, s) : launch_product<_Float16>(A, s));
    return SPD_OK;
}

}  // extern "C"
