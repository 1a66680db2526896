// Rows to 8-bit integers, and the product of such rows with packed 8-bit weights, for gfx950.
#include <mutex>
#include <type_traits>

#include "spd_q8_internal.h"
#include "spd_testing.h"

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

// A thread's sum of squares.  Squares of fp32 values leave fp32 on both sides: those that may are added up once more, of values 2^80 times larger and
// smaller.  A row whose mean is 1e-30 at most has no others (a row's length is below 2^30), and in one whose mean is 1e38 the others do not count.
struct Squares {
    float plain = 0.f, of_small = 0.f, of_large = 0.f;
    // (a call of the norm of 16 rows of 8192 takes 0.03 us more than with the plain sum alone, of 8192 rows 0.4 of 87; without the branch 0.1 and 1.1)
    template <int N>
    __device__ __forceinline__ void add(const float (&s)[N]) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) t += s[i] * s[i];
        plain += t;
        if (N > 1 && t > 1e-20f && t < 1e30f) return;      // (one by itself is not worth a branch)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float up = s[i] * 0x1p80f, down = s[i] * 0x1p-80f;
            of_small += up * up;
            of_large += down * down;
        }
    }
};
// 1 / sqrt(mean + eps) of a row, `ss` the sum of all threads' plain sums.  The others are joined, by way of `sh`, only where they are called for,
// which all of a workgroup see alike.
__device__ __forceinline__ float norm_factor(float ss, const Squares &q, int n, float eps, float *sh) {
    const float mean = ss / (float)n + eps;
    if (mean > 1e-30f && mean < 1e38f) return 1.f / sqrtf(mean);
    const bool small = mean <= 1e-30f;
    float t = small ? q.of_small : q.of_large;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) t += __shfl_xor(t, d, 64);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = t;
    __syncthreads();
    t = 0.f;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) t += sh[w];
    return small ? 0x1p80f / sqrtf(t / (float)n + eps * 0x1p80f * 0x1p80f) : 0x1p-80f / sqrtf(t / (float)n + eps * 0x1p-80f * 0x1p-80f);
}

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
    Squares squares;
    float most = 0.f;
    bool fine = true;
    for (int i = threadIdx.x; i < A.n; i += 256) {
        const float v = src.value(i);
        if constexpr (KIND == ROW_NORM) {
            const float s[1] = {src.sum(i)};
            squares.add(s);
        }
        fine = fine && fabsf(v) <= 3.402823466e38f;
        most = fmaxf(most, fabsf(v));
    }
    if (!fine) most = __builtin_inff();
    float ss = squares.plain;
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
    float factor = 1.f;
    if constexpr (KIND == ROW_NORM) {
        __shared__ float far[4];
        factor = norm_factor(ss, squares, A.n, A.eps, far);
    }
    // (a row of zeros without an eps has a factor of infinity, and 0 times it is NaN)
    const bool ok = most < __builtin_inff() && (KIND != ROW_NORM || most * factor < __builtin_inff());
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

// The same with rows in registers (up to 16384 elements): eight per thread and chunk.  Bound by what is read and written: 8192 rows of
// 8192 in 16 bits with a summand, 85 us (470 MB: 5.5 TB/s), as they are 36.5 (201 MB: 5.5).  SwiGLU is bound by its vector instructions, 37 an
// element, most of them of the exponential and the division, which fill the SIMDs: 8192 rows of 3584 35 us (147 MB: 4.2 TB/s), 2048 13.5.  Longer rows are read twice, one workgroup of 256 threads each: 2048 SwiGLU rows of
// 28672 166 us (1.8 TB/s).
template <class T>
struct Eight {
    T v[8];
};
template <class T>
__device__ __forceinline__ Eight<T> load8(const T *p) {
    return *(const Eight<T> *)__builtin_assume_aligned(p, 16);
}

// eight elements wherever they lie (the hardware takes global accesses of any alignment), `there` of them
template <class T>
__device__ __forceinline__ Eight<T> load8_any(const T *p, int there) {
    Eight<T> q;
    if (there >= 8) __builtin_memcpy(&q, p, sizeof(q));
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) q.v[e] = e < there ? p[e] : (T)0.f;
    }
    return q;
}
template <class T>
__device__ __forceinline__ void store8_any(T *p, const Eight<T> &q, int there) {
    if (there >= 8) __builtin_memcpy(p, &q, sizeof(q));
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < there) p[e] = q.v[e];
    }
}

// WHOLE: rows are whole chunks, 16-byte aligned.  Otherwise chunks lie anywhere and the last one may be short (its missing elements count as 0).
template <class T, int KIND, bool ADD, int CH, bool WHOLE>
__global__ void __launch_bounds__(CH >= 4 ? 256 : 1024) k_rows_q8_wide(RowArgs A) {
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const T *x = (const T *)A.x + row * A.ld_x, *add = ADD ? (const T *)A.add + row * A.ld_add : nullptr;
    const int at = threadIdx.x * 8, stride = blockDim.x * 8;
    Eight<T> in[CH], in2[ADD || KIND == ROW_SWIGLU ? CH : 1];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = at + c * stride < A.n ? at + c * stride : 0;      // (past the row: not used)
        if constexpr (WHOLE) {
            in[c] = load8(x + i);
            if constexpr (ADD) in2[c] = load8(add + i);
            if constexpr (KIND == ROW_SWIGLU) in2[c] = load8(x + A.n + i);
        } else {
            in[c] = load8_any(x + i, A.n - i);
            if constexpr (ADD) in2[c] = load8_any(add + i, A.n - i);
            if constexpr (KIND == ROW_SWIGLU) in2[c] = load8_any(x + A.n + i, A.n - i);
        }
    }
    Squares squares;
    float v[CH][8], most = 0.f;
    bool fine = true;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (at + c * stride >= A.n) continue;
        if constexpr (KIND == ROW_NORM) {
            const int there = A.n - at - c * stride;
            const Eight<float> gain = WHOLE ? load8(A.gain + at + c * stride) : load8_any(A.gain + at + c * stride, there);
            Eight<T> out;
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[e] = (float)in[c].v[e];
                if constexpr (ADD) s[e] += (float)in2[c].v[e];
                out.v[e] = (T)s[e];
                v[c][e] = s[e] * gain.v[e];
            }
            squares.add(s);
            T *to = (T *)A.sum + row * A.ld_sum + at + c * stride;
            if (A.sum) {
                if constexpr (WHOLE) *(Eight<T> *)__builtin_assume_aligned(to, 16) = out;
                else store8_any(to, out, there);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = (float)in[c].v[e];
                if constexpr (KIND == ROW_SWIGLU) v[c][e] = g / (1.f + __builtin_expf(-g)) * (float)in2[c].v[e];
                else v[c][e] = g;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            fine = fine && fabsf(v[c][e]) <= 3.402823466e38f;
            most = fmaxf(most, fabsf(v[c][e]));
        }
    }
    if (!fine) most = __builtin_inff();
    float ss = squares.plain;
    __shared__ float sh[2][16];
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
    ss = sh[0][0];
    most = sh[1][0];
    for (int w = 1; w < waves; ++w) {
        ss += sh[0][w];
        most = fmaxf(most, sh[1][w]);
    }
    float factor = 1.f;
    if constexpr (KIND == ROW_NORM) {
        __shared__ float far[16];
        factor = norm_factor(ss, squares, A.n, A.eps, far);
    }
    // (a row of zeros without an eps has a factor of infinity, and 0 times it is NaN)
    const bool ok = most < __builtin_inff() && (KIND != ROW_NORM || most * factor < __builtin_inff());
    const float a = fmaxf(most * factor, 0x1p-90f), up = 127.f / a;
    if (threadIdx.x == 0) A.scales[row] = ok ? a / 127.f : __builtin_nanf("");
    int8_t *codes = A.codes + row * A.ld_codes;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (at + c * stride >= A.n) continue;
        unsigned lo = 0, hi = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo |= ((unsigned)(int)rintf(v[c][e] * factor * up) & 255u) << (8 * e);
            hi |= ((unsigned)(int)rintf(v[c][4 + e] * factor * up) & 255u) << (8 * e);
        }
        const uint2 q = ok ? make_uint2(lo, hi) : make_uint2(0u, 0u);
        if constexpr (WHOLE) *(uint2 *)(codes + at + c * stride) = q;
        else store8_any(codes + at + c * stride, __builtin_bit_cast(Eight<int8_t>, q), A.n - at - c * stride);
    }
}

template <class T, int KIND, bool ADD>
hipError_t launch_rows_of(int rows, const RowArgs &A, hipStream_t s) {
    const uintptr_t bits = (uintptr_t)A.x | (uintptr_t)A.add | (uintptr_t)A.sum | (uintptr_t)A.gain;
    const int64_t strides = A.ld_x | A.ld_add | (A.sum ? A.ld_sum : 0) | A.ld_codes;
    if (A.n > 16384) {
        hipLaunchKernelGGL((k_rows_q8<T, KIND, ADD>), dim3(rows), dim3(256), 0, s, A);
        return hipGetLastError();
    }
    const bool whole = !(A.n % 8 || bits % 16 || strides % 8 || (uintptr_t)A.codes % 8);
    // few rows: as many threads as there are chunks, so that all of a row is asked for at once; many: four chunks a thread
    const int chunks = (A.n + 7) / 8, most = rows <= 512 ? 1024 : 256;
    int threads = 64;
    while (threads < most && threads * (rows <= 512 ? 1 : 4) < chunks) threads *= 2;
    const int each = (chunks + threads - 1) / threads;
    auto launch = [&](auto ch) {
        constexpr int CH = decltype(ch)::value;
        if (whole) hipLaunchKernelGGL((k_rows_q8_wide<T, KIND, ADD, CH, true>), dim3(rows), dim3(threads), 0, s, A);
        else hipLaunchKernelGGL((k_rows_q8_wide<T, KIND, ADD, CH, false>), dim3(rows), dim3(threads), 0, s, A);
        return hipGetLastError();
    };
    if (each <= 1) return launch(std::integral_constant<int, 1>());
    if (each <= 2) return launch(std::integral_constant<int, 2>());
    if (each <= 4) return launch(std::integral_constant<int, 4>());
    return launch(std::integral_constant<int, 8>());
}

template <class T>
hipError_t launch_rows(int kind, int rows, const RowArgs &A, hipStream_t s) {
    if (kind == ROW_NORM) return A.add ? launch_rows_of<T, ROW_NORM, true>(rows, A, s) : launch_rows_of<T, ROW_NORM, false>(rows, A, s);
    return kind == ROW_PLAIN ? launch_rows_of<T, ROW_PLAIN, false>(rows, A, s) : launch_rows_of<T, ROW_SWIGLU, false>(rows, A, s);
}

int rows_impl(int kind, int32_t dtype, int32_t rows, const RowArgs &A, void *stream) {
    const int64_t width = kind == ROW_SWIGLU ? 2 * (int64_t)A.n : A.n;
    if (dtype != SPD_F32 && dtype != SPD_BF16 && dtype != SPD_F16) return SPD_EINVAL;
    if (rows < 0 || rows > (1 << 23) || A.n < 0 || A.n > (1 << 30)) return SPD_EINVAL;
    if (rows == 0 || A.n == 0) return SPD_OK;
    if (!A.x || !A.codes || !A.scales || A.ld_x < width || A.ld_codes < A.n) return SPD_EINVAL;
    if ((kind == ROW_NORM && !A.gain) || (A.add && A.ld_add < A.n) || (A.sum && A.ld_sum < A.n)) return SPD_EINVAL;
    const uintptr_t es = dtype == SPD_F32 ? 4 : 2;
    if ((uintptr_t)A.x % es || (uintptr_t)A.add % es || (uintptr_t)A.sum % es || (uintptr_t)A.scales % 4 || (uintptr_t)A.gain % 4) return SPD_EINVAL;
    // a sum takes the place of a summand, or of neither; codes that of nothing
    const int64_t n = A.n, e = (int64_t)es;
    const spd_extent x{A.x, rows, width * e, A.ld_x * e}, add{A.add, rows, n * e, A.ld_add * e}, sum{A.sum, rows, n * e, A.ld_sum * e},
        codes{A.codes, rows, n, A.ld_codes};
    if (A.sum == A.x ? A.ld_sum != A.ld_x : spd_share_memory(x, sum)) return SPD_EINVAL;
    if (A.sum && A.sum == A.add ? A.ld_sum != A.ld_add : spd_share_memory(add, sum)) return SPD_EINVAL;
    if (spd_share_memory(x, codes) || spd_share_memory(add, codes) || spd_share_memory(sum, codes)) return SPD_EINVAL;
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
    int quads;               // rows of out and add hold whole, aligned groups of four columns
};

template <class T>
struct Quad {            // four elements of T
    T v[4];
};

template <class T>
struct Piece {           // 16 bytes of them
    T v[16 / sizeof(T)];
};

// four columns of a row, n a multiple of 4; a place past the matrix: nothing.  sm, sn: scales of the row and of the columns
template <class T>
__device__ __forceinline__ void q8_store(const Q8Args &A, int m, int n, i32x4 acc, float sm, f32x4 sn) {
    if (m >= A.rows || n >= A.N) return;
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)acc[i] * sm * sn[i];
    T *out = (T *)A.out + m * A.ld_out + n;
    const T *add = A.add ? (const T *)A.add + m * A.ld_add + n : nullptr;
    if (A.quads) {       // whole and aligned
        if (add) {
            const Quad<T> q = *(const Quad<T> *)__builtin_assume_aligned(add, sizeof(Quad<T>));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += (float)q.v[i];
        }
        Quad<T> q;
#pragma unroll
        for (int i = 0; i < 4; ++i) q.v[i] = (T)v[i];
        *(Quad<T> *)__builtin_assume_aligned(out, sizeof(Quad<T>)) = q;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < A.N) out[i] = (T)(add ? v[i] + (float)add[i] : v[i]);
}
__device__ __forceinline__ float q8_row_scale(const Q8Args &A, int m) { return A.scales[m < A.rows ? m : A.rows - 1]; }
// (the scales are padded to whole n-tiles)
__device__ __forceinline__ f32x4 q8_col_scales(const Q8Args &A, int nt, int g) {
    return *(const f32x4 *)((const float *)A.packed + (nt < A.NT ? nt : A.NT - 1) * 16 + 4 * g);
}

// ------------------------------------------------------------------------------------------
// Few rows: the weights are streamed once.  A workgroup takes NP n-tiles and all of K, its eight waves a share of the k-tiles each; both
// operands go straight into registers, a batch of k-tiles ahead of the one in use, and the waves' integer sums meet in the LDS.  Bound by what
// a compute unit draws through its load path: (NP + MT) KiB per k-tile.  K 8192, N 7168, 16 rows: 14.2 us a call (59 MB of
// weights: 4.1 TB/s); loads and their use in turn: 15.1.
// ------------------------------------------------------------------------------------------
template <class T, int MT, int NP>
__global__ void __launch_bounds__(512) k_q8_skinny(Q8Args A) {
    constexpr int NB = MT >= 4 ? 2 : 4;                        // k-tiles asked for at a time
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nt0 = blockIdx.x * NP, m0 = blockIdx.y * (MT * 16);
    const int r = lane & 15, g = lane >> 4;
    const int per = (A.KT + 7) / 8, kt0 = wave * per, kt1 = kt0 + per < A.KT ? kt0 + per : A.KT;
    const char *w[NP];
    const int8_t *x[MT];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int nt = nt0 + i < A.NT ? nt0 + i : A.NT - 1;
        w[i] = A.packed + spd_q8_weights_at(A.N) + (size_t)nt * A.KT * 1024 + lane * 16;
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int m = m0 + 16 * j + r;
        x[j] = A.codes + (int64_t)(m < A.rows ? m : A.rows - 1) * A.ld_codes;
    }
    const int k_last = (A.K - 1) & ~15;                        // past K: anything, the weights are zero there
    i32x4 acc[NP][MT];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
    struct Batch {
        i32x4 a[NB][NP], b[NB][MT];
    };
    auto load = [&](Batch &f, int kt) __attribute__((always_inline)) {      // (k-tiles past the share: its last one, not used)
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const int t = kt + u < kt1 ? kt + u : kt1 - 1;
            int k = t * 64 + 16 * g;
            k = k < k_last ? k : k_last;
#pragma unroll
            for (int i = 0; i < NP; ++i) f.a[u][i] = __builtin_nontemporal_load((const i32x4 *)(w[i] + (size_t)t * 1024));
#pragma unroll
            for (int j = 0; j < MT; ++j) f.b[u][j] = *(const i32x4 *)(x[j] + k);
        }
    };
    auto use = [&](const Batch &f, int kt) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NB; ++u)
            if (kt + u < kt1) {
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int j = 0; j < MT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.a[u][i], f.b[u][j], acc[i][j], 0, 0, 0);
            }
    };
    if (kt0 < kt1) {
        Batch f0, f1;
        load(f0, kt0);
        for (int kt = kt0; kt < kt1; kt += 2 * NB) {      // the next batch is on its way while one is used
            if (kt + NB < kt1) load(f1, kt + NB);
            use(f0, kt);
            if (kt + NB < kt1) {
                if (kt + 2 * NB < kt1) load(f0, kt + 2 * NB);
                use(f1, kt + NB);
            }
        }
    }
    __shared__ i32x4 part[8][NP * MT][64];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) part[wave][i * MT + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < NP * MT; t += 8) {
        i32x4 v = part[0][t][lane];
#pragma unroll
        for (int u = 1; u < 8; ++u) v += part[u][t][lane];
        const int i = t / MT, j = t % MT;
        q8_store<T>(A, m0 + 16 * j + r, (nt0 + i) * 16 + 4 * g, v, q8_row_scale(A, m0 + 16 * j + r), q8_col_scales(A, nt0 + i, g));
    }
}

// ------------------------------------------------------------------------------------------
// Many rows: tiles of WN TI n-tiles x WM TJ m-tiles through the LDS, NST stages of KPS k-tiles, copied there directly.  Copies go through
// buffer descriptors of the tile's panels; rows and inputs past the matrix repeat its last ones.  While the MFMAs of a k-tile run, the fragments of
// the next are read between them.  KPS 2: a step is two k-tiles with a barrier between them, and in the second one the copies of the stage NST
// steps ahead go out.  KPS 1: a barrier per k-tile, the copies go out five k-tiles ahead.  Two k-tiles of a row of codes are a cache line, which
// KPS 2 copies at once and KPS 1 twice: it pays from K 7168 on, where far rows (K a multiple of 4096 above all) answer late.  2000 rows, N 7168, us
// with KPS 2 / 1: K 2048 33.1 / 33.9, 5120 69.0 / 69.6, 7168 100 / 94, 8192 120 / 107, 8256 111 / 109, 16384 244 / 209; K 1728 25.5 / 29.1.
// The results leave through the LDS in whole cache lines: stored as
// they lie in the registers (32 bytes a row and store) they took 2.2 times as long as K = 1024 did beside them (8192 rows, N 8192: 146 us a
// call, now 79).  8192 rows, K 8192, N 7168: 406 to 417 us, 2.3 P operations a second (torch's library product of 8-bit integers: 400).  Bound by
// the copies beside the MFMAs: 8192 cubed takes 472 us, without the copies 348, and all workgroups at one tile, out of the L2, 456; MFMAs
// alone run at 3.55 P a second.  (A workgroup that goes on with its next tile's copies before it stores needs its descriptors in vector
// registers: 559 us; four waves of 128 x 128 each, a third less read from the LDS: 445 beside 431; copies of the waves at different MFMAs: 426 to 496.)
// ------------------------------------------------------------------------------------------
struct Q8Big {       // 256 x 256
    static constexpr int WN = 4, WM = 2, TI = 4, TJ = 8, KPS = 2, NST = 2;
};
struct Q8Deep {      // the same for a long K: stages of one k-tile, copied five ahead
    static constexpr int WN = 4, WM = 2, TI = 4, TJ = 8, KPS = 1, NST = 5;
};
constexpr int Q8_DEEP_KT = 112;
struct Q8Half {      // 256 x 128
    static constexpr int WN = 4, WM = 2, TI = 4, TJ = 4, KPS = 2, NST = 3;
};
struct Q8Square {    // 128 x 128
    static constexpr int WN = 4, WM = 2, TI = 2, TJ = 4, KPS = 2, NST = 4;
};
struct Q8Small {     // 128 x 64, two workgroups per compute unit
    static constexpr int WN = 4, WM = 2, TI = 2, TJ = 2, KPS = 2, NST = 3;
};
constexpr int waitcnt_imm(int vm, int lgkm) { return (vm & 15) | ((vm >> 4) << 14) | (7 << 4) | (lgkm << 8); }

template <class T, class G>
__global__ void __launch_bounds__(G::WN *G::WM * 64, 1) k_q8_gemm(Q8Args A, spd_tile_order ord, int tile0, int n_tiles, int msub) {
    constexpr int TI = G::TI, TJ = G::TJ, NST = G::NST, KPS = G::KPS, NW = G::WN * G::WM, BN = G::WN * TI, BM = G::WM * TJ;
    constexpr int W_BYTES = BN * KPS * 1024, STAGE = W_BYTES + BM * KPS * 1024;
    constexpr int CW = BN * KPS / NW, CX = BM * KPS / NW, NCP = CW + CX;
    static_assert(BN * KPS % NW == 0 && BM * KPS % NW == 0 && (NST - 1) * NCP < 64, "tile shape");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % G::WN, wm = wave / G::WN;
    const int KT = A.KT, l16 = lane * 16, r = lane & 15, g = lane >> 4;
    const unsigned pitch = (unsigned)KT * 1024;
    const int k16 = (A.K + 15) & ~15;
    // the last k-tile's lanes past K repeat its last 16 inputs
    const int tail = (KT - 1) * 64 + 16 * g > k16 - 16 ? k16 - 16 - (KT - 1) * 64 - 16 * g : 0;
    int nt0, m0;
    {
        // n_tiles tiles of the order from tile0 on, each cut into msub along the rows (2: the last round of a launch of tiles twice as high)
        const int idx = msub == 1 ? spd_tile_deal((int)blockIdx.x, n_tiles) : (int)blockIdx.x / msub;
        if (idx < 0) return;                 // spare workgroup of a ragged share (whole workgroup, before any barrier)
        int tn, tm;
        spd_tile_at(ord, tile0 + idx, tn, tm);
        nt0 = tn * BN;
        m0 = (tm * msub + (msub == 1 ? 0 : (int)blockIdx.x % msub)) * BM * 16;
        if (m0 >= A.rows) return;            // (whole workgroup)
    }
    const int n_rows = A.NT - nt0 < BN ? A.NT - nt0 : BN, m_rows = A.rows - m0 < BM * 16 ? A.rows - m0 : BM * 16;
    const __amdgpu_buffer_rsrc_t
        wbuf = __builtin_amdgcn_make_buffer_rsrc((void *)(A.packed + spd_q8_weights_at(A.N) + (size_t)nt0 * pitch), 0, (int)(n_rows * pitch), 0x00020000),
        xbuf = __builtin_amdgcn_make_buffer_rsrc((void *)(A.codes + m0 * A.ld_codes), 0, (int)((m_rows - 1) * (unsigned)A.ld_codes + k16), 0x00020000);
    unsigned wsrc[CW], xoff[CX];             // (wsrc: wave-uniform)
#pragma unroll
    for (int n = 0; n < CW; ++n) {
        const int t = (wave * CW + n) / KPS;
        wsrc[n] = (unsigned)(t < n_rows ? t : n_rows - 1) * pitch;
    }
#pragma unroll
    for (int n = 0; n < CX; ++n) {
        const int m = ((wave * CX + n) / KPS) * 16 + r;
        xoff[n] = (unsigned)(m < m_rows ? m : m_rows - 1) * (unsigned)A.ld_codes + 16 * g;
    }
    i32x4 acc[TI][TJ];
    auto copy1 = [&](int st, int slot, int n) __attribute__((always_inline)) {
        if (n < CW) {
            int kt = KPS * st + (wave * CW + n) % KPS;
            if constexpr (KPS > 1) kt = kt < KT ? kt : KT - 1;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wbuf, (__attribute__((address_space(3))) void *)(lds + slot * STAGE + (wave * CW + n) * 1024), 16,
                                                     l16, __builtin_amdgcn_readfirstlane((int)(wsrc[n] + kt * 1024)), 0, 0);
        } else {
            const int c = n - CW;
            int kt = KPS * st + (wave * CX + c) % KPS;
            if constexpr (KPS > 1) kt = kt < KT ? kt : KT - 1;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (__attribute__((address_space(3))) void *)(lds + slot * STAGE + W_BYTES + (wave * CX + c) * 1024),
                                                     16, (int)(xoff[c] + (kt == KT - 1 ? tail : 0)), kt * 64, 0, 0);
        }
    };
    const char *a_base = lds + wn * TI * KPS * 1024 + l16, *b_base = lds + W_BYTES + wm * TJ * KPS * 1024 + l16;
    auto read1 = [&](int slot, int p, int f, i32x4(&a)[TI], i32x4(&b)[TJ]) __attribute__((always_inline)) {
        if (f < TJ) b[f] = *(const i32x4 *)(b_base + slot * STAGE + (KPS * f + p) * 1024);
        else a[f - TJ] = *(const i32x4 *)(a_base + slot * STAGE + ((f - TJ) * KPS + p) * 1024);
    };
    const int n_stages = (KT + KPS - 1) / KPS, n_steps = KT / 2;
    auto first_copies = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < NST; ++st)
            if (st < n_stages) {
#pragma unroll
                for (int n = 0; n < NCP; ++n) copy1(st, st, n);
            }
    };
    i32x4 a0[TI], a1[TI], b0[TJ], b1[TJ];
    auto substep = [&](auto copy_, const i32x4(&a)[TI], const i32x4(&b)[TJ], i32x4(&an)[TI], i32x4(&bn)[TJ], int rslot, int rp, int cst,
                       int cslot) __attribute__((always_inline)) {
        constexpr int NR = TI + TJ, NM = TI * TJ;
        const bool copy = copy_;                 // (a constant, or uniform)
        int f = 0, cp = 0;
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                const int n = i * TJ + j;
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                while (f < NR && n >= (2 * NR <= NM ? 2 * f : f * NM / NR)) read1(rslot, rp, f++, an, bn);
                while (cp < NCP && n >= (NM >= NCP ? cp * (NM / NCP) : cp * NM / NCP)) {
                    if (copy) copy1(cst, cslot, cp);
                    ++cp;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    first_copies();
    __builtin_amdgcn_sched_barrier(0);
    if (n_stages >= NST) __builtin_amdgcn_s_waitcnt(waitcnt_imm((NST - 1) * NCP, 0));
    else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
#pragma unroll
    for (int f = 0; f < TI + TJ; ++f) read1(0, 0, f, a0, b0);
    int slot = 0;
    if constexpr (KPS == 1) {
        // One k-tile: the copies of the next one have landed in every wave, and every wave holds the fragments of this one.  (Copies are left out by
        // branches: steps of their own without them double the code, and the accumulators do not survive it in registers.)
        auto step = [&](const i32x4(&a)[TI], const i32x4(&b)[TJ], i32x4(&an)[TI], i32x4(&bn)[TJ], int s) __attribute__((always_inline)) {
            const int next = slot + 1 == NST ? 0 : slot + 1;
            const bool more = s + NST < KT;
            if (more) __builtin_amdgcn_s_waitcnt(waitcnt_imm((NST - 2) * NCP, 0));
            else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            substep(more, a, b, an, bn, next, 0, s + NST, slot);      // (in the last step: fragments read and never used)
            slot = next;
        };
        for (int s = 0;;) {
            step(a0, b0, a1, b1, s);
            if (++s == KT) break;
            step(a1, b1, a0, b0, s);
            if (++s == KT) break;
        }
    } else {
        auto step = [&](auto copy_, int s) __attribute__((always_inline)) {
            constexpr bool COPY = decltype(copy_)::value;
            const int next = slot + 1 == NST ? 0 : slot + 1;
            substep(std::false_type(), a0, b0, a1, b1, slot, 1, 0, 0);
            // the next stage's copies of this wave have landed, every read of the current stage is done
            __builtin_amdgcn_s_waitcnt(waitcnt_imm(COPY ? (NST - 2) * NCP : 0, 0));
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            substep(copy_, a1, b1, a0, b0, next, 0, s + NST, slot);      // (in the last step: fragments read and never used)
            slot = next;
        };
        int s = 0;
        for (; s + NST < n_stages; ++s) step(std::true_type(), s);
        for (; s < n_steps; ++s) step(std::false_type(), s);
    }
    if (KPS == 2 && (KT & 1)) {                            // the odd k-tile on its own (its fragments are read already)
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a0[i], b0[j], acc[i][j], 0, 0, 0);
    }
    f32x4 sn[TI];
    float sm[TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i) sn[i] = q8_col_scales(A, nt0 + wn * TI + i, g);
#pragma unroll
    for (int j = 0; j < TJ; ++j) sm[j] = q8_row_scale(A, m0 + (wm * TJ + j) * 16 + r);
    if (A.quads == 2) {
        // through the LDS, a wave's own part of it, so that a row of the wave's columns leaves in whole cache lines
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, 0));
        asm volatile("s_barrier" ::: "memory");
        const int n0 = (nt0 + wn * TI) * 16;
        // S: what waits in the LDS, T, or fp32 where a summand joins before the rounding
        auto rows_out = [&](auto s_) __attribute__((always_inline)) {
            typedef decltype(s_) S;
            constexpr bool ADD = !std::is_same<S, T>::value || std::is_same<T, float>::value;
            constexpr int E = 16 / sizeof(T), PIECES = TI * 16 / E, ROW = TI * 16 + 16 / sizeof(S);      // elements in 16 bytes of output; row pitch
            static_assert(NW * 16 * ROW * sizeof(S) <= NST * STAGE, "rows fit");
            S *mine = (S *)lds + wave * 16 * ROW;
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    Quad<S> q;
#pragma unroll
                    for (int e = 0; e < 4; ++e) q.v[e] = (S)((float)acc[i][j][e] * sm[j] * sn[i][e]);
                    *(Quad<S> *)__builtin_assume_aligned(mine + r * ROW + i * 16 + 4 * g, sizeof(Quad<S>)) = q;
                }
                const int m1 = m0 + (wm * TJ + j) * 16;
#pragma unroll
                for (int p = lane; p < 16 * PIECES; p += 64) {
                    const int row = p / PIECES, c = (p % PIECES) * E;
                    if (m1 + row >= A.rows || n0 + c >= A.N) continue;
                    Piece<T> v;
                    if constexpr (ADD) {
                        Piece<T> y;
                        if (A.add) y = *(const Piece<T> *)__builtin_assume_aligned((const T *)A.add + (m1 + row) * A.ld_add + n0 + c, 16);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float x = (float)mine[row * ROW + c + e];
                            v.v[e] = (T)(A.add ? x + (float)y.v[e] : x);
                        }
                    } else v = *(const Piece<T> *)__builtin_assume_aligned(mine + row * ROW + c, 16);
                    *(Piece<T> *)__builtin_assume_aligned((T *)A.out + (m1 + row) * A.ld_out + n0 + c, 16) = v;
                }
            }
        };
        if (A.add) rows_out(0.f);
        else rows_out(T());
        return;
    }
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int i = 0; i < TI; ++i)
            q8_store<T>(A, m0 + (wm * TJ + j) * 16 + r, (nt0 + wn * TI + i) * 16 + 4 * g, acc[i][j], sm[j], sn[i]);
}

// Rows too far apart for 32-bit offsets inside a panel: one wave per 64 columns x 64 rows, operands straight from memory
template <class T>
__global__ void __launch_bounds__(256) k_q8_far(Q8Args A) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nt0 = (blockIdx.y * 4 + wave) * 4;
    const int64_t m0 = (int64_t)blockIdx.x * 64;
    if (nt0 >= A.NT) return;
    const int r = lane & 15, g = lane >> 4;
    const char *w[4];
    const int8_t *x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int nt = nt0 + i < A.NT ? nt0 + i : A.NT - 1;
        const int64_t m = m0 + 16 * i + r;
        w[i] = A.packed + spd_q8_weights_at(A.N) + (size_t)nt * A.KT * 1024 + lane * 16;
        x[i] = A.codes + (m < A.rows ? m : A.rows - 1) * A.ld_codes;
    }
    const int k_last = (A.K - 1) & ~15;
    i32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
    for (int kt = 0; kt < A.KT; ++kt) {
        int k = kt * 64 + 16 * g;
        k = k < k_last ? k : k_last;
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
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + 16 * j + r;
            if (m < A.rows) q8_store<T>(A, (int)m, (nt0 + i) * 16 + 4 * g, acc[i][j], A.scales[m], q8_col_scales(A, nt0 + i, g));
        }
}

template <class T, int MT, int NP>
hipError_t launch_skinny(const Q8Args &A, hipStream_t s) {
    hipLaunchKernelGGL((k_q8_skinny<T, MT, NP>), dim3((A.NT + NP - 1) / NP, (A.rows + 16 * MT - 1) / (16 * MT)), dim3(512), 0, s, A);
    return hipGetLastError();
}
// tiles tile0 .. of the order of tiles msub times as high as G's
template <class T, class G>
hipError_t launch_gemm(const Q8Args &A, hipStream_t s, int tile0 = 0, int n_tiles = -1, int msub = 1) {
    constexpr int BN = G::WN * G::TI, BM = G::WM * G::TJ, LDS = G::NST * (BN + BM) * G::KPS * 1024;
    static_assert(LDS <= 160 * 1024, "the stages must fit the LDS of a compute unit");
    static std::once_flag once;
    static hipError_t attr = hipSuccess;
    std::call_once(once, [] { attr = hipFuncSetAttribute((const void *)k_q8_gemm<T, G>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS); });
    if (attr != hipSuccess) return attr;
    const int high = BM * 16 * msub;
    spd_tile_order ord;
    ord.TN = (A.NT + BN - 1) / BN;
    ord.TM = (int)(((int64_t)A.rows + high - 1) / high);
    spd_pick_block(ord.TN, ord.TM, BN * 16, high, ord.bn, ord.bm);
    if (n_tiles < 0) n_tiles = ord.TN * ord.TM - tile0;
    hipLaunchKernelGGL((k_q8_gemm<T, G>), dim3(msub == 1 ? spd_tile_launch_size(n_tiles) : n_tiles * msub), dim3(G::WN * G::WM * 64), LDS, s, A, ord,
                       tile0, n_tiles, msub);
    return hipGetLastError();
}

enum Q8Kind { Q8_FAR, Q8_11, Q8_12, Q8_14, Q8_22, Q8_42, Q8_SMALL, Q8_SQUARE, Q8_HALF, Q8_BIG, Q8_BIG_HALF };      // (spd_testing.h)

// Which kernel: the one that is estimated to end first.  A round of workgroups, one per compute unit, costs what a unit draws through its load
// path (skinny kernels, small tiles) or multiplies (large ones) over K, and what comes before and after.  The figures, in us for a K of 8192
// and beside it, are fits to measured calls of 1 to 8192 rows, K 1024 to 8192, N 1280 to 8192.
Q8Kind q8_pick(int rows, int N, int KT, int64_t ld_codes) {
    // 256 rows of a panel within 2^31 bytes.  (Few rows too, whose kernels would take them: codes 4 MiB apart are no layout of rows that this library
    // writes, and were not timed.)
    if (ld_codes > (1 << 22)) return Q8_FAR;
    const double k = KT / 128.0;
    const int64_t NT = spd_q8_ntiles(N), MT = ((int64_t)rows + 15) / 16;
    auto rounds = [](int64_t n) { return (double)((n + 255) / 256); };
    auto tiles = [&](int bn, int bm) { return ((NT + bn - 1) / bn) * ((MT + bm - 1) / bm); };
    Q8Kind best = Q8_BIG;
    double least = 1e30;
    auto offer = [&](Q8Kind kind, double us) {
        if (us < least) {
            least = us;
            best = kind;
        }
    };
    if (rows <= 512) {
        offer(Q8_11, rounds(tiles(1, 1)) * (k * 3.4 * 2 + 1.6));
        offer(Q8_12, rounds(tiles(2, 1)) * (k * 3.4 * 3 + 1.7));
        offer(Q8_14, rounds(tiles(4, 1)) * (k * 3.4 * 5 + 1.9));
        offer(Q8_22, rounds(tiles(2, 2)) * (k * 3.4 * 4 + 1.9));
        offer(Q8_42, rounds(tiles(2, 4)) * (k * 3.4 * 6 + 2.3));
    }
    offer(Q8_SMALL, (tiles(8, 4) <= 256 ? 1.0 : 0.85) * rounds(tiles(8, 4)) * (k * 28 + 2));
    offer(Q8_SQUARE, rounds(tiles(8, 8)) * (k * 38 + 2.7));
    offer(Q8_HALF, rounds(tiles(16, 8)) * (k * 63 + 4));
    const int64_t big = tiles(16, 16);
    const double round = k * (KT >= Q8_DEEP_KT ? 98 : 104) + 8;
    offer(Q8_BIG, rounds(big) * round);
    if (big > 256 && big % 256) offer(Q8_BIG_HALF, (double)(big / 256) * round + rounds(2 * (big % 256)) * (k * 63 + 4));
    return best;
}

template <class T>
hipError_t launch_big(const Q8Args &A, hipStream_t s, int tile0 = 0, int n_tiles = -1) {
    return A.KT >= Q8_DEEP_KT ? launch_gemm<T, Q8Deep>(A, s, tile0, n_tiles) : launch_gemm<T, Q8Big>(A, s, tile0, n_tiles);
}

template <class T>
hipError_t launch_product(const Q8Args &A, hipStream_t s) {
    switch (q8_pick(A.rows, A.N, A.KT, A.ld_codes)) {
        case Q8_FAR:
            hipLaunchKernelGGL((k_q8_far<T>), dim3((unsigned)(((int64_t)A.rows + 63) / 64), (A.NT + 15) / 16), dim3(256), 0, s, A);
            return hipGetLastError();
        case Q8_11: return launch_skinny<T, 1, 1>(A, s);
        case Q8_12: return launch_skinny<T, 1, 2>(A, s);
        case Q8_14: return launch_skinny<T, 1, 4>(A, s);
        case Q8_22: return launch_skinny<T, 2, 2>(A, s);
        case Q8_42: return launch_skinny<T, 4, 2>(A, s);
        case Q8_SMALL: return launch_gemm<T, Q8Small>(A, s);
        case Q8_SQUARE: return launch_gemm<T, Q8Square>(A, s);
        case Q8_HALF: return launch_gemm<T, Q8Half>(A, s);
        case Q8_BIG: return launch_big<T>(A, s);
        case Q8_BIG_HALF: {
            const int big = ((A.NT + 15) / 16) * (int)(((int64_t)A.rows + 255) / 256), rest = big % 256;
            const hipError_t e = launch_big<T>(A, s, 0, big - rest);
            return e != hipSuccess ? e : launch_gemm<T, Q8Half>(A, s, big - rest, rest, 2);
        }
    }
    return hipErrorInvalidValue;
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

int spd_q8_kernel_of(int32_t rows, int32_t K, int32_t N, int64_t ld_codes) {
    if (rows < 1 || rows > (1 << 28) || !spd_q8_weight_bytes(K, N) || ld_codes < K) return SPD_EINVAL;
    const int kind = q8_pick(rows, N, spd_q8_ktiles(K), ld_codes);
    return kind >= Q8_BIG && spd_q8_ktiles(K) >= Q8_DEEP_KT ? kind + 2 : kind;
}

size_t spd_q8_matmul_workspace(int32_t rows, int32_t K, int32_t N) {
    (void)rows;
    (void)K;
    (void)N;
    return 0;
}

int spd_q8_matmul(int32_t rows, int32_t K, int32_t N, const int8_t *codes, int64_t ld_codes, const float *scales, const void *packed,
                  int32_t out_dtype, const void *add, int64_t ld_add, void *out, int64_t ld_out, void *workspace, void *stream) {
    if (rows < 0 || rows > (1 << 28) || !spd_q8_weight_bytes(K, N) || (int64_t)rows * N > (int64_t)1 << 38) return SPD_EINVAL;
    if (out_dtype != SPD_F32 && out_dtype != SPD_BF16 && out_dtype != SPD_F16) return SPD_EINVAL;
    if (rows == 0) return SPD_OK;
    if (!codes || !scales || !packed || !out || ((uintptr_t)codes & 15) || ((uintptr_t)packed & 255) || ((uintptr_t)scales & 3)) return SPD_EINVAL;
    if (ld_codes % 16 || ld_codes < (K + 15) / 16 * 16 || ld_out < N || (add && ld_add < N)) return SPD_EINVAL;
    const uintptr_t es = out_dtype == SPD_F32 ? 4 : 2;
    if ((uintptr_t)out % es || (uintptr_t)add % es) return SPD_EINVAL;
    // the output takes the place of the summand, or of nothing that is read
    const int64_t e = (int64_t)es;
    const spd_extent sums{out, rows, N * e, ld_out * e};
    if (add == out ? ld_add != ld_out : spd_share_memory({add, rows, N * e, ld_add * e}, sums)) return SPD_EINVAL;
    if (spd_share_memory({codes, rows, K, ld_codes}, sums)) return SPD_EINVAL;
    (void)workspace;
    (void)hipGetLastError();
    const uintptr_t quad = 4 * es;
    const bool quads = N % 4 == 0 && ld_out % 4 == 0 && (uintptr_t)out % quad == 0 && (!add || (ld_add % 4 == 0 && (uintptr_t)add % quad == 0));
    const Q8Args A{codes, scales, (const char *)packed, add, out, ld_codes, ld_add, ld_out, rows, K, N, spd_q8_ktiles(K), spd_q8_ntiles(N),
                   quads ? (N % (16 / es) == 0 && ld_out % (16 / es) == 0 && (uintptr_t)out % 16 == 0 && ld_add % (16 / es) == 0 && (uintptr_t)add % 16 == 0 ? 2 : 1) : 0};
    hipStream_t s = (hipStream_t)stream;
    SPD_HIP(out_dtype == SPD_F32 ? launch_product<float>(A, s) : out_dtype == SPD_BF16 ? launch_product<__bf16>(A, s) : launch_product<_Float16>(A, s));
    return SPD_OK;
}

}  // extern "C"
