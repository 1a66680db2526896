// Host side of the 8-bit product: sizes and packers.  Nothing in this file touches a device.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "spd_q8_internal.h"

namespace {

bool sizes_ok(int32_t K, int32_t N) { return K >= 1 && K <= SPD_Q8_MAX_K && N >= 1 && N <= (1 << 24); }

// code(k, n) -> the packed fragments, scale(n) -> the scales
template <class Code, class Scale>
void pack(int K, int N, void *packed, Code code, Scale scale) {
    const int KT = spd_q8_ktiles(K), NT = spd_q8_ntiles(N);
    char *base = (char *)packed;
    std::memset(base, 0, spd_q8_weights_at(N));
    for (int n = 0; n < N; ++n) ((float *)base)[n] = scale(n);
    char *frags = base + spd_q8_weights_at(N);
    spd_parallel_for(NT, [&](int nt) {
        for (int kt = 0; kt < KT; ++kt) {
            int8_t *f = (int8_t *)frags + ((size_t)nt * KT + kt) * 1024;
            for (int j = 0; j < 64; ++j) {
                const int k = kt * 64 + j;
                for (int r = 0; r < 16; ++r) {
                    const int n = nt * 16 + r;
                    f[((j >> 4) * 16 + r) * 16 + (j & 15)] = k < K && n < N ? code(k, n) : 0;
                }
            }
        }
    });
}

}  // namespace

extern "C" {

size_t spd_q8_weight_bytes(int32_t K, int32_t N) {
    if (!sizes_ok(K, N)) return 0;
    return spd_align256(spd_q8_weights_at(N) + (size_t)spd_q8_ntiles(N) * spd_q8_ktiles(K) * 1024);
}

int spd_q8_pack(int32_t K, int32_t N, const float *w, int64_t ld, void *packed_host) {
    if (!sizes_ok(K, N) || !w || !packed_host || ld < N) return SPD_EINVAL;
    try {
        std::vector<float> most(N, 0.f);
        for (int k = 0; k < K; ++k) {
            const float *row = w + (size_t)k * ld;
            for (int n = 0; n < N; ++n) {
                if (!std::isfinite(row[n])) return SPD_EINVAL;
                most[n] = std::max(most[n], std::fabs(row[n]));
            }
        }
        for (float &m : most) m = std::max(m, 0x1p-90f) / 127.f;
        pack(K, N, packed_host, [&](int k, int n) {
            const float c = std::nearbyint(w[(size_t)k * ld + n] / most[n]);
            return (int8_t)std::min(127.f, std::max(-127.f, c));
        }, [&](int n) { return most[n]; });
    } catch (...) {      // (no memory)
        return SPD_EINVAL;
    }
    return SPD_OK;
}

int spd_q8_pack_codes(int32_t K, int32_t N, const int8_t *w, int64_t ld, const float *w_scale, void *packed_host) {
    if (!sizes_ok(K, N) || !w || !w_scale || !packed_host || ld < N) return SPD_EINVAL;
    try {
        pack(K, N, packed_host, [&](int k, int n) { return w[(size_t)k * ld + n]; }, [&](int n) { return w_scale[n]; });
    } catch (...) {
        return SPD_EINVAL;
    }
    return SPD_OK;
}

int spd_q8_unpack(int32_t K, int32_t N, const void *packed_host, int8_t *w, int64_t ld, float *w_scale) {
    if (!sizes_ok(K, N) || !packed_host || !w || !w_scale || ld < N) return SPD_EINVAL;
    const int KT = spd_q8_ktiles(K);
    const char *base = (const char *)packed_host;
    std::memcpy(w_scale, base, (size_t)N * 4);
    const int8_t *frags = (const int8_t *)base + spd_q8_weights_at(N);
    for (int k = 0; k < K; ++k)
        for (int n = 0; n < N; ++n)
            w[(size_t)k * ld + n] = frags[((size_t)(n >> 4) * KT + (k >> 6)) * 1024 + (((k & 63) >> 4) * 16 + (n & 15)) * 16 + (k & 15)];
    return SPD_OK;
}

}  // extern "C"
