// Matrix product in 8-bit floating point (e4m3) with a scale for each block of 128:
//     out[n][v] = sum over b of xs[n][b] * ws[v / 128][b] * (sum over i in block b of x[n][i] * w[v][i]).
#include <type_traits>

#include "../../include/specee.h"
#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;  // elements, or rows of w, that share a scale
constexpr int kOne = 0x7f7f7f7f;  // block scales of 2^0 for the matrix instruction

// 32 codes of a row on a lane: pieces q and q + 4 of 16 in every block
union Codes {
    uintx4 piece[2];
    intx8 all;
};

// The codes as halves (exact), eight to a register group
struct Halves {
    half8 part[4];
    __device__ __forceinline__ explicit Halves(const Codes &c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uintx4 o;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int word = c.all[2 * k + e];
                o[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.f, false));
                o[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.f, true));
            }
            part[k] = __builtin_bit_cast(half8, o);
        }
    }
};

// Sums of one block for 16 rows of w (quads 4q .. 4q + 3 of the result) and 16 of x (column lane % 16)
__device__ __forceinline__ floatx4 block_product(const Codes &w, const Codes &x) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.all, x.all, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, kOne, 0, kOne);
}
__device__ __forceinline__ floatx4 block_product(const Halves &w, const Halves &x) {
    floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.part[k], x.part[k], c, 0, 0, 0);
    return c;
}

template <typename T>
__device__ __forceinline__ void store_quad(T *out, size_t at, int left, const floatx4 &v) {
    typedef T quad __attribute__((ext_vector_type(4)));
    if (left >= 4 && (at & 3) == 0) {
        quad o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)v[e];
        *reinterpret_cast<quad *>(out + at) = o;
    } else {
        for (int e = 0; e < 4 && e < left; ++e) out[at + e] = (T)v[e];
    }
}

constexpr int kTile = 128;  // rows of w and of x per workgroup

// T: type of the result.  fp16 results take the codes as they are, fp32 results as halves.
template <typename T>
__global__ __launch_bounds__(256) void matmul_f8_kernel(MatmulF8Params p) {
    constexpr bool kExact = sizeof(T) == 4;
    typedef typename std::conditional<kExact, Halves, Codes>::type Operand;
    __shared__ uintx4 wt[2][kTile * 8], xt[2][kTile * 8];
    __shared__ float st[2][kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4, c = lane & 15;
    const int v0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
    const int wv = (wave & 1) * 64, wn = (wave >> 1) * 64;

    uintx4 wr[4], xr[4];
    float sr = 0.f;
    auto load = [&](int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + i * 32, k = b * kBlock + (tid & 7) * 16;
            const bool in = k < p.d;
            const int ks = in ? k : 0;
            wr[i] = *reinterpret_cast<const uintx4 *>(p.w + (size_t)min(v0 + r, p.V - 1) * p.d + ks);
            xr[i] = *reinterpret_cast<const uintx4 *>(p.x + (size_t)min(n0 + r, p.N - 1) * p.d + ks);
            if (!in) wr[i] = xr[i] = uintx4{0, 0, 0, 0};
        }
        if (tid < kTile) sr = p.xs[(size_t)min(n0 + tid, p.N - 1) * p.blocks + b] * p.ws[(size_t)blockIdx.x * p.blocks + b];
    };
    auto keep = [&](int buf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + i * 32, at = r * 8 + ((tid & 7) ^ (r & 7));
            wt[buf][at] = wr[i];
            xt[buf][at] = xr[i];
        }
        if (tid < kTile) st[buf][tid] = sr;
    };
    auto operand = [&](const uintx4 *t, int r) {
        Codes o;
        o.piece[0] = t[r * 8 + (q ^ (r & 7))];
        o.piece[1] = t[r * 8 + ((q + 4) ^ (r & 7))];
        return o;
    };

    floatx4 acc[4][4] = {};
    load(0);
    keep(0);
    __syncthreads();
    for (int b = 0; b < p.blocks; ++b) {
        const int buf = b & 1;
        if (b + 1 < p.blocks) load(b + 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Operand x(operand(xt[buf], wn + j * 16 + c));
            const float s = st[buf][wn + j * 16 + c];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const floatx4 t = block_product(Operand(operand(wt[buf], wv + i * 16 + c)), x);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, t[e], acc[i][j][e]);
            }
        }
        if (b + 1 < p.blocks) keep(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + wn + j * 16 + c;
        if (n >= p.N) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = v0 + wv + i * 16 + 4 * q;
            if (v < p.V) store_quad(static_cast<T *>(p.out), (size_t)n * p.V + v, p.V - v, acc[i][j]);
        }
    }
}

}  // namespace

size_t matmul_f8_workspace(int N, int V, int d) {
    return 0;
}

hipError_t launch_matmul_f8(const MatmulF8Params &p, bool half, hipStream_t s) {
    const dim3 grid((p.V + kTile - 1) / kTile, (p.N + kTile - 1) / kTile);
    if (half)
        hipLaunchKernelGGL(matmul_f8_kernel<half_t>, grid, dim3(256), 0, s, p);
    else
        hipLaunchKernelGGL(matmul_f8_kernel<float>, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace specee
