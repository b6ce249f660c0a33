// What stands between two blocks of a decoder, in one pass over the hidden states: the norm behind a block, its gate and
// residual scale, the residual sum, and the norm before what reads the sum next, in fp16 or as the 8-bit operand of
// specee_matmul_f8.  Per row, r(v) = 1 / sqrt(mean(v^2) + eps):
//     t = branch * r(branch) * gamma_post   (or branch itself),
//     s = hidden_scale * hidden + branch_scale * gate * t,        hidden_out = fp16(s),
//     x = s * r(s) * gamma;   x8: per 128 elements  scale = max|x| / 448,  code = e4m3(x / scale).
// Everything between the loads and the stores is in fp32; x is formed from s as it is before its rounding.
// A workgroup holds a row in registers (8 or 16 elements per thread), so there are two meetings for the two sums of squares
// and nothing is read twice; the 16 lanes of a DPP row hold the 128 elements that share a scale.  Many rows are dealt out over
// as many workgroups as the GPU holds, which keep the weights and have the next row on its way while they work on one.
#include <float.h>

#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

constexpr float kF8Max = 448.f;

typedef int intx2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float row16_max(float v) {
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    return fmaxf(v, dpp_f32<kDppMirror>(v));
}

// Sum over the workgroup in a fixed order; part: one slot per wavefront, used by this sum alone
__device__ __forceinline__ float workgroup_sum(float v, float *part) {
    v = wave_sum(v);
    const int waves = blockDim.x / kWave;
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    float sum = 0.f;
    for (int w = 0; w < waves; ++w) sum += part[w];
    return sum;
}

__device__ __forceinline__ void store_half8(half_t *p, const float *v) {
    half8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (half_t)v[e];
    __builtin_nontemporal_store(o, reinterpret_cast<half8 *>(p));
}

// EACH: every row has a gate of its own.  Otherwise gate * gamma_post, exact in fp32, is one factor per element, formed once.
template <int VPT, bool EACH>
__global__ __launch_bounds__(1024) void block_norm_kernel(BlockNormParams p) {
    __shared__ float part[2][2][16];
    const int nvec = p.d / 8;
    // A call without a branch has hidden in its place, and zeros for what is loaded: no load waits behind a condition
    const half_t *branch = p.branch ? p.branch : p.hidden;
    half8 h[VPT], y[VPT], gamma[VPT];
    float factor[VPT][8];
    bool in[VPT];
    int at[VPT];
    int n = blockIdx.x;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = threadIdx.x + j * blockDim.x;
        in[j] = vec < nvec;
        at[j] = (in[j] ? vec : nvec - 1) * 8;
        y[j] = load_half8_stream(branch + (size_t)n * p.d + at[j]);
        h[j] = load_half8_stream(p.hidden + (size_t)n * p.d + at[j]);
        gamma[j] = load_half8((p.gamma ? p.gamma : p.hidden) + at[j]);
        const half8 post = load_half8((p.gamma_post ? p.gamma_post : p.hidden) + at[j]);
        const half8 gate = load_half8((!EACH && p.gate ? p.gate : p.hidden) + at[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            factor[j][e] = p.gamma_post ? (float)post[e] : 1.f;
            if (!EACH && p.gate) factor[j][e] *= (float)gate[e];
        }
    }
    for (int turn = 0; n < p.N; n += gridDim.x, turn ^= 1) {
        const size_t row = (size_t)n * p.d;
        const size_t next = (size_t)min(n + (int)gridDim.x, p.N - 1) * p.d;  // (or the last row once more)
        half8 hn[VPT], yn[VPT], g[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if (EACH) g[j] = load_half8_stream(p.gate + row + at[j]);
            yn[j] = load_half8_stream(branch + next + at[j]);
            hn[j] = load_half8_stream(p.hidden + next + at[j]);
            if (!p.branch) y[j] = zero_half8();
        }
        float r_branch = p.branch_scale;
        if (p.gamma_post) {
            float ssq = 0.f;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf((float)y[j][e], (float)y[j][e], sum);
                ssq += in[j] ? sum : 0.f;
            }
            r_branch *= rsqrtf(workgroup_sum(ssq, part[turn][0]) / p.d + p.eps);
        }
        float s[VPT][8], ssq = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = r_branch * (EACH ? factor[j][e] * (float)g[j][e] : factor[j][e]);
                s[j][e] = fmaf((float)y[j][e], f, p.hidden_scale * (float)h[j][e]);
                sum = fmaf(s[j][e], s[j][e], sum);
            }
            ssq += in[j] ? sum : 0.f;
            if (p.hidden_out && in[j]) store_half8(p.hidden_out + row + at[j], s[j]);
        }
        if (p.x || p.x8) {
            const float r = rsqrtf(workgroup_sum(ssq, part[turn][1]) / p.d + p.eps);
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[j][e] *= r * (float)gamma[j][e];
                    top = fmaxf(top, fabsf(s[j][e]));
                }
                if (p.x && in[j]) store_half8(p.x + row + at[j], s[j]);
                if (p.x8) {
                    top = row16_max(in[j] ? top : 0.f);
                    // (a scale that is no normal number would not divide back)
                    const float scale = top > 0.f ? fmaxf(top / kF8Max, FLT_MIN) : 1.f, inv = 1.f / scale;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {  // s / scale: the remainder of the product puts its rounding right
                        const float f = s[j][e] * inv;
                        s[j][e] = fmaf(fmaf(-f, scale, s[j][e]), inv, f);
                    }
                    intx2 code;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        code[e] = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * e], s[j][4 * e + 1], 0, false);
                        code[e] = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * e + 2], s[j][4 * e + 3], code[e], true);
                    }
                    if (in[j]) {
                        __builtin_nontemporal_store(code, reinterpret_cast<intx2 *>(p.x8 + row + at[j]));
                        if ((at[j] & 127) == 0) p.x8_scales[(size_t)n * ((p.d + 127) / 128) + at[j] / 128] = scale;
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            h[j] = hn[j];
            y[j] = yn[j];
        }
    }
}

}  // namespace

hipError_t launch_block_norm(const BlockNormParams &p, hipStream_t s) {
    const int nvec = p.d / 8;
    // 16 elements per thread from rows of 4104 on: workgroups of 10 to 16 wavefronts leave a CU half empty (5120: 74 -> 72.5
    // us for 8192 rows, 8192: 96 -> 89; at 4096 both fill it)
    const int vpt = nvec > 512 ? 2 : 1;
    const int threads = ((nvec + vpt - 1) / vpt + kWave - 1) / kWave * kWave;
    const bool each = p.gate && p.gate_rows > 1;
    // wavefronts that the registers of a variant leave room for, and rows dealt out evenly over what that makes resident
    const int fit = (vpt == 2 ? 20 : each ? 28 : 32) * kWave / threads, resident = 256 * (fit > 16 ? 16 : fit < 1 ? 1 : fit);
    const int turns = (p.N + resident - 1) / resident, grid = (p.N + turns - 1) / turns;
    const auto kern = vpt == 1 ? (each ? block_norm_kernel<1, true> : block_norm_kernel<1, false>)
                               : (each ? block_norm_kernel<2, true> : block_norm_kernel<2, false>);
    hipLaunchKernelGGL(kern, dim3(grid), dim3(threads), 0, s, p);
    return hipGetLastError();
}

}  // namespace specee
