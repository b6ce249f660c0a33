// What stands between two blocks of a decoder, in one pass over the hidden states: the norm behind a block, its gate and
// residual scale, the residual sum, and the norm before what reads the sum next, in fp16 or as the 8-bit operand of
// specee_matmul_f8.  Per row, r(v) = 1 / sqrt(mean(v^2) + eps):
//     t = branch * r(branch) * gamma_post   (or branch itself),
//     s = hidden_scale * hidden + branch_scale * gate * t,        hidden_out = fp16(s),
//     x = s * r(s) * gamma;   x8: per 128 elements  scale = max|x| / 448,  code = e4m3(x / scale).
// Everything between the loads and the stores is in fp32; x is formed from s as it is before its rounding.
// One workgroup per row, a row in registers (8 or 16 elements per thread), so two meetings for the two sums of squares and
// nothing is read twice; the 16 lanes of a DPP row hold the 128 elements that share a scale.
#include <float.h>

#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

constexpr float kF8Max = 448.f;

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

template <int VPT>
__global__ __launch_bounds__(1024) void block_norm_kernel(BlockNormParams p) {
    __shared__ float part[2][16];
    const int n = blockIdx.x, nvec = p.d / 8;
    const size_t row = (size_t)n * p.d;
    // What a call leaves out is read from hidden instead and not used: no load waits behind a branch
    const half_t *branch = p.branch ? p.branch + row : p.hidden + row;
    const half_t *gate = p.gate ? p.gate + (p.gate_rows > 1 ? row : 0) : p.hidden + row;
    const half_t *post = p.gamma_post ? p.gamma_post : p.hidden + row;
    const half_t *gamma = p.gamma ? p.gamma : p.hidden + row;
    half8 h[VPT], y[VPT], g[VPT], gp[VPT], gm[VPT];
    bool in[VPT];
    int at[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = threadIdx.x + j * blockDim.x;
        in[j] = vec < nvec;
        at[j] = (in[j] ? vec : nvec - 1) * 8;
        y[j] = load_half8(branch + at[j]);
        h[j] = load_half8(p.hidden + row + at[j]);
        gp[j] = load_half8(post + at[j]);
        g[j] = load_half8(gate + at[j]);
        gm[j] = load_half8(gamma + at[j]);
    }
    float r_branch = 1.f;
    if (p.gamma_post) {
        float ssq = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (in[j])
#pragma unroll
                for (int e = 0; e < 8; ++e) ssq += (float)y[j][e] * (float)y[j][e];
        r_branch = rsqrtf(workgroup_sum(ssq, part[0]) / p.d + p.eps);
    }
    float s[VPT][8], ssq = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float t = 0.f;
            if (p.branch) {
                t = (float)y[j][e];
                if (p.gamma_post) t = t * r_branch * (float)gp[j][e];
                if (p.gate) t *= (float)g[j][e];
            }
            s[j][e] = fmaf(p.branch_scale, t, p.hidden_scale * (float)h[j][e]);
            if (in[j]) ssq += s[j][e] * s[j][e];
        }
        if (p.hidden_out && in[j]) {
            half8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (half_t)s[j][e];
            *reinterpret_cast<half8 *>(p.hidden_out + row + at[j]) = o;
        }
    }
    if (!p.x && !p.x8) return;
    const float r = rsqrtf(workgroup_sum(ssq, part[1]) / p.d + p.eps);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[j][e] = s[j][e] * r * (float)gm[j][e];
            top = fmaxf(top, fabsf(s[j][e]));
        }
        if (p.x && in[j]) {
            half8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (half_t)s[j][e];
            *reinterpret_cast<half8 *>(p.x + row + at[j]) = o;
        }
        if (p.x8) {
            top = row16_max(in[j] ? top : 0.f);
            // (a scale that is no normal number would not divide back)
            const float scale = top > 0.f ? fmaxf(top / kF8Max, FLT_MIN) : 1.f;
            int code[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float *v = s[j] + 4 * e;
                code[e] = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] / scale, v[1] / scale, 0, false);
                code[e] = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] / scale, v[3] / scale, code[e], true);
            }
            if (in[j]) {
                *reinterpret_cast<int2 *>(p.x8 + row + at[j]) = make_int2(code[0], code[1]);
                if ((at[j] & 127) == 0) p.x8_scales[(size_t)n * ((p.d + 127) / 128) + at[j] / 128] = scale;
            }
        }
    }
}

}  // namespace

hipError_t launch_block_norm(const BlockNormParams &p, hipStream_t s) {
    const int nvec = p.d / 8;
    const int vpt = nvec > 1024 ? 2 : 1;
    const int threads = ((nvec + vpt - 1) / vpt + kWave - 1) / kWave * kWave;
    if (vpt == 1)
        hipLaunchKernelGGL(block_norm_kernel<1>, dim3(p.N), dim3(threads), 0, s, p);
    else
        hipLaunchKernelGGL(block_norm_kernel<2>, dim3(p.N), dim3(threads), 0, s, p);
    return hipGetLastError();
}

}  // namespace specee
