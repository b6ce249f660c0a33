// Matrix product in 8-bit floating point (e4m3) with a scale for each block of 128:
//     out[n][v] = sum over b of xs[n][b] * ws[v / 128][b] * (sum over i in block b of x[n][i] * w[v][i]).
// The sum of a block is one matrix instruction of 16 x 16 x 128 (or four of 32) into zeros; one multiply-add in fp32 folds it
// into the result with the product of its scales, so every block is scaled once, exactly as it was quantised.
// fp16 results take the codes as they are: the instruction aligns its 128 products before it adds them, which is off by 1e-5 to
// 5e-5 of their 2-norm, a tenth of what the result's own rounding is at that size.  fp32 results would show that: their codes become
// halves first (exact) and are multiplied by the fp16 instruction (off by 1e-7), at twice the time per product.
//
// Few rows of x are a stream over w: 1 x 32000 x 4096 takes 23.5 us and 60 x 128256 x 8192 in fp32 199 us, 5.6 and 5.3 TB/s of w
// (a kernel that only reads gets 7.1).  Every tile reads x again (the latter in tiles of 128 rows: 217 us, 197 without the loads
// of x), so higher tiles are taken where they leave no CU idle.  Many rows are bound by the overlap of a CU's loads with its
// products: 8192 x 8192 x 8192 takes 520 us in fp16 (2.11 PFLOP/s; 513 to 531 between runs), the products alone 415, the loads alone 400.
//
// A workgroup's tile goes through its elements block by block.  Loads go to LDS without registers, one to two blocks ahead; a
// meeting of the workgroup per block (two where x has one place less, see below) keeps them apart from the reads.
#include <algorithm>
#include <type_traits>

#include "../../include/specee.h"
#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;  // elements, or rows of w, that share a scale

// 32 codes of a row on a lane: pieces q and q + 4 of 16 in every block
union Codes {
    uintx4 piece[2];
    intx8 all;
    __device__ __forceinline__ Codes() {}
};

// The codes as halves (exact), eight to a register group
struct Halves {
    half8 part[4];
    __device__ __forceinline__ Halves() {}
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
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.all, x.all, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ floatx4 block_product(const Halves &w, const Halves &x) {
    floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.part[k], x.part[k], c, 0, 0, 0);
    return c;
}

// Floats of a part in the workspace: whole quads, so that each part begins at 16 bytes
__host__ __device__ constexpr size_t part_floats(int N, int V) { return ((size_t)N * V + 3) / 4 * 4; }

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

// 16 (4) bytes per lane from base + off to LDS at lds + 16 (4) * lane, without a stop in registers.  The compiler does not
// count these loads (with its own builtin it waits for all of them before any read of LDS): landed<n>() waits for all but the
// last n of them.
__device__ __forceinline__ void load_lds16(uint32_t lds, uint32_t off, const void *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
// (for what is read once)
__device__ __forceinline__ void load_lds16_once(uint32_t lds, uint32_t off, const void *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_lds4(uint32_t lds, uint32_t off, const void *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
// ... and for the wavefront's LDS traffic, then meets the workgroup
template <int N>
__device__ __forceinline__ void landed() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A workgroup's tile: WV by WN wavefronts, each with I * 16 rows of w by J * 16 of x
// ONCE: no other workgroup reads its rows of w (or w is small)
template <int WV_, int WN_, int I_, int J_, int BUFFERS, bool ONCE>
struct Tile {
    static constexpr int WV = WV_, WN = WN_, I = I_, J = J_;
    static constexpr bool once = ONCE;
    static constexpr int waves = WV * WN, threads = waves * kWave;
    static constexpr int rows = WV * I * 16, states = WN * J * 16;
    static constexpr int w_bytes = rows * kBlock, x_bytes = states * kBlock, groups = (states + 63) / 64;
    static constexpr int buffer = w_bytes + x_bytes + groups * 256;  // of one block, with the scales of x
    static constexpr int buffers = BUFFERS;
    static constexpr int w_loads = rows / 8 / waves, x_loads = states / 8 / waves;  // of a wavefront, 8 rows each
    static constexpr int loads = w_loads + x_loads + 1;
    static_assert(w_loads * waves * 8 == rows && x_loads * waves * 8 == states && 128 % (I * 16) == 0, "");
};

// Brings one block of a workgroup's tile to LDS.  A load brings eight rows, a row's eight pieces of 16 bytes in the order
// piece ^ (row % 8): the 16 rows that the lanes of an operand read then lie in different banks.
template <typename S>
struct Loader {
    const uint8_t *wbase, *xbase;
    const float *sbase;
    uint32_t woff[S::w_loads], xoff[S::x_loads], soff;
    uint32_t lds0;
    int d, piece, wave, lane;
    unsigned char *smem;

    __device__ __forceinline__ Loader(const MatmulF8Params &p, int v0, int n0, int wave_, int lane_, unsigned char *smem_)
        : d(p.d), wave(wave_), lane(lane_), smem(smem_) {
        lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
        const int sub = lane >> 3;
        piece = ((lane & 7) ^ sub) * 16;
        wbase = p.w + (size_t)v0 * p.d;
        xbase = p.x + (size_t)n0 * p.d;
#pragma unroll
        for (int i = 0; i < S::w_loads; ++i)
            woff[i] = (uint32_t)min((wave * S::w_loads + i) * 8 + sub, p.V - 1 - v0) * (uint32_t)p.d + piece;
#pragma unroll
        for (int i = 0; i < S::x_loads; ++i)
            xoff[i] = (uint32_t)min((wave * S::x_loads + i) * 8 + sub, p.N - 1 - n0) * (uint32_t)p.d + piece;
        // (a scale is loaded by every wavefront that has none of its own to load)
        sbase = p.xs + (size_t)n0 * p.blocks;
        soff = (uint32_t)min((wave % S::groups) * 64 + lane, p.N - 1 - n0) * (uint32_t)p.blocks * 4;
    }
    // Rows behind their ends hold zeros: a last block may be shorter
    template <int LOADS>
    __device__ __forceinline__ void short_block(int b, unsigned char *to, const uint8_t *base, const uint32_t (&off)[LOADS]) const {
        const int k0 = b * kBlock;
        const bool in = k0 + piece < d;
        uintx4 *dst = reinterpret_cast<uintx4 *>(to) + lane;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uintx4 v = *reinterpret_cast<const uintx4 *>(base + (in ? k0 + off[i] : 0u));
            if (!in) v = uintx4{0, 0, 0, 0};
            dst[(wave * LOADS + i) * 64] = v;
        }
    }
    __device__ __forceinline__ void load_w(int b, int slot) const {
        const int k0 = b * kBlock;
        if (k0 + kBlock > d) {
            short_block(b, smem + slot * S::buffer, wbase, woff);
            return;
        }
#pragma unroll
        for (int i = 0; i < S::w_loads; ++i) {
            const uint32_t to = lds0 + slot * S::buffer + (wave * S::w_loads + i) * 1024;
            if (S::once)
                load_lds16_once(to, woff[i], wbase + k0);
            else
                load_lds16(to, woff[i], wbase + k0);
        }
    }
    __device__ __forceinline__ void load_x(int b, int slot) const {
        const int k0 = b * kBlock;
        const uint32_t at = lds0 + slot * S::buffer + S::w_bytes;
        if (k0 + kBlock > d) {
            short_block(b, smem + slot * S::buffer + S::w_bytes, xbase, xoff);
        } else {
#pragma unroll
            for (int i = 0; i < S::x_loads; ++i) load_lds16(at + (wave * S::x_loads + i) * 1024, xoff[i], xbase + k0);
        }
        load_lds4(at + S::x_bytes + (wave % S::groups) * 256, soff, sbase + b);
    }
};

// The scales of 128 rows of w (a scalar load: a vector load would be waited for behind the tiles that are in flight)
typedef const __attribute__((address_space(4))) float *scalar_ptr;
__device__ __forceinline__ scalar_ptr row_scales(const MatmulF8Params &p, int v) {
    return (scalar_ptr)(uintptr_t)(p.ws + (size_t)(min(v, p.V - 1) >> 7) * p.blocks);
}

__device__ __forceinline__ Codes read_codes(const unsigned char *t, int i, int frag) {
    Codes o;
    o.piece[0] = *reinterpret_cast<const uintx4 *>(t + i * 16 * kBlock + frag);
    o.piece[1] = *reinterpret_cast<const uintx4 *>(t + i * 16 * kBlock + (frag ^ 64));
    return o;
}

template <typename T, int I, int J>
__device__ __forceinline__ void store_tile(const MatmulF8Params &p, const floatx4 (&acc)[I][J], int v0, int n0) {
    const bool parts = gridDim.z > 1;
    const int q = (threadIdx.x & 63) >> 4, c = threadIdx.x & 15;
    float *part = static_cast<float *>(p.workspace) + blockIdx.z * part_floats(p.N, p.V);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int n = n0 + j * 16 + c;
        if (n >= p.N) continue;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int v = v0 + i * 16 + 4 * q;
            if (v >= p.V) continue;
            if (parts)
                store_quad(part, (size_t)n * p.V + v, p.V - v, acc[i][j]);
            else
                store_quad(static_cast<T *>(p.out), (size_t)n * p.V + v, p.V - v, acc[i][j]);
        }
    }
}

// T: type of the result.  fp16 results take the codes as they are, fp32 results as halves.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, 2) void matmul_f8_kernel(MatmulF8Params p) {
    constexpr int I = S::I, J = S::J;
    typedef typename std::conditional<sizeof(T) == 4, Halves, Codes>::type Operand;
    extern __shared__ __attribute__((aligned(1024))) unsigned char f8_smem[];
    const int lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wv = wave / S::WN, wn = wave % S::WN;
    const int v0 = blockIdx.x * S::rows, n0 = blockIdx.y * S::states;
    const int b0 = (int)((long long)p.blocks * blockIdx.z / gridDim.z);
    const int b1 = (int)((long long)p.blocks * (blockIdx.z + 1) / gridDim.z);
    const Loader<S> load(p, v0, n0, wave, lane, f8_smem);
    // Rows of w that are read once: the workgroups begin at different elements and go round, since rows a power of
    // two apart have the same elements in few memory channels (60 states on 128256 x 8192, fp16 result: 226 -> 202 us).
    // The order is the same for all states of a call and every time; another N may take other tiles or parts, and so another order.
    const int turn = S::once ? (int)(blockIdx.x * 37u % (unsigned)(b1 - b0)) : 0;
    auto block = [&](int b) { return S::once && b + turn >= b1 ? b + turn - (b1 - b0) : b + turn; };

    floatx4 acc[I][J] = {};
    const int frag = c * kBlock + ((q ^ (c & 7)) << 4);
    const scalar_ptr ws = row_scales(p, v0 + wv * I * 16);
    float sw = ws[block(b0)];
    constexpr bool kTwo = S::buffers == 2;
    // Where x has one place less the workgroup meets once x is in registers.  Operands of w that are read together with it (512 x
    // 5120 x 5120, fp16 result: 35 us with none, 30.5 with four; fp32 results, whose operands take twice the registers, gain
    // nothing: 300 x 32000 x 4096 103 and 105), and the row of tiles before which the workgroup meets: wavefronts of eight
    // rows begin to multiply before (8192 x 8192 x 8192 fp16 540 -> 528 us; those of four lose, 30.5 -> 33.5).
    constexpr int kEarly = sizeof(T) == 4 ? 0 : I == 8 ? 2 : I < 4 ? I : 4;
    constexpr int kMeet = sizeof(T) == 2 && I == 8 ? 2 : 0;
#pragma unroll
    for (int k = 0; k < S::buffers - 1; ++k)
        if (b0 + k < b1) {
            load.load_x(block(b0 + k), k);
            load.load_w(block(b0 + k), k);
        }
    if (kTwo && b0 + 1 < b1) load.load_x(block(b0 + 1), 1);
    for (int b = b0; b < b1; ++b) {
        const int slot = (b - b0) % S::buffers;
        if (b + (kTwo ? 1 : S::buffers - 2) >= b1)
            landed<0>();
        else if (kTwo)
            landed<S::x_loads + 1>();  // the next block's x may be on its way
        else
            landed<(S::buffers - 2) * S::loads>();
        const unsigned char *buf = f8_smem + slot * S::buffer;
        const unsigned char *wt = buf + wv * I * 16 * kBlock, *xt = buf + S::w_bytes + wn * J * 16 * kBlock;
        const float *st = reinterpret_cast<const float *>(buf + S::w_bytes + S::x_bytes) + wn * J * 16 + c;
        float s[J];
        Operand x[J];
        Codes xc[J], wc[I];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            xc[j] = read_codes(xt, j, frag);
            s[j] = st[j * 16];
        }
#pragma unroll
        for (int i = 0; i < kEarly; ++i) wc[i] = read_codes(wt, i, frag);
        if (kTwo) {
            // x is in registers once all have read it: its place is free for the block after the next
            if (b + 1 < b1) load.load_w(block(b + 1), slot ^ 1);
            if (kMeet == 0) {
                meet();
                if (b + 2 < b1) load.load_x(block(b + 2), slot);
            }
        } else {
            const int ahead = b + S::buffers - 1;
            if (ahead < b1) {
                load.load_x(block(ahead), (ahead - b0) % S::buffers);
                load.load_w(block(ahead), (ahead - b0) % S::buffers);
            }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            x[j] = Operand(xc[j]);
            s[j] *= sw;
        }
        const float sw_next = ws[block(min(b + 1, b1 - 1))];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (i + kEarly < I) wc[i + kEarly] = read_codes(wt, i + kEarly, frag);
            if (kTwo && kMeet > 0 && i == kMeet) {
                __builtin_amdgcn_sched_barrier(0);
                meet();
                if (b + 2 < b1) load.load_x(block(b + 2), slot);
                __builtin_amdgcn_sched_barrier(0);
            }
            const Operand w(wc[i]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const floatx4 t = block_product(w, x[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s[j], t[e], acc[i][j][e]);
            }
        }
        sw = sw_next;
    }
    store_tile<T, I, J>(p, acc, v0 + wv * I * 16, n0 + wn * J * 16);
}

// Sums of the parts, in their order
template <typename T>
__global__ __launch_bounds__(256) void matmul_f8_join_kernel(const float *part, int parts, size_t stride, size_t n, T *out) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const int left = n - i < 4 ? (int)(n - i) : 4;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s)
        for (int e = 0; e < left; ++e) sum[e] += part[s * stride + i + e];
    store_quad(out, i, left, sum);
}

// ---- few states -------------------------------------------------------------------------------------------------------
// Up to 16 rows of x: a stream over w.  The elements are cut over the wavefronts of a workgroup, CPW blocks each, whose x
// stays in registers as codes; a tile is 16 rows of w, a unit one to four of them, and a wavefront has kAhead blocks of 16 rows
// (2 KB each) in flight at any time, across tiles and units.  Loads take whole 128-byte lines of eight rows with the
// non-temporal hint; two of them become an operand by exchanging halves of 16 lanes.  The wavefronts' sums meet in LDS once
// per unit and are added in ascending order of elements.
constexpr int kAhead = 4;
constexpr int kStreamBlocks = 64;  // of a pass: 16 wavefronts of 4

template <typename T, int CPW, bool WHOLE>
__global__ __launch_bounds__(1024) void matmul_f8_stream_kernel(MatmulF8Params p, int unit_tiles) {
    constexpr int RING = kAhead / CPW;  // tiles in flight
    typedef typename std::conditional<sizeof(T) == 4, Halves, Codes>::type Operand;
    extern __shared__ __attribute__((aligned(16))) floatx4 f8_sums[];  // [tile][wavefront][lane]
    const int lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int part0 = (int)((long long)p.blocks * blockIdx.y / gridDim.y);
    const int part1 = (int)((long long)p.blocks * (blockIdx.y + 1) / gridDim.y);
    const int first = part0 + wave * CPW;
    const int units = (p.V + 16 * unit_tiles - 1) / (16 * unit_tiles);

    // a lane's piece of a load: piece q + 4 * (c / 8) of row c % 8 (and 8 + c % 8)
    const int piece = (q + 4 * (c >> 3)) * 16, sub = c & 7;
    uintx4 ring[RING][CPW][2];
    // tile t of a unit, or of the one behind it
    auto load = [&](int unit, int next, int t, int k, uintx4 (&r)[2]) {
        const int row = (t < unit_tiles ? unit * unit_tiles + t : next * unit_tiles + t - unit_tiles) * 16, last = p.V - 1 - row;
        const uint8_t *base = p.w + (last < 0 ? (long long)p.V - 1 : (long long)row) * p.d + (size_t)first * kBlock;
        const bool have = WHOLE || (first + k < part1 && (first + k) * kBlock + piece < p.d);
        const int col = have ? k * kBlock + piece : -first * kBlock;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int off = max(min(sub + 8 * h, last), 0) * p.d + col;
            const uint8_t *at = WHOLE ? base + (uint32_t)off : base + off;
            r[h] = __builtin_nontemporal_load(reinterpret_cast<const uintx4 *>(at));
        }
    };
    int unit = blockIdx.x;
#pragma unroll
    for (int u = 0; u < RING; ++u)
#pragma unroll
        for (int k = 0; k < CPW; ++k) load(unit, unit, u, k, ring[u][k]);

    Codes x[CPW];
    float sx[CPW];
    bool in[CPW][2];  // whether a lane's pieces exist
#pragma unroll
    for (int k = 0; k < CPW; ++k) {
        const int b = first + k;
        const uint8_t *row = p.x + (size_t)min(c, p.N - 1) * p.d;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = b * kBlock + (q + 4 * h) * 16;
            in[k][h] = WHOLE || (b < part1 && at < p.d);
            uintx4 v = *reinterpret_cast<const uintx4 *>(row + (in[k][h] ? at : 0));
            if (!in[k][h]) v = uintx4{0, 0, 0, 0};
            x[k].piece[h] = v;
        }
        sx[k] = WHOLE || b < part1 ? p.xs[(size_t)min(c, p.N - 1) * p.blocks + min(b, part1 - 1)] : 0.f;
    }

    for (; unit < units; unit += gridDim.x) {
        const int next = min(unit + (int)gridDim.x, units - 1);
        const scalar_ptr ws = row_scales(p, unit * 16 * unit_tiles);
        float f[CPW];
#pragma unroll
        for (int k = 0; k < CPW; ++k) f[k] = sx[k] * ws[min(first + k, p.blocks - 1)];
#pragma unroll 1
        for (int t0 = 0; t0 < unit_tiles; t0 += RING) {
#pragma unroll
            for (int u = 0; u < RING; ++u) {
                floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < CPW; ++k) {
                    Codes w;
                    w.piece[0] = ring[u][k][0];
                    w.piece[1] = ring[u][k][1];
                    whole_lines(w.piece[0], w.piece[1]);
                    load(unit, next, t0 + u + RING, k, ring[u][k]);
                    if (!WHOLE) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (!in[k][h]) w.piece[h] = uintx4{0, 0, 0, 0};
                    }
                    Codes xk = x[k];
                    if (sizeof(T) == 4)  // the halves of x are formed again for every tile: kept, they would cost a workgroup per CU
                        asm volatile("" : "+v"(xk.all));
                    const floatx4 s = block_product(Operand(w), Operand(xk));
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = fmaf(f[k], s[e], acc[e]);
                }
                f8_sums[((t0 + u) * waves + wave) * kWave + lane] = acc;
            }
        }
        __syncthreads();
        for (int t = wave; t < unit_tiles; t += waves) {
            floatx4 sum = f8_sums[t * waves * kWave + lane];
            for (int w = 1; w < waves; ++w) sum += f8_sums[(t * waves + w) * kWave + lane];
            const int v = (unit * unit_tiles + t) * 16 + 4 * q;
            if (c < p.N && v < p.V) {
                if (gridDim.y > 1)
                    store_quad(static_cast<float *>(p.workspace) + blockIdx.y * part_floats(p.N, p.V), (size_t)c * p.V + v,
                               p.V - v, sum);
                else
                    store_quad(static_cast<T *>(p.out), (size_t)c * p.V + v, p.V - v, sum);
            }
        }
        __syncthreads();
    }
}

// The tiles that there are, rows of w by rows of x.  Up to 128 rows of x are one tile wide, and w a stream; up to 128 rows of w
// fit twice on a CU, where the one workgroup multiplies while the other waits; larger tiles read less per product.
template <int K>
struct TileOf;
template <> struct TileOf<0> { using type = Tile<4, 1, 2, 2, 3, true>; };   // 128 x 32
template <> struct TileOf<1> { using type = Tile<4, 1, 2, 4, 3, true>; };   // 128 x 64
template <> struct TileOf<2> { using type = Tile<4, 1, 4, 4, 3, true>; };   // 256 x 64
template <> struct TileOf<3> { using type = Tile<8, 1, 4, 4, 2, true>; };   // 512 x 64, fp16 results
template <> struct TileOf<4> { using type = Tile<2, 2, 4, 4, 2, true>; };   // 128 x 128
template <> struct TileOf<5> { using type = Tile<4, 2, 4, 4, 2, true>; };   // 256 x 128, fp16 results
template <> struct TileOf<6> { using type = Tile<2, 2, 4, 4, 2, false>; };  // 128 x 128
template <> struct TileOf<7> { using type = Tile<2, 4, 8, 3, 2, false>; };  // 256 x 192
template <> struct TileOf<8> { using type = Tile<2, 4, 8, 4, 2, false>; };  // 256 x 256

struct Shape {
    int tile, parts;  // tile -1: the stream for few states
};

Shape shape_of(int N, int V, int d, bool half) {
    const int blocks = (d + kBlock - 1) / kBlock;
    // few rows of w: the stream, whose workgroups cut the elements up and need no second launch to join them (one state, 1024 x
    // 5120 6.9 us against 10.9 in tiles, 5120 x 5120 10.9 / 12.5; 8192 x 8192 20.6 / 18.5, 32000 x 4096 26.3 / 24.3)
    if (N <= 16 && V <= 6144) return Shape{-1, (blocks + kStreamBlocks - 1) / kStreamBlocks};
    auto tiles = [&](int rows, int states) { return (long)((V + rows - 1) / rows) * ((N + states - 1) / states); };
    // What a block of 128 elements takes a CU, in 10 ns: two workgroups of a tile of 128 rows of w, one of them alone, one
    // workgroup of larger tiles.  Measured with the fp16 result and with the fp32 result, for up to 64 rows of x and up to 128 on
    // 131072, 65536 and 32768 x 4096 (60 rows, fp16: 50280 x 4096 51 -> 42 us in tiles of 256; 128256 x 8192 203 -> 187 in those
    // and 172 in tiles of 512; 32000 x 4096 27, in tiles of 256 39), for more at 8192 x 8192 x 8192 and 512 x 5120 x 5120.
    struct Option {
        int tile, rows, states, cost, alone;
    };
    static const Option options[2][9] = {
        {{0, 128, 32, 1, 1}, {1, 128, 64, 182, 92}, {2, 256, 64, 152, 0}, {3, 512, 64, 282, 0}, {4, 128, 128, 216, 124},
         {5, 256, 128, 200, 0}, {6, 128, 128, 123, 75}, {7, 256, 192, 155, 0}, {8, 256, 256, 207, 0}},
        {{0, 128, 32, 1, 1}, {1, 128, 64, 192, 107}, {2, 256, 64, 177, 0}, {-1, 0, 0, 0, 0}, {4, 128, 128, 265, 148},
         {-1, 0, 0, 0, 0}, {6, 128, 128, 195, 130}, {7, 256, 192, 260, 0}, {8, 256, 256, 370, 0}}};
    const int from = N <= 32 ? 0 : N <= 64 ? 1 : N <= 128 ? 4 : 6, to = N <= 32 ? 1 : N <= 64 ? 4 : N <= 128 ? 6 : 9;
    Shape best{-1, 1};
    long n = 0, least = 0;
    // Small matrices, which the caches hold: the smallest tiles that leave no CU with two (512 x 2048 x 2048, fp32 result: 21 us
    // in tiles of 128 x 128, 12 of 128 x 32; 1000 x 1000 x 1024 12.9 and 7.5; 60 x 2048 x 2048 11.8 and 9.8 of 128 x 64 and 128 x
    // 32, but 40 x 8192 x 8192 23 and 25)
    if (N > 32 && (long)V * d <= 24l << 20)
        for (int k = 1; k >= 0; --k)
            if (tiles(128, 32 << k) <= 256) {
                best.tile = k;
                n = tiles(128, 32 << k);
            }
    const bool small = best.tile >= 0;
    for (int k = from; k < to && !small; ++k) {
        const Option &o = options[half ? 0 : 1][k];
        if (o.rows == 0) continue;
        const long t = tiles(o.rows, o.states), rest = t % 512;
        const long cost = o.alone ? t / 512 * o.cost + (rest == 0 ? 0 : rest <= 256 ? o.alone : o.cost) : (t + 255) / 256 * o.cost;
        if (best.tile < 0 || cost < least) {
            least = cost;
            best.tile = o.tile;
            n = t;
        }
    }
    // parts of the elements while there is a CU for each and they are long enough (40 x 8192 x 8192, fp32 result: 49 us in one
    // part, 30 in two, 23 in four, 27 in eight)
    while (best.parts < 8 && n * best.parts * 2 <= 256 && blocks >= best.parts * 2 * 5) best.parts *= 2;
    return best;
}

template <typename T, int CPW, bool WHOLE>
hipError_t launch_stream(const MatmulF8Params &p, int parts, hipStream_t s) {
    const int blocks = (p.blocks + parts - 1) / parts, waves = (blocks + CPW - 1) / CPW;
    const auto kern = matmul_f8_stream_kernel<T, CPW, WHOLE>;
    // two workgroups of up to eight wavefronts fit on a CU; smaller units where larger ones would leave CUs without any
    // (1024 x 5120 by one state: 13.7 us in units of four, 6.9 of one)
    const int most = 256 * (waves > 8 ? 1 : 2), tiles = (p.V + 15) / 16;
    int unit = 4;
    while (unit > kAhead / CPW && (tiles + unit - 1) / unit * parts < most * 3 / 4) unit /= 2;
    const int units = (tiles + unit - 1) / unit, lds = unit * waves * kWave * (int)sizeof(floatx4);  // at most 64 KB
    hipLaunchKernelGGL(kern, dim3(units < most ? units : most, parts), dim3(waves * kWave), lds, s, p, unit);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_few(const MatmulF8Params &p, int parts, hipStream_t s) {
    const int blocks = (p.blocks + parts - 1) / parts;
    const int cpw = blocks <= 8 ? 1 : blocks <= 16 ? 2 : 4;
    const bool whole = p.d % (kBlock * cpw * parts) == 0;
    switch (cpw * 2 + whole) {
        case 2: return launch_stream<T, 1, false>(p, parts, s);
        case 3: return launch_stream<T, 1, true>(p, parts, s);
        case 4: return launch_stream<T, 2, false>(p, parts, s);
        case 5: return launch_stream<T, 2, true>(p, parts, s);
        case 8: return launch_stream<T, 4, false>(p, parts, s);
        default: return launch_stream<T, 4, true>(p, parts, s);
    }
}

template <typename T, int K>
hipError_t launch_tile(const MatmulF8Params &p, int parts, hipStream_t s) {
    using S = typename TileOf<K>::type;
    const auto kern = matmul_f8_kernel<T, S>;
    const int lds = S::buffers * S::buffer;
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    const dim3 grid((p.V + S::rows - 1) / S::rows, (p.N + S::states - 1) / S::states, parts);
    hipLaunchKernelGGL(kern, grid, dim3(S::threads), lds, s, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_shape(const MatmulF8Params &p, const Shape &sh, hipStream_t s) {
    hipError_t e = hipErrorInvalidValue;
    if constexpr (sizeof(T) == 2) {
        if (sh.tile == 3) e = launch_tile<T, 3>(p, sh.parts, s);
        if (sh.tile == 5) e = launch_tile<T, 5>(p, sh.parts, s);
    }
    switch (sh.tile) {
        case -1: e = launch_few<T>(p, sh.parts, s); break;
        case 0: e = launch_tile<T, 0>(p, sh.parts, s); break;
        case 1: e = launch_tile<T, 1>(p, sh.parts, s); break;
        case 2: e = launch_tile<T, 2>(p, sh.parts, s); break;
        case 4: e = launch_tile<T, 4>(p, sh.parts, s); break;
        case 6: e = launch_tile<T, 6>(p, sh.parts, s); break;
        case 7: e = launch_tile<T, 7>(p, sh.parts, s); break;
        case 8: e = launch_tile<T, 8>(p, sh.parts, s); break;
    }
    if (e != hipSuccess || sh.parts == 1) return e;
    const size_t n = (size_t)p.N * p.V;
    hipLaunchKernelGGL(matmul_f8_join_kernel<T>, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, s,
                       static_cast<const float *>(p.workspace), sh.parts, part_floats(p.N, p.V), n, static_cast<T *>(p.out));
    return hipGetLastError();
}

}  // namespace

// (for either type of the result)
size_t matmul_f8_workspace(int N, int V, int d) {
    if (N < 1) return 0;
    const int parts = std::max(shape_of(N, V, d, false).parts, shape_of(N, V, d, true).parts);
    return parts > 1 ? parts * part_floats(N, V) * sizeof(float) : 0;
}

// Every N from 1 to `most`: shape_of answers the same from one multiple of 32 (or 16) up to the next, so the largest N of each
// such range is asked for, from the largest that may have parts down to where eight of them could not need more.
size_t matmul_f8_workspace_up_to(int most, int V, int d) {
    size_t need = matmul_f8_workspace(most, V, d);
    const int high = (int)std::min<long>(most, 128l * 256 / ((V + 511) / 512));  // (no tile is larger, and parts have at most 128)
    for (int N = high / 32 * 32; N >= 32 && 8 * part_floats(N, V) * sizeof(float) > need; N -= 32)
        need = std::max(need, matmul_f8_workspace(N, V, d));
    return std::max(need, matmul_f8_workspace(std::min(most, 16), V, d));
}

hipError_t launch_matmul_f8(const MatmulF8Params &p, bool half, hipStream_t s) {
    const Shape sh = shape_of(p.N, p.V, p.d, half);
    return half ? launch_shape<half_t>(p, sh, s) : launch_shape<float>(p, sh, s);
}

}  // namespace specee
