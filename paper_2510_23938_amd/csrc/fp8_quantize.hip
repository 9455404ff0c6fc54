// fp8_quantize.hip -- the operators whose output is codes and scales: a
// matrix's quantisation by rows or blocks, the root-mean-square norm with the
// residual's addition, and silu(gate) * up (hv_fp8.h has the formulas).
//
// All of them read and write each element once and are bound by HBM, where a copy
// reaches 5.1 TB/s (bfloat16): norm with residual of 16384 x 8192 182 us (5.2 TB/s), gate of
// 2048 x 28672 51 us (5.7), quantisation of 28672 x 8192 by blocks 150 us (4.7); one
// row of 8192 takes 4 us, a launch and two trips to memory.  A lane holds 8
// consecutive columns (16 bytes of a 16-bit type), so 16 lanes, one DPP row, hold a
// group of 128: its largest magnitude is four rotations of the row away, without LDS.
// Values stay in 32 bits until the one rounding to codes (and of h to its type).
#include <type_traits>

#include "fp8_device.h"
#include "hv_kernels.h"

namespace hv {
namespace {

constexpr uint32_t kMaxGrid = 1u << 20;  // workgroups of a launch; longer work loops

__device__ __forceinline__ uint32_t valid_of(uint32_t col, uint32_t cols) { return col < cols ? cols - col : 0; }

// ---------------------------------------------------------------------------
// element-wise operators, quantised by rows

template <typename T>
struct RowsOf {  // the matrix itself
    const T* x;
    uint64_t ld;
    __device__ __forceinline__ void get(uint64_t row, uint32_t col, uint32_t valid, float (&y)[8]) const {
        load_eight(x + row * ld + col, valid, y);
    }
};

template <typename T>
struct GatedOf {  // gate / (1 + exp(-gate)) * up
    const T* gate;
    const T* up;
    uint64_t ld_gate, ld_up;
    __device__ __forceinline__ void get(uint64_t row, uint32_t col, uint32_t valid, float (&y)[8]) const {
        float u[8];
        const T *const g = gate + row * ld_gate + col, *const f = up + row * ld_up + col;
        if (valid >= 8) {  // one branch: both are asked for before either is waited for
            load_eight(g, 8, y);
            load_eight(f, 8, u);
        } else {
            load_eight(g, valid, y);
            load_eight(f, valid, u);
        }
        // Where exp(-gate) comes near 2^128 its reciprocal is subnormal, which the reciprocal
        // instruction does not give, and from there on 1 + exp(-gate) is exp(-gate) in 32 bits: y is then
        // gate * up * exp(gate), by halves of the exponent, so that large factors up keep it in range.  A
        // branch that few vectors take: one comparison of eight gates' least.
        float low = y[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) low = fminf(low, y[i]);
        if (low < -87.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float half = expf(0.5f * y[i]);
                y[i] = y[i] < -87.0f ? (y[i] * half) * (u[i] * half) : ordinary(y[i], u[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = ordinary(y[i], u[i]);
        }
    }
    // For gates from -87 on: the reciprocal instruction is within one unit in the last place of a normal
    // result; a division takes ten instructions more (2048 x 28672: a quarter more time).
    static __device__ __forceinline__ float ordinary(float gate, float up) {
        return gate * __builtin_amdgcn_rcpf(1.0f + __expf(-gate)) * up;
    }
};

// blockDim.x lanes (a multiple of 16) along a row, blockDim.y rows.
template <typename Src>
__global__ void __launch_bounds__(256) rows_kernel(Src src, uint32_t rows, uint32_t cols, uint8_t* __restrict__ codes,
                                                   uint64_t ld_codes, float* __restrict__ scales) {
    const uint32_t groups = (cols + kFp8Group - 1) / kFp8Group;
    const uint32_t col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
    if (col / kFp8Group >= groups) return;  // whole DPP rows leave
    const uint32_t valid = valid_of(col, cols);
    for (uint64_t row = (uint64_t)blockIdx.y * blockDim.y + threadIdx.y; row < rows;
         row += (uint64_t)gridDim.y * blockDim.y) {
        float y[8];
        src.get(row, col, valid, y);
        const float scale = fp8_scale(row16_max(finite_largest(y)));
        store_codes(codes + row * ld_codes + col, valid, fp8_codes(y, scale));
        if (threadIdx.x % 16 == 0) scales[row * groups + col / kFp8Group] = scale;
    }
}

template <typename Src>
hipError_t launch_rows(const Src& src, uint64_t rows, uint64_t cols, uint8_t* codes, uint64_t ld_codes, float* scales,
                       hipStream_t s) {
    const uint32_t lanes = (uint32_t)((cols + 7) / 8);
    // as many lanes as divide the row evenly (1777 x 4104: three times 176; 30000 x 300 11.9
    // us, 13.9 with a power of two)
    const uint32_t across = (lanes + 255) / 256, tx = ((lanes + across - 1) / across + 15) / 16 * 16;
    const dim3 block(tx, 256 / tx);
    const uint64_t gy = (rows + block.y - 1) / block.y;
    const dim3 grid(across, (uint32_t)(gy < 65535 ? gy : 65535));
    rows_kernel<Src><<<grid, block, 0, s>>>(src, (uint32_t)rows, (uint32_t)cols, codes, ld_codes, scales);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// quantisation by blocks: a workgroup holds a block of 128 x 128 in registers

template <typename T>
__global__ void __launch_bounds__(256) blocks_kernel(const T* __restrict__ x, uint64_t ld, uint32_t rows,
                                                     uint32_t cols, uint8_t* __restrict__ codes, uint64_t ld_codes,
                                                     float* __restrict__ scales, uint32_t groups, uint64_t n_blocks) {
    __shared__ float part[4];
    const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (uint64_t b = blockIdx.x; b < n_blocks; b += gridDim.x) {
        const uint64_t row0 = b / groups * kFp8Group + ty;
        const uint32_t col = (uint32_t)(b % groups) * kFp8Group + tx * 8;
        const uint32_t valid = valid_of(col, cols);
        float y[8][8], m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t row = row0 + 16 * i;
            load_eight(x + (row < rows ? row : 0) * ld + col, row < rows ? valid : 0, y[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_largest(y[i]));
#pragma unroll
        for (int w = 32; w > 0; w /= 2) m = fmaxf(m, __shfl_xor(m, w));
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
        __syncthreads();
        const float scale = fp8_scale(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t row = row0 + 16 * i;
            if (row < rows) store_codes(codes + row * ld_codes + col, valid, fp8_codes(y[i], scale));
        }
        if (threadIdx.x == 0) scales[b] = scale;
    }
}

// ---------------------------------------------------------------------------
// root-mean-square norm

// Sum over the blockDim.x lanes of a row, in all of them: within a wave by
// shuffles, across waves (then the workgroup has one row) through LDS.
__device__ __forceinline__ float row_sum(float v, float* part) {
    const uint32_t width = blockDim.x < 64 ? blockDim.x : 64;
    for (uint32_t w = width / 2; w > 0; w /= 2) v += __shfl_xor(v, (int)w);
    if (blockDim.x <= 64) return v;
    __syncthreads();  // the last row's readers are done
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    const uint32_t waves = blockDim.x / 64;
    float sum = 0.0f;
    for (uint32_t i = 0; i < waves; ++i) sum += part[i];
    return sum;
}

// V x blockDim.x lanes of 8 columns cover a row, which stays in registers
// between the sum of its squares and the output.  V = 0: a longer row, read
// twice.  residual_out may be x or residual: every element is read by the lane that
// writes it, and written after the last read of it.
template <typename T, int V, bool kResidual>
__global__ void __launch_bounds__(1024) norm_kernel(const T* x, uint64_t ld_x, const T* residual, uint64_t ld_residual,
                                                    const T* __restrict__ weight, float eps, uint32_t rows,
                                                    uint32_t cols, T* residual_out, uint64_t ld_out,
                                                    uint8_t* __restrict__ codes, uint64_t ld_codes,
                                                    float* __restrict__ scales) {
    __shared__ float part[16];
    constexpr int kUnroll = V > 0 ? V : 1;
    const uint32_t groups = (cols + kFp8Group - 1) / kFp8Group;
    const uint32_t step = blockDim.x * 8;
    const uint32_t trips = V > 0 ? V : (cols + step - 1) / step;
    const uint32_t tile = gridDim.x * blockDim.y;
    for (uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y; row < rows; row += tile) {
        auto sum_at = [&](uint32_t col, uint32_t valid, float (&h)[8]) {
            load_eight(x + row * ld_x + col, valid, h);
            if (kResidual) {
                float r[8];
                load_eight(residual + row * ld_residual + col, valid, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += r[i];
            }
        };
        float h[kUnroll][8];
        float squares = 0.0f;
#pragma unroll kUnroll
        for (uint32_t t = 0; t < trips; ++t) {
            const uint32_t col = t * step + threadIdx.x * 8;
            float(&e)[8] = h[V > 0 ? t : 0];
            sum_at(col, valid_of(col, cols), e);
#pragma unroll
            for (int i = 0; i < 8; ++i) squares = fmaf(e[i], e[i], squares);
        }
        const float mean = row_sum(squares, part) / (float)cols;
        const float factor = 1.0f / sqrtf(mean + eps);
#pragma unroll kUnroll
        for (uint32_t t = 0; t < trips; ++t) {
            const uint32_t col = t * step + threadIdx.x * 8;
            if (col / kFp8Group >= groups) break;  // whole DPP rows leave
            const uint32_t valid = valid_of(col, cols);
            float(&e)[8] = h[V > 0 ? t : 0];
            if (V == 0) sum_at(col, valid, e);
            if (kResidual) store_eight(residual_out + row * ld_out + col, valid, e);
            float y[8];
            load_eight(weight + col, valid, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= e[i] * factor;
            const float scale = fp8_scale(row16_max(finite_largest(y)));
            store_codes(codes + row * ld_codes + col, valid, fp8_codes(y, scale));
            if (threadIdx.x % 16 == 0) scales[row * groups + col / kFp8Group] = scale;
        }
    }
}

template <typename T, bool kResidual>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    const uint32_t lanes = (uint32_t)((a.cols + 7) / 8);
    // two vectors a lane: more workgroups on a compute unit, so that some load while
    // others wait at their row's sum (16384 x 8192 with a residual: 1024 lanes 270 us,
    // 512 210, 256 230)
    uint32_t tx = 16;
    while (tx < 1024 && 2 * tx < lanes) tx *= 2;
    const dim3 block(tx, tx <= 64 ? 256 / tx : 1);  // see row_sum
    const uint64_t need = (a.rows + block.y - 1) / block.y;
    const uint32_t grid = (uint32_t)(need < kMaxGrid ? need : kMaxGrid);
    auto run = [&](auto kernel) {
        kernel<<<grid, block, 0, s>>>((const T*)a.x, a.ld_x, (const T*)a.residual, a.ld_residual, (const T*)a.weight,
                                      a.eps, (uint32_t)a.rows, (uint32_t)a.cols, (T*)a.residual_out, a.ld_out, a.codes,
                                      a.ld_codes, a.scales);
        return hipGetLastError();
    };
    if (lanes <= tx) return run(norm_kernel<T, 1, kResidual>);
    if (lanes <= 2 * tx) return run(norm_kernel<T, 2, kResidual>);
    if (lanes <= 3 * tx) return run(norm_kernel<T, 3, kResidual>);
    if (lanes <= 4 * tx) return run(norm_kernel<T, 4, kResidual>);
    return run(norm_kernel<T, 0, kResidual>);
}

// f(a pointer to the element type) for a type code that the caller has checked.
template <typename F>
hipError_t by_type(int type, F f) {
    switch (type) {
        case kTypeBf16: return f((__bf16*)nullptr);
        case kTypeF16: return f((_Float16*)nullptr);
        default: return f((float*)nullptr);
    }
}

}  // namespace

hipError_t launch_fp8_quantize(int type, const void* x, uint64_t ld_x, uint64_t rows, uint64_t cols, bool blocks,
                               uint8_t* codes, uint64_t ld_codes, float* scales, hipStream_t s) {
    return by_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (!blocks) return launch_rows(RowsOf<T>{(const T*)x, ld_x}, rows, cols, codes, ld_codes, scales, s);
        const uint64_t groups = (cols + kFp8Group - 1) / kFp8Group;
        const uint64_t n = (rows + kFp8Group - 1) / kFp8Group * groups;
        blocks_kernel<T><<<(uint32_t)(n < kMaxGrid ? n : kMaxGrid), 256, 0, s>>>(
            (const T*)x, ld_x, (uint32_t)rows, (uint32_t)cols, codes, ld_codes, scales, (uint32_t)groups, n);
        return hipGetLastError();
    });
}

hipError_t launch_fp8_gated(int type, const void* gate, uint64_t ld_gate, const void* up, uint64_t ld_up,
                            uint64_t rows, uint64_t cols, uint8_t* codes, uint64_t ld_codes, float* scales,
                            hipStream_t s) {
    return by_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch_rows(GatedOf<T>{(const T*)gate, (const T*)up, ld_gate, ld_up}, rows, cols, codes, ld_codes,
                           scales, s);
    });
}

hipError_t launch_fp8_rms_norm(int type, const NormArgs& a, hipStream_t s) {
    return by_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return a.residual ? launch_norm<T, true>(a, s) : launch_norm<T, false>(a, s);
    });
}

}  // namespace hv
