// Rotary positions with several axes: pair i of a head turns by positions[axis(i)][token] * frequencies[i].
#include <cuda_runtime.h>

#include "decode_common.cuh"
#include "decode_step.h"
#include "epilogue.cuh"

namespace huffllm {

// The axis of pair i where the axes' pairs are dealt in turn: rounds of those axes that have pairs left.
__device__ __forceinline__ uint32_t axis_in_turn(const RotaryArgs &A, uint32_t i) {
    uint32_t done = 0;                                   // pairs that an axis still in the game has had
    for (;;) {
        uint32_t live = 0, least = 0xFFFFFFFFu;
        for (uint32_t a = 0; a < A.axes; ++a)
            if (A.sections[a] > done) {
                ++live;
                least = min(least, A.sections[a]);
            }
        if (live == 0) return 0;
        const uint32_t dealt = (least - done) * live;    // until the next axis has had all of its pairs
        if (i < dealt) {
            uint32_t k = i % live;
            for (uint32_t a = 0; a < A.axes; ++a)
                if (A.sections[a] > done && k-- == 0) return a;
        }
        i -= dealt;
        done = least;
    }
}
__device__ __forceinline__ uint32_t axis_of(const RotaryArgs &A, uint32_t i) {
    if (A.in_turn) return axis_in_turn(A, i);
    uint32_t a = 0;
    while (a + 1 < A.axes && i >= A.sections[a]) i -= A.sections[a++];
    return a;
}

// Sine and cosine of position * frequency.  The product is taken in turns and in 64 bits: 2^31 turns are off by 2^-23 of one at most,
// those of a position of a million by 2^-33, and what is left behind the whole turns is exact in either.
__device__ __forceinline__ float2 turn_of(int32_t position, float frequency) {
    const double turns = (double)position * (double)frequency * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    return make_float2(c, s);
}

template <bool F16>
__global__ void __launch_bounds__(128) rotary_kernel(const __grid_constant__ RotaryArgs A) {
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t token = blockIdx.x, pairs = A.rot / 2;
    for (uint32_t i = threadIdx.x; i < (A.dim - A.rot) + pairs; i += blockDim.x) {
        const bool turned = i < pairs;
        const float2 cs = turned ? turn_of(__ldcg(A.positions + (uint64_t)axis_of(A, i) * A.tokens + token), __ldcg(A.frequencies + i)) : make_float2(1, 0);
        const uint32_t a = !turned ? A.rot + i - pairs : A.neighbours ? 2 * i : i, b = !turned ? a : A.neighbours ? 2 * i + 1 : i + pairs;
        for (int w = 0; w < 2; ++w) {
            const uint16_t *in = A.in[w] + token * A.in_stride[w];
            uint16_t *out = A.out[w] + token * A.out_stride[w];
            for (uint32_t h = 0; h < A.heads[w]; ++h) {
                const uint16_t xa = __ldcg(in + h * A.dim + a), xb = __ldcg(in + h * A.dim + b);
                if (!turned) {
                    out[h * A.dim + a] = xa;
                    continue;
                }
                const float va = widen16<F16>(xa), vb = widen16<F16>(xb);
                out[h * A.dim + a] = round16<F16>(va * cs.x - vb * cs.y);
                out[h * A.dim + b] = round16<F16>(vb * cs.x + va * cs.y);
            }
        }
    }
}

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t stream) {
    return launch_behind(a.fp16 ? rotary_kernel<true> : rotary_kernel<false>, dim3(a.tokens), 128, 0, stream, a);
}

}  // namespace huffllm
