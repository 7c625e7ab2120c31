// Rotary positions with one or several axes: queries and keys of a token turn by the same angles in every head.
//
// Bound by memory: 2 bytes in and 2 bytes out per value.  A block takes a token with all its heads, so that each angle (a product
// in 64 bits, a sine and a cosine) is computed once a token; the values are on their way meanwhile.  As many threads as the heads keep
// busy in whole rounds.  Measured: 8160 tokens with 72 heads of 128 56 us (5.4 TB/s; 64 us with 256 threads, a quarter of them idle in the last
// round), 2048 tokens with 64 heads 17.3 us, where the start of a block (positions, then angles, then the first store) counts.  Blocks that
// go on with another token, its values under way: 95 and 19 us, since fewer values are on their way.
#include "pd_rotate.cuh"

namespace pd {
namespace {

constexpr int kThreads = 256;

template <int D, bool BF16, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs a) {
    __shared__ float2 cs[D / 2];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the previous kernel drains
    turn_token<D, BF16, INTERLEAVED>(a.x, a.out, a.heads, blockIdx.x, a.r, cs, a.status, [](int &) { return true; });
}

template <int D, bool BF16>
pd_status launch(const RopeArgs &a, bool interleaved, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_tokens));
    cfg.blockDim = dim3(static_cast<unsigned>(turn_threads(a.heads[0] + a.heads[1], D, kThreads)));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    return cuda_ok(interleaved ? cudaLaunchKernelEx(&cfg, rope_kernel<D, BF16, true>, a) : cudaLaunchKernelEx(&cfg, rope_kernel<D, BF16, false>, a));
}

}  // namespace

pd_status launch_rope(const RopeArgs &a, bool interleaved, bool bf16, cudaStream_t stream) {
    if (a.head_dim == 128) return bf16 ? launch<128, true>(a, interleaved, stream) : launch<128, false>(a, interleaved, stream);
    return bf16 ? launch<64, true>(a, interleaved, stream) : launch<64, false>(a, interleaved, stream);
}

}  // namespace pd
