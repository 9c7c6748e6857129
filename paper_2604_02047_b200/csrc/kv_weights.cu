// The attention that every cached row got from a chunk's tokens: W[s][hk][j] += sum_{i, h in group hk} exp(x_ihj - lse_ih), x_ihj = scale q_ih . k_j,
// over the tokens i >= j - ctx.
//
// A warp a row of a head, four of the head's elements a lane.
#include "goose_internal.cuh"

namespace goose {

constexpr int kWeightThreads = 256;

__global__ void __launch_bounds__(kWeightThreads)
kv_weights_kernel(const KvWeights a, int32_t* __restrict__ status) {
    const int s = blockIdx.z, hk = blockIdx.y, lane = threadIdx.x & 31, g = a.H / a.Hkv;
    pdl_wait();
    pdl_trigger();
    const int nn = nodes_of(a.n_new, s, a.B), ctx = a.ctx_len[s];
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0 && nodes_bad(a.n_new, s, a.B)) atomicOr(&status[s], GOOSE_ST_BAD_NODES);
    if (nn == 0) return;
    if (rows_outside(0, ctx, nn, a.pages.room(a.ldw))) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(&status[s], GOOSE_ST_BAD_ROWS);
        return;
    }
    const int warps = gridDim.x * (kWeightThreads / 32);
    auto unpack = [](uint2 v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    };
    for (int j = blockIdx.x * (kWeightThreads / 32) + (threadIdx.x >> 5); j < ctx + nn; j += warps) {
        const int64_t row = a.pages.row(s, j);
        if (row < 0) {
            if (lane == 0) atomicOr(&status[s], GOOSE_ST_BAD_ROWS);
            continue;
        }
        float k[4], q[4], sum = 0.f;
        unpack(*reinterpret_cast<const uint2*>(a.k_cache + ((size_t)row * a.Hkv + hk) * kHeadDim + 4 * lane), k);
        for (int i = max(j - ctx, 0); i < nn; ++i)
            for (int u = 0; u < g; ++u) {
                const size_t at = ((size_t)s * a.B + i) * a.H + hk * g + u;
                unpack(*reinterpret_cast<const uint2*>(a.q + at * kHeadDim + 4 * lane), q);
                float x = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
                for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, w);
                const float lse = a.lse[at];
                if (lse != -INFINITY) sum += __expf(x * a.scale - lse);
            }
        if (lane == 0) a.row_weight[((size_t)s * a.Hkv + hk) * a.ldw + j] += sum;
    }
}

cudaError_t launch_kv_weights(goose_ctx* c, const KvWeights& a, cudaStream_t st) {
    if (a.S == 0) return cudaSuccess;
    const int64_t room = a.pages.room(a.ldw), per = kWeightThreads / 32;
    const dim3 grid((unsigned)((room + per - 1) / per < 1024 ? (room + per - 1) / per : 1024), a.Hkv, a.S);
    cudaError_t e = launch_pdl(kv_weights_kernel, grid, dim3(kWeightThreads), 0, st, a, c->status);
    c->launches++;
    return e;
}

cudaError_t init_weights_kernels() { return load_kernels({(const void*)kv_weights_kernel}); }

}  // namespace goose
