// Attention of a chunk of new tokens over the pages of its sequence: out_i = sum_j p_ij v_j, p_ij = exp(x_ij - lse_i), x_ij = scale q_i . k_j,
// lse_i = log sum_j exp(x_ij), over the rows j <= ctx + i.
//
// A warp a query row, four of the head's elements a lane, one pass over the rows with the running maximum and sum.
#include "goose_internal.cuh"

namespace goose {

constexpr int kChunkThreads = 256;

__global__ void __launch_bounds__(kChunkThreads)
chunk_attn_kernel(const ChunkAttn a, int32_t* __restrict__ status) {
    const int s = blockIdx.y, lane = threadIdx.x & 31;
    const int64_t r = (int64_t)blockIdx.x * (kChunkThreads / 32) + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    const int i = (int)(r / a.H), h = (int)(r - (int64_t)i * a.H), hk = h / (a.H / a.Hkv);
    const int nn = nodes_of(a.n_new, s, a.B), ctx = a.ctx_len[s];
    if (r == 0 && lane == 0 && nodes_bad(a.n_new, s, a.B)) atomicOr(&status[s], GOOSE_ST_BAD_NODES);
    if (i >= nn) return;
    bool bad = rows_outside(0, ctx, nn, a.pages.room(0));
    const size_t at = ((size_t)s * a.B + i) * a.H + h;
    const uint2 qv = *reinterpret_cast<const uint2*>(a.q + at * kHeadDim + 4 * lane);
    auto unpack = [](uint2 v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    };
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    unpack(qv, q);
    for (int j = 0; j <= ctx + i && !bad; ++j) {
        const int64_t row = a.pages.row(s, j);
        if (row < 0) { bad = true; break; }
        const size_t from = ((size_t)row * a.Hkv + hk) * kHeadDim + 4 * lane;
        float k[4], v[4];
        unpack(*reinterpret_cast<const uint2*>(a.k_cache + from), k);
        unpack(*reinterpret_cast<const uint2*>(a.v_cache + from), v);
        float x = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, w);
        x *= a.scale;
        const float m_new = fmaxf(m, x), old = m == -INFINITY ? 0.f : __expf(m - m_new), p = __expf(x - (m_new == -INFINITY ? 0.f : m_new));
        l = l * old + p;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * old + p * v[e];
        m = m_new;
    }
    const float inv = bad ? 0.f : 1.f / l;
    __nv_bfloat162 r2[2] = {__floats2bfloat162_rn(o[0] * inv, o[1] * inv), __floats2bfloat162_rn(o[2] * inv, o[3] * inv)};
    if (bad) r2[0] = r2[1] = __floats2bfloat162_rn(0.f, 0.f);
    *reinterpret_cast<uint2*>(a.out + at * kHeadDim + 4 * lane) = *reinterpret_cast<uint2*>(r2);
    if (a.lse && lane == 0) a.lse[at] = bad ? 0.f : m + logf(l);
    if (bad && lane == 0) atomicOr(&status[s], GOOSE_ST_BAD_ROWS);
}

cudaError_t launch_chunk_attn(goose_ctx* c, const ChunkAttn& a, cudaStream_t st) {
    if (a.S == 0) return cudaSuccess;
    const int64_t rows = (int64_t)a.B * a.H;
    cudaError_t e = launch_pdl(chunk_attn_kernel, dim3((unsigned)((rows + kChunkThreads / 32 - 1) / (kChunkThreads / 32)), a.S), dim3(kChunkThreads), 0, st, a,
                               c->status);
    c->launches++;
    return e;
}

cudaError_t init_chunk_kernels() { return load_kernels({(const void*)chunk_attn_kernel}); }

}  // namespace goose
