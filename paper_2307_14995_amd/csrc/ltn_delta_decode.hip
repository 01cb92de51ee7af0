// Gated delta rule, token by token (the first line of ltn_delta.h): the running state is read once, kept in registers over
// the call's tokens and written once; fp32 whatever the tensors' type.  Columns of a state are independent: a workgroup
// holds 32 of them, a thread eight rows of four.  With A = a S the state before the token's own term,
//
//     u = beta (v - A^T k),   S = A + k u^T,   o = scale (A^T q + (q . k) u),
//
// so both sums over rows are taken in one pass over A and meet once.
// Bound by HBM for a batch: 2048 states of 128 x 128 53.7 us (5.05 TB/s; 41 where the memory-side cache holds them); one
// sequence of 32 heads by the host's call, 5.6 us, of which the kernel takes 3.6.  Slices of 32 columns make four workgroups a
// state of 128 x 128, enough of them for one sequence.
#include "ltn_delta.h"

namespace ltn {
namespace {

constexpr int kCols = 32;

template <class T, int DK>
__global__ __launch_bounds__(DK)
void delta_decode_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, T* __restrict__ o,
                         float* __restrict__ kv, const float* __restrict__ g, const float* __restrict__ beta, float scale,
                         int Hk, int H, int steps, int Dv) {
    constexpr int TX = kCols / 4, TY = DK / TX, IT = DK / TY, NW = DK / 64;
    __shared__ float qs[2][DK], ks[2][DK];
    __shared__ float4 pk[2][NW][TX], pq[2][NW][TX];
    __shared__ float qk[2][NW];
    const int ns = Dv / kCols, chain = blockIdx.x / ns, col0 = (blockIdx.x - chain * ns) * kCols;
    const int tid = threadIdx.x, tx = tid % TX, ty = tid / TX, w = tid / 64;
    const int b = chain / H, h = chain - b * H;
    const size_t key_row = ((size_t)b * Hk + h / (H / Hk)) * steps, row = (size_t)chain * steps;
    float4* const S = (float4*)(kv + (size_t)chain * DK * Dv + col0) + tx;
    float4 s[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) s[it] = S[(size_t)(ty + TY * it) * (Dv / 4)];
    for (int step = 0; step < steps; ++step) {
        const int p = step & 1;
        const float qv = (float)q[(key_row + step) * DK + tid], kv1 = (float)k[(key_row + step) * DK + tid];
        qs[p][tid] = qv;
        ks[p][tid] = kv1;
        float dot = qv * kv1;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) dot += __shfl_xor(dot, d, 64);
        if (tid % 64 == 0) qk[p][w] = dot;
        const float a = expf(g[row + step]), bt = beta[row + step];
        const T* vp = v + (row + step) * Dv + col0 + 4 * tx;
        const float4 vv = {(float)vp[0], (float)vp[1], (float)vp[2], (float)vp[3]};
        __syncthreads();
        float4 ak = {0.f, 0.f, 0.f, 0.f}, aq = ak;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const float ki = ks[p][ty + TY * it], qi = qs[p][ty + TY * it];
            s[it].x *= a;
            s[it].y *= a;
            s[it].z *= a;
            s[it].w *= a;
            ak.x = fmaf(ki, s[it].x, ak.x);
            ak.y = fmaf(ki, s[it].y, ak.y);
            ak.z = fmaf(ki, s[it].z, ak.z);
            ak.w = fmaf(ki, s[it].w, ak.w);
            aq.x = fmaf(qi, s[it].x, aq.x);
            aq.y = fmaf(qi, s[it].y, aq.y);
            aq.z = fmaf(qi, s[it].z, aq.z);
            aq.w = fmaf(qi, s[it].w, aq.w);
        }
#pragma unroll
        for (int d = TX; d < 64; d *= 2) {
            ak.x += __shfl_xor(ak.x, d, 64);
            ak.y += __shfl_xor(ak.y, d, 64);
            ak.z += __shfl_xor(ak.z, d, 64);
            ak.w += __shfl_xor(ak.w, d, 64);
            aq.x += __shfl_xor(aq.x, d, 64);
            aq.y += __shfl_xor(aq.y, d, 64);
            aq.z += __shfl_xor(aq.z, d, 64);
            aq.w += __shfl_xor(aq.w, d, 64);
        }
        float both = qk[p][0];
        if constexpr (NW > 1) {
            if (tid % 64 < TX) {
                pk[p][w][tx] = ak;
                pq[p][w][tx] = aq;
            }
            __syncthreads();
            ak = pk[p][0][tx];
            aq = pq[p][0][tx];
#pragma unroll
            for (int i = 1; i < NW; ++i) {
                const float4 x = pk[p][i][tx], y = pq[p][i][tx];
                ak.x += x.x;
                ak.y += x.y;
                ak.z += x.z;
                ak.w += x.w;
                aq.x += y.x;
                aq.y += y.y;
                aq.z += y.z;
                aq.w += y.w;
                both += qk[p][i];
            }
        }
        const float4 u = {bt * (vv.x - ak.x), bt * (vv.y - ak.y), bt * (vv.z - ak.z), bt * (vv.w - ak.w)};
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const float ki = ks[p][ty + TY * it];
            s[it].x = fmaf(ki, u.x, s[it].x);
            s[it].y = fmaf(ki, u.y, s[it].y);
            s[it].z = fmaf(ki, u.z, s[it].z);
            s[it].w = fmaf(ki, u.w, s[it].w);
        }
        if (tid < TX) {
            T* const op = o + (row + step) * Dv + col0 + 4 * tx;
            op[0] = (T)(scale * fmaf(both, u.x, aq.x));
            op[1] = (T)(scale * fmaf(both, u.y, aq.y));
            op[2] = (T)(scale * fmaf(both, u.z, aq.z));
            op[3] = (T)(scale * fmaf(both, u.w, aq.w));
        }
        // (the next token's parity keeps its writes apart from these reads; the one after it waits at the barrier between)
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) S[(size_t)(ty + TY * it) * (Dv / 4)] = s[it];
}

template <class T, int DK>
hipError_t launch_t(const void* q, const void* k, const void* v, void* o, float* kv, const float* g, const float* beta,
                    float scale, int Bt, int Hk, int H, int steps, int Dv, hipStream_t stream) {
    hipLaunchKernelGGL((delta_decode_kernel<T, DK>), dim3((unsigned)((long long)Bt * H * (Dv / kCols))), dim3(DK), 0, stream,
                       (const T*)q, (const T*)k, (const T*)v, (T*)o, kv, g, beta, scale, Hk, H, steps, Dv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_decode(const void* q, const void* k, const void* v, void* o, float* kv, const float* g,
                               const float* beta, float scale, int Bt, int Hk, int H, int steps, int Dk, int Dv, int is_bf16,
                               hipStream_t stream) {
    auto launch = [&](auto f) { return f(q, k, v, o, kv, g, beta, scale, Bt, Hk, H, steps, Dv, stream); };
    if (Dk == 64) return is_bf16 ? launch(launch_t<__bf16, 64>) : launch(launch_t<float, 64>);
    return is_bf16 ? launch(launch_t<__bf16, 128>) : launch(launch_t<float, 128>);
}

}  // namespace ltn
