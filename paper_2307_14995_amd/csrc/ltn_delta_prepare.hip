// Gated delta rule, per chunk of 64 tokens and value head (ltn_delta.h has the formulas): the decays, P = scale R (.) Q K^T
// and the inverse T' = (I + L diag(beta))^-1, its diagonal of ones left out.
//
// Q K^T and K K^T are taken transposed: a lane holds four neighbours of one token's row, which go to memory (P) and to LDS
// (L) as they are.  The inverse is taken in fp32 whatever the tensors' type: blocks of 16 on the diagonal by substitution, a
// lane a column; then pairs of blocks are merged, T21 = -T22 (A21 T11), to 32 and to 64 with fp32 matrix instructions.
// (Keys that repeat are why it is not a product of powers: those of L grow before they vanish.)
// Little work between loads and stores, in steps that wait for each other: what counts is how many workgroups a unit holds,
// four at 35 KB of LDS and 119 registers.  4 rows of 8192 tokens, 32 heads of 128 features, bf16: 161 us at 5.0 (gradients: T'
// in one part) to 5.8 TB/s of q, k, T' and P, a copy's rate; 47 chunks of 32 heads, two rounds of workgroups, 22 us.
#include "ltn_delta.h"

namespace ltn {
namespace {

constexpr int kThreads = 256;
constexpr int LA = kChunk + 4;             // fp32 rows of L and of the inverse

// 16 x 16 x 16, summed index 4 (lane / 16) + j
__device__ __forceinline__ f32x4 mma16x16(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ void store4(__bf16* p, const f32x4& x) { *(bf16x4*)p = to_bf16(x); }
__device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }

template <class T, int DK> struct PrepareLds {
    static constexpr int INV = kChunk * LA * 4, KB = Tile<T, DK>::BYTES > INV ? Tile<T, DK>::BYTES : INV;
    static constexpr int L = KB, BYTES = KB + INV;                       // K, later the inverse; L
};

constexpr double kLog2e = 1.4426950408889634;

template <class T, int DK>
__global__ __launch_bounds__(kThreads, 3)
void delta_prepare_kernel(DeltaArgs a) {
    typedef PrepareLds<T, DK> Lds;
    typedef typename El<T>::F F;
    __shared__ __attribute__((aligned(1024))) char lds[Lds::BYTES];
    __shared__ double G[kChunk];
    __shared__ float B[kChunk];
    float* const L = (float*)(lds + Lds::L);
    float* const Tm = (float*)lds;

    const int h = blockIdx.x % a.H, slot = blockIdx.x / a.H;
    DeltaSeq s;
    int chunk;
    if (!delta_find(a, slot, s, chunk)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, grp = lane >> 4;
    const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first + t0;
    const size_t gate_row = ((size_t)s.row * a.H + h) * a.N + s.first + t0;
    const size_t at = (size_t)slot * a.H + h;
    const unsigned base = lds_address(lds);
    const int r = 16 * w + m;              // the lane's token
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    // (in this order: loads come back in theirs, and the decays are worked on while K is still on its way)
    float gl = 0.f, b = 0.f;
    if (w == 0 && lane < rows) {
        gl = a.g[gate_row + lane];
        b = a.beta[gate_row + lane];
    }
    F q[DK / 32];
    {
        const T* const row = (const T*)a.q + (key_row + (r < rows ? r : 0)) * DK + 8 * grp;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) q[kb] = *(const F*)(row + 32 * kb);
    }
    TileFetch<T, DK, 4> k;
    k.fetch((const char*)a.k + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, base, w, lane);
    if (w == 0) {
        // log decays below -200 (exp underflows from -104 on) count as -200: sums of them stay finite, an infinite one's too
        double x = gl < -200.f ? -200.0 : (double)gl;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double y = __shfl_up(x, d, 64);
            if (lane >= d) x += y;
        }
        G[lane] = x * kLog2e;
        B[lane] = b;
        const double last = __shfl(x, 63, 64);
        float* const vec = a.vec + at * kVec;
        vec[lane] = expf((float)x);
        vec[kChunk + lane] = expf((float)(last - x));
        vec[2 * kChunk + lane] = b;
        vec[3 * kChunk + lane] = (float)x;
        vec[4 * kChunk + lane] = (float)(x - (double)(float)x);
    }
    if constexpr (sizeof(T) == 2) wait_dma<0>();
    k.put(base, w, lane);
    __syncthreads();

    f32x4 kk[4], qk[4];                    // row r, columns 16 ct + 4 grp + i
    {
        const RowReader<T, DK> own(base, r, lane), other(base, m, lane);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) kk[ct] = qk[ct] = zero;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            const F b = own.frag(0, kb);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const F f = other.frag(16 * ct * Tile<T, DK>::RB, kb);
                kk[ct] = mma(f, b, kk[ct]);
                qk[ct] = mma(f, q[kb], qk[ct]);
            }
        }
    }
    {
        constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
        T* const P = (T*)(a.p + at * kTile) + r * kChunk + 4 * grp;
        const double gr = G[r];
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
            const int c = 16 * ct + 4 * grp;
            f32x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float ratio = __builtin_amdgcn_exp2f((float)(gr - G[c + i]));    // (a rounding as large as that of an exponent to e)
                x[i] = r > c + i ? ratio * kk[ct][i] : 0.f;
                y[i] = r >= c + i && r < rows ? a.scale * ratio * qk[ct][i] : 0.f;
            }
            *(f32x4*)(L + r * LA + c) = x;
            store4(P + 16 * ct, y);
        }
    }
    __syncthreads();                       // L is there, and K is read: the inverse takes its place

    if (lane < 16) {                       // block w of the diagonal, column m: each row's result goes into all rows below at once
        const float* const Lb = L + 16 * w * LA + 16 * w;
        const float* const bb = B + 16 * w;
        f32x4 l[16][4];
        float x[16];
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            x[n] = n == m ? 1.f : 0.f;
#pragma unroll
            for (int i = 0; 4 * i < n; ++i) l[n][i] = *(const f32x4*)(Lb + n * LA + 4 * i);
        }
#pragma unroll
        for (int i = 0; i < 15; ++i) {
            const float y = -bb[i] * x[i];
#pragma unroll
            for (int n = i + 1; n < 16; ++n) x[n] = fmaf(l[n][i / 4][i % 4], y, x[n]);
        }
#pragma unroll
        for (int n = 0; n < 16; ++n) Tm[(16 * w + n) * LA + 16 * w + m] = x[n];
    }
    __syncthreads();
    // block (rt, ct) of L diag(beta): row m of the row tile, summed index 4 grp + j of the column tile
    auto block = [&](int rt, int ct) {
        f32x4 x = *(const f32x4*)(L + (16 * rt + m) * LA + 16 * ct + 4 * grp);
        return x * *(const f32x4*)(B + 16 * ct + 4 * grp);
    };
    auto rows_of = [&](int rt, int ct) { return *(const f32x4*)(Tm + (16 * rt + m) * LA + 16 * ct + 4 * grp); };
    auto cols_of = [&](int rt, int ct) {
        f32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = Tm[(16 * rt + 4 * grp + j) * LA + 16 * ct + m];
        return x;
    };
    auto put = [&](int rt, int ct, const f32x4& x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) Tm[(16 * rt + 4 * grp + i) * LA + 16 * ct + m] = -x[i];
    };
    const int half = w & 1;
    if (w < 2) {                           // 32 x 32 blocks: `half` of the diagonal
        const int b = 2 * half;
        const f32x4 M = mma16x16(block(b + 1, b), cols_of(b, b), zero);
        put(b + 1, b, mma16x16(rows_of(b + 1, b + 1), M, zero));
    }
    __syncthreads();
    {                                      // the whole: 16 columns, row tile 2 or 3
        const int rt = 2 + (w >> 1);
        f32x4 M[2], x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            M[i] = mma16x16(block(2 + i, 1), cols_of(1, half), zero);
            if (half == 0) M[i] = mma16x16(block(2 + i, 0), cols_of(0, 0), M[i]);
        }
        x = mma16x16(rows_of(rt, 2), M[0], zero);
        if (rt == 3) x = mma16x16(rows_of(3, 3), M[1], x);
        put(rt, half, x);
    }
    __syncthreads();
    constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
#pragma unroll
    for (int i = 0; i < 2; ++i) {          // (above the diagonal's blocks nothing was written)
        const int n = 32 * i + (tid >> 3), c = 8 * (tid & 7);
        f32x4 x = zero, y = zero;
        if (c <= (n | 15)) {
            x = *(const f32x4*)(Tm + n * LA + c);
            y = *(const f32x4*)(Tm + n * LA + c + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j >= n) x[j] = 0.f;
                if (c + 4 + j >= n) y[j] = 0.f;
            }
        }
        const F f = frag_of<T>(x, y);
        *(F*)((T*)(a.tq + at * kTile) + n * kChunk + c) = f;
        if constexpr (sizeof(T) == 2)
            if (a.tl) *(F*)((T*)(a.tl + at * kTile) + n * kChunk + c) = rest_of(f, x, y);
    }
}

template <class T, int DK>
hipError_t launch_t(const DeltaArgs& a, hipStream_t stream) {
    static_assert(PrepareLds<T, DK>::BYTES <= 150 * 1024, "LDS");
    hipLaunchKernelGGL((delta_prepare_kernel<T, DK>), dim3((unsigned)(a.slots * (long long)a.H)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_prepare(const DeltaArgs& a, int Dk, int is_bf16, hipStream_t stream) {
    if (Dk == 64) return is_bf16 ? launch_t<__bf16, 64>(a, stream) : launch_t<float, 64>(a, stream);
    return is_bf16 ? launch_t<__bf16, 128>(a, stream) : launch_t<float, 128>(a, stream);
}

}  // namespace ltn
