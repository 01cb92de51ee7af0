// Gated delta rule, per chunk of 64 tokens and value head (ltn_delta.h has the formulas): the decays, P = scale R (.) Q K^T
// and the inverse T' = (I + L diag(beta))^-1 (for gradients T = (I + diag(beta) L)^-1 too), its diagonal of ones left out.
//
// The inverse is taken in fp32 whatever the tensors' type: blocks of 16 on the diagonal by substitution, a lane a column;
// then pairs of blocks are merged, T21 = -T22 (A21 T11), to 32 and to 64 with fp32 matrix instructions.  (Substitution and
// merging are as exact for keys that are alike, where powers of L grow before they vanish.)
#include "ltn_delta.h"

namespace ltn {
namespace {

constexpr int kThreads = 256;
constexpr int LA = kChunk + 4;             // fp32 rows of L and of the inverses

// 16 x 16 x 16: A's element (m, k) at a[m * LA + k], summed index 4 (lane / 16) + j
__device__ __forceinline__ f32x4 mma16x16(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

template <class T> __device__ __forceinline__ void store8(T* p, const f32x4& x, const f32x4& y) {
    *(typename El<T>::F*)p = frag_of<T>(x, y);
}

// Row r, columns c .. c + 7 of a tile of 64 x 64: hi in the tensors' type, and what rounding left in `lo` (bf16)
template <class T> __device__ __forceinline__ void store_tile8(T* hi, T* lo, int r, int c, const float* src) {
    const f32x4 x = *(const f32x4*)(src + r * LA + c), y = *(const f32x4*)(src + r * LA + c + 4);
    store8<T>(hi + r * kChunk + c, x, y);
    if constexpr (sizeof(T) == 2) {
        if (lo) *(bf16x8*)(lo + r * kChunk + c) = rest_of(frag_of<T>(x, y), x, y);
    }
}

template <class T, int DK, bool BWD>
__global__ __launch_bounds__(kThreads)
void delta_prepare_kernel(DeltaArgs a) {
    constexpr int LD = DK + El<T>::PAD;
    __shared__ __attribute__((aligned(16))) char lds[2 * kChunk * LD * sizeof(T) + (BWD ? 3 : 2) * kChunk * LA * sizeof(float)];
    T* const K = (T*)lds;
    T* const Q = K + kChunk * LD;
    float* const L = (float*)(Q + kChunk * LD);
    float* const inv = L + kChunk * LA;    // T', and behind it T
    float* const P = (float*)lds;          // in K and Q's place once they have been read
    __shared__ double G[kChunk];
    __shared__ float B[kChunk];
    static_assert(2 * kChunk * LD * sizeof(T) >= kChunk * LA * sizeof(float), "P takes K and Q's place");

    const int h = blockIdx.x % a.H, slot = blockIdx.x / a.H;
    DeltaSeq s;
    int chunk;
    if (!delta_find(a, slot, s, chunk)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = lane & 15, grp = lane >> 4;
    const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first + t0;
    const size_t gate_row = ((size_t)s.row * a.H + h) * a.N + s.first + t0;
    const size_t at = (size_t)slot * a.H + h;

    load_tile<T, LD, DK, kThreads>(K, (const T*)a.k + key_row * DK, DK, rows, tid);
    load_tile<T, LD, DK, kThreads>(Q, (const T*)a.q + key_row * DK, DK, rows, tid);
    if (w == 0) {
        // log decays below -200 (exp underflows from -104 on) count as -200: sums of them stay finite, an infinite one's too
        double x = 0.0;
        if (lane < rows) {
            const float gl = a.g[gate_row + lane];
            x = gl < -200.f ? -200.0 : (double)gl;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double y = __shfl_up(x, d, 64);
            if (lane >= d) x += y;
        }
        G[lane] = x;
        B[lane] = lane < rows ? a.beta[gate_row + lane] : 0.f;
        const double last = __shfl(x, 63, 64);
        float* const vec = a.vec + at * kVec;
        vec[lane] = expf((float)x);
        vec[kChunk + lane] = expf((float)(last - x));
        vec[2 * kChunk + lane] = B[lane];
        vec[3 * kChunk + lane] = (float)x;
        vec[4 * kChunk + lane] = (float)(x - (double)(float)x);
    }
    for (int i = tid; i < (BWD ? 2 : 1) * kChunk * LA; i += kThreads) inv[i] = 0.f;
    __syncthreads();

    // rows 16 w .. +15 of K K^T and Q K^T, columns up to the diagonal
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        kk[ct] = qk[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (ct > w) continue;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            const auto b = row_frag_p<T, LD>(K, 16 * ct + m, kb, lane);
            kk[ct] = mma(row_frag_p<T, LD>(K, 16 * w + m, kb, lane), b, kk[ct]);
            qk[ct] = mma(row_frag_p<T, LD>(Q, 16 * w + m, kb, lane), b, qk[ct]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        const int c = 16 * ct + m;
        const double gc = G[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * w + 4 * grp + i;
            const float ratio = expf((float)(G[r] - gc));
            L[r * LA + c] = r > c ? ratio * kk[ct][i] : 0.f;
            P[r * LA + c] = r >= c ? a.scale * ratio * qk[ct][i] : 0.f;
        }
    }
    __syncthreads();

    // Columns of L times beta: T'.  Rows of L times beta: T.
    if (lane < (BWD ? 32 : 16)) {          // block w of the diagonal, inverse lane / 16, column m
        const int kind = grp;
        const float* const Lb = L + 16 * w * LA + 16 * w;
        const float* const bb = B + 16 * w;
        float x[16], y[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < r; ++i) sum = fmaf(Lb[r * LA + i], y[i], sum);
            x[r] = (r == m ? 1.f : 0.f) - (kind ? bb[r] * sum : sum);
            y[r] = kind ? x[r] : bb[r] * x[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) inv[(kind * kChunk + 16 * w + r) * LA + 16 * w + m] = x[r];
    }
    __syncthreads();
    const int half = w & 1, kind = w >> 1;
    float* const Tm = inv + kind * kChunk * LA;
    // block (row tile, column tile) of the matrix that is inverted, rows row tile, summed index 16 ct + 4 grp + j
    auto block = [&](int rt, int ct) {
        f32x4 x = *(const f32x4*)(L + (16 * rt + m) * LA + 16 * ct + 4 * grp);
        const float br = kind ? B[16 * rt + m] : 1.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= kind ? br : B[16 * ct + 4 * grp + j];
        return x;
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
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (kind == 0 || BWD) {                // 32 x 32 blocks: `half` of the diagonal
        const int b = 2 * half;
        const f32x4 M = mma16x16(block(b + 1, b), cols_of(b, b), zero);
        put(b + 1, b, mma16x16(rows_of(b + 1, b + 1), M, zero));
    }
    __syncthreads();
    if (kind == 0 || BWD) {                // the whole: 16 columns
        f32x4 M[2];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
            M[rt] = mma16x16(block(2 + rt, 1), cols_of(1, half), zero);
            if (half == 0) M[rt] = mma16x16(block(2 + rt, 0), cols_of(0, 0), M[rt]);
        }
        put(2, half, mma16x16(rows_of(2, 2), M[0], zero));
        put(3, half, mma16x16(rows_of(3, 3), M[1], mma16x16(rows_of(3, 2), M[0], zero)));
    }
    __syncthreads();
    if (tid < kChunk) {
        inv[tid * LA + tid] = 0.f;
        if constexpr (BWD) inv[(kChunk + tid) * LA + tid] = 0.f;
    }
    __syncthreads();
    constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
#pragma unroll
    for (int half8 = 0; half8 < 2; ++half8) {
        const int r = tid >> 2, c = 16 * (tid & 3) + 8 * half8;
        store_tile8<T>((T*)(a.tq + at * kTile), sizeof(T) == 2 ? (T*)(a.tl + at * kTile) : nullptr, r, c, inv);
        store_tile8<T>((T*)(a.p + at * kTile), nullptr, r, c, P);
        if constexpr (BWD) store_tile8<T>((T*)(a.tt + at * kTile), nullptr, r, c, inv + kChunk * LA);
    }
}

template <class T, int DK, bool BWD>
hipError_t launch_t(const DeltaArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((delta_prepare_kernel<T, DK, BWD>), dim3((unsigned)(a.slots * (long long)a.H)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_prepare(const DeltaArgs& a, int Dk, int is_bf16, int is_bwd, hipStream_t stream) {
#define LTN_PREPARE(dk)                                                                                                        \
    if (Dk == dk) {                                                                                                            \
        if (is_bf16) return is_bwd ? launch_t<__bf16, dk, true>(a, stream) : launch_t<__bf16, dk, false>(a, stream);           \
        return is_bwd ? launch_t<float, dk, true>(a, stream) : launch_t<float, dk, false>(a, stream);                          \
    }
    LTN_PREPARE(64) LTN_PREPARE(128)
#undef LTN_PREPARE
    return hipErrorInvalidValue;
}

}  // namespace ltn
