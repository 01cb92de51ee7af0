// Gated delta rule: the sweeps over the chunks of a chain (ltn_delta.h has the formulas).  A wave owns 16 CT columns of the
// state: all Dk rows of them stay in its accumulators from the first chunk to the last, and as the columns of S, X, Z, U,
// O (and of dS, dU, dY) are independent, no wave ever waits for another's result.  The state's rows and the tokens are dealt
// to the accumulators' rows so (paired()) that one product's results are, lane by lane, the next one's right operand:
// nothing between the products passes through LDS.  What the waves share are the chunk's tiles, the left operands.
//
// bf16: S, X, U and T' enter the products of the state in two parts of 8 bits of significand each (three products of
// four for T' X): the state that the forward hands on is fp32 and stays as exact as sums of fp32 products to some 4e-6;
// in one part each it would be off by 2.4e-3.  O, rounded to bf16 anyway, takes the larger parts alone.
#include "ltn_delta.h"

namespace ltn {
namespace {

// v - gam (K S) etc. for the four tokens that a lane holds of row tile rt: 32 (rt / 2) + 8 (lane / 16) + 4 (rt % 2) .. +3
__device__ __forceinline__ int token_of(int rt, int grp) { return 32 * (rt >> 1) + 8 * grp + 4 * (rt & 1); }

// Columns of a wave in a [token][column] LDS tile for the lane's four tokens of row tile rt
template <int LD> __device__ __forceinline__ f32x4 col_values(const __bf16* tile, int rt, int c0, int lane) {
    const int s = lane & 15;
    Frag f;
    f.h[0] = lds_tr16((const char*)(tile + (token_of(rt, lane >> 4) + (s >> 2)) * LD + c0 + 4 * (s & 3)));
    return __builtin_convertvector(f.b[0], f32x4);
}
template <int LD> __device__ __forceinline__ f32x4 col_values(const float* tile, int rt, int c0, int lane) {
    const float* p = tile + token_of(rt, lane >> 4) * LD + c0 + (lane & 15);
    return f32x4{p[0], p[LD], p[2 * LD], p[3 * LD]};
}

template <class T> __device__ __forceinline__ void store_frag(T* p, const typename El<T>::F& f) { *(typename El<T>::F*)p = f; }

// Forward.  SAVE: Z and the states before chunks are written, for the gradients, and O is not.
template <class T, int DK, int CT, int W, bool SAVE>
__global__ __launch_bounds__(64 * W)
void delta_fwd_kernel(DeltaArgs a, int Dv, int per_chain) {
    constexpr bool BF = sizeof(T) == 2;
    constexpr int LD = DK + El<T>::PAD, LT = kChunk + El<T>::PAD, COLS = 16 * CT * W, LV = COLS + El<T>::PAD;
    constexpr int NT = DK / 16, TH = 64 * W;
    typedef typename El<T>::F F;
    __shared__ __attribute__((aligned(16))) T K[kChunk * LD], Q[SAVE ? 8 : kChunk * LD], Tq[kChunk * LT], Tl[BF ? kChunk * LT : 8],
        P[SAVE ? 8 : kChunk * LT], V[kChunk * LV];
    __shared__ __attribute__((aligned(16))) float vec[3 * kChunk];       // gam, end, beta

    int chain, split;
    const int chains = a.seqs * a.H;
    map_workgroup(blockIdx.x, per_chain, chains, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = lane & 15, grp = lane >> 4;
    const int wg0 = split * COLS, c0 = 16 * CT * w;                      // the workgroup's and the wave's first column
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first;
    const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first;

    f32x4 S[NT][CT];
    {
        const float* in = a.kv_in ? a.kv_in + (size_t)chain * DK * Dv + wg0 + c0 + m : nullptr;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const int f = token_of(t, grp);                          // the same dealing for features
#pragma unroll
                for (int i = 0; i < 4; ++i) S[t][c][i] = in ? in[(size_t)(f + i) * Dv + 16 * c] : 0.f;
            }
    }
    const int chunks = (s.len + kChunk - 1) / kChunk;
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        __syncthreads();
        load_tile<T, LD, DK, TH>(K, (const T*)a.k + (key_row + t0) * DK, DK, rows, tid);
        if constexpr (!SAVE) load_tile<T, LD, DK, TH>(Q, (const T*)a.q + (key_row + t0) * DK, DK, rows, tid);
        load_tile<T, LV, COLS, TH>(V, (const T*)a.v + (val_row + t0) * Dv + wg0, Dv, rows, tid);
        constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
        load_tile<T, LT, kChunk, TH>(Tq, (const T*)(a.tq + at * kTile), kChunk, kChunk, tid);
        if constexpr (BF) load_tile<T, LT, kChunk, TH>(Tl, (const T*)(a.tl + at * kTile), kChunk, kChunk, tid);
        if constexpr (!SAVE) load_tile<T, LT, kChunk, TH>(P, (const T*)(a.p + at * kTile), kChunk, kChunk, tid);
        for (int i = tid; i < 3 * kChunk; i += TH)
            vec[i] = i < 2 * kChunk ? a.vec[at * 2 * kChunk + i] : (i - 2 * kChunk < rows ? a.beta[val_row + t0 + i - 2 * kChunk] : 0.f);
        __syncthreads();
        const float whole = vec[kChunk - 1];

#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int col = c0 + 16 * c;
            F Sh[NT / 2], Sl[BF ? NT / 2 : 1];
#pragma unroll
            for (int p = 0; p < NT / 2; ++p) {
                Sh[p] = frag_of<T>(S[2 * p][c], S[2 * p + 1][c]);
                if constexpr (BF) Sl[p] = rest_of(Sh[p], S[2 * p][c], S[2 * p + 1][c]);
                if constexpr (SAVE) {
                    T* const out = (T*)a.s0 + (at * Dv + wg0 + col + m) * DK + 32 * p + 8 * grp;
                    store_frag<T>(out, Sh[p]);
                }
            }
            f32x4 Z[4], O[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                O[rt] = x;
                const int row = paired(rt, m);
#pragma unroll
                for (int p = 0; p < NT / 2; ++p) {
                    const F kf = row_frag<T, LD>(K, row, p, lane);
                    x = mma(kf, Sh[p], x);
                    if constexpr (BF) x = mma(kf, Sl[p], x);
                    if constexpr (!SAVE) O[rt] = mma(row_frag<T, LD>(Q, row, p, lane), Sh[p], O[rt]);
                }
                const f32x4 gam = *(const f32x4*)(vec + token_of(rt, grp));
                Z[rt] = col_values<LV>(V, rt, col, lane) - gam * x;
                if constexpr (!SAVE) O[rt] *= gam * a.scale;
            }
            F Xh[2], Xl[BF ? 2 : 1];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                Xh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
                if constexpr (BF) Xl[b] = rest_of(Xh[b], Z[2 * b], Z[2 * b + 1]);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                for (int b = 0; b <= rt / 2; ++b) {
                    const F tf = row_frag<T, LT>(Tq, paired(rt, m), b, lane);
                    Z[rt] = mma(tf, Xh[b], Z[rt]);
                    if constexpr (BF) {
                        Z[rt] = mma(tf, Xl[b], Z[rt]);
                        Z[rt] = mma(row_frag<T, LT>(Tl, paired(rt, m), b, lane), Xh[b], Z[rt]);
                    }
                }
            F Uh[2], Ul[BF ? 2 : 1];
            if constexpr (SAVE) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    store_frag<T>((T*)a.z + (at * Dv + wg0 + col + m) * kChunk + 32 * b + 8 * grp, frag_of<T>(Z[2 * b], Z[2 * b + 1]));
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] *= *(const f32x4*)(vec + 2 * kChunk + token_of(rt, grp));    // U
            if constexpr (!SAVE) {
#pragma unroll
                for (int b = 0; b < 2; ++b) Uh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
#pragma unroll
                for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                    for (int b = 0; b <= rt / 2; ++b) O[rt] = mma(row_frag<T, LT>(P, paired(rt, m), b, lane), Uh[b], O[rt]);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] *= *(const f32x4*)(vec + kChunk + token_of(rt, grp));
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                Uh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
                if constexpr (BF) Ul[b] = rest_of(Uh[b], Z[2 * b], Z[2 * b + 1]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                S[t][c] *= whole;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const F kf = col_frag<LD, true>(K, b, t, lane);
                    S[t][c] = mma(kf, Uh[b], S[t][c]);
                    if constexpr (BF) S[t][c] = mma(kf, Ul[b], S[t][c]);
                }
            }
            if constexpr (!SAVE) {
                // the wave's columns of V have been read: O takes their place and is read back a token a row
#pragma unroll
                for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) V[(token_of(rt, grp) + i) * LV + col + m] = (T)O[rt][i];
            }
        }
        if constexpr (!SAVE) {
            constexpr int E = 16 / sizeof(T), PER = 16 * CT / E;         // pieces of 16 bytes of a token's columns of this wave
            asm volatile("" : : : "memory");                             // (a wave's LDS accesses stay in order; so does the compiler)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int r = (i * 64 + lane) / PER, c = c0 + (i * 64 + lane) % PER * E;
                if (r < rows) *(u32x4*)((T*)a.o + (val_row + t0 + r) * Dv + wg0 + c) = *(const u32x4*)(V + r * LV + c);
            }
        }
    }
    if (!SAVE && a.kv_out) {
        float* const out = a.kv_out + (size_t)chain * DK * Dv + wg0 + c0 + m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) out[(size_t)(token_of(t, grp) + i) * Dv + 16 * c] = S[t][c][i];
    }
}

// Backward, from the last chunk to the first: dY and the derivatives of the states behind chunks.
template <class T, int DK, int CT, int W>
__global__ __launch_bounds__(64 * W)
void delta_bwd_kernel(DeltaArgs a, int Dv, int per_chain) {
    constexpr int LD = DK + El<T>::PAD, LT = kChunk + El<T>::PAD, COLS = 16 * CT * W, LV = COLS + El<T>::PAD;
    constexpr int NT = DK / 16, TH = 64 * W;
    typedef typename El<T>::F F;
    __shared__ __attribute__((aligned(16))) T K[kChunk * LD], Q[kChunk * LD], Tt[kChunk * LT], P[kChunk * LT], G[kChunk * LV];
    __shared__ __attribute__((aligned(16))) float vec[3 * kChunk];

    int chain, split;
    const int chains = a.seqs * a.H;
    map_workgroup(blockIdx.x, per_chain, chains, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = lane & 15, grp = lane >> 4;
    const int wg0 = split * COLS, c0 = 16 * CT * w;
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first;
    const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first;

    f32x4 S[NT][CT];                       // dS
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) S[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (s.len + kChunk - 1) / kChunk;
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        __syncthreads();
        load_tile<T, LD, DK, TH>(K, (const T*)a.k + (key_row + t0) * DK, DK, rows, tid);
        load_tile<T, LD, DK, TH>(Q, (const T*)a.q + (key_row + t0) * DK, DK, rows, tid);
        load_tile<T, LV, COLS, TH>(G, (const T*)a.d_o + (val_row + t0) * Dv + wg0, Dv, rows, tid);
        constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
        load_tile<T, LT, kChunk, TH>(Tt, (const T*)(a.tt + at * kTile), kChunk, kChunk, tid);
        load_tile<T, LT, kChunk, TH>(P, (const T*)(a.p + at * kTile), kChunk, kChunk, tid);
        for (int i = tid; i < 3 * kChunk; i += TH)
            vec[i] = i < 2 * kChunk ? a.vec[at * 2 * kChunk + i] : (i - 2 * kChunk < rows ? a.beta[val_row + t0 + i - 2 * kChunk] : 0.f);
        __syncthreads();
        const float whole = vec[kChunk - 1];

#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int col = c0 + 16 * c;
            F Sf[NT / 2];
#pragma unroll
            for (int p = 0; p < NT / 2; ++p) {
                Sf[p] = frag_of<T>(S[2 * p][c], S[2 * p + 1][c]);
                store_frag<T>((T*)a.ds + (at * Dv + wg0 + col + m) * DK + 32 * p + 8 * grp, Sf[p]);
            }
            F gf[2];                       // dO
#pragma unroll
            for (int b = 0; b < 2; ++b) gf[b] = col_frag<LV, false>(G + col, b, 0, lane);
            f32x4 Y[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                Y[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 0; p < NT / 2; ++p) Y[rt] = mma(row_frag<T, LD>(K, paired(rt, m), p, lane), Sf[p], Y[rt]);
                Y[rt] *= *(const f32x4*)(vec + kChunk + token_of(rt, grp));
#pragma unroll
                for (int b = rt / 2; b < 2; ++b) Y[rt] = mma(col_frag<LT, true>(P, b, rt, lane), gf[b], Y[rt]);
            }
            F uf[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) uf[b] = frag_of<T>(Y[2 * b], Y[2 * b + 1]);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                for (int b = rt / 2; b < 2; ++b) Y[rt] = mma(col_frag<LT, true>(Tt, b, rt, lane), uf[b], Y[rt]);
            F xf[2], of[2];                // -gam dV, scale gam dO
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                store_frag<T>((T*)a.dy + (at * Dv + wg0 + col + m) * kChunk + 32 * b + 8 * grp, frag_of<T>(Y[2 * b], Y[2 * b + 1]));
                const f32x4 g0 = *(const f32x4*)(vec + 32 * b + 8 * grp), g1 = *(const f32x4*)(vec + 32 * b + 8 * grp + 4);
                const f32x4 b0 = *(const f32x4*)(vec + 2 * kChunk + 32 * b + 8 * grp), b1 = *(const f32x4*)(vec + 2 * kChunk + 32 * b + 8 * grp + 4);
                xf[b] = frag_of<T>(-g0 * b0 * Y[2 * b], -g1 * b1 * Y[2 * b + 1]);
                f32x4 o0, o1;
                values_of(gf[b], o0, o1);
                of[b] = frag_of<T>(a.scale * g0 * o0, a.scale * g1 * o1);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                S[t][c] *= whole;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    S[t][c] = mma(col_frag<LD, true>(K, b, t, lane), xf[b], S[t][c]);
                    S[t][c] = mma(col_frag<LD, true>(Q, b, t, lane), of[b], S[t][c]);
                }
            }
        }
    }
}

template <class T, int DK, bool SAVE>
hipError_t launch_fwd_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    constexpr int CT = 1, W = 4;
    const int per = Dv / (16 * CT * W);
    hipLaunchKernelGGL((delta_fwd_kernel<T, DK, CT, W, SAVE>), dim3((unsigned)((long long)a.seqs * a.H * per)), dim3(64 * W), 0, stream, a, Dv, per);
    return hipGetLastError();
}
template <class T, int DK>
hipError_t launch_bwd_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    constexpr int CT = 1, W = 4;
    const int per = Dv / (16 * CT * W);
    hipLaunchKernelGGL((delta_bwd_kernel<T, DK, CT, W>), dim3((unsigned)((long long)a.seqs * a.H * per)), dim3(64 * W), 0, stream, a, Dv, per);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    if (a.slots > 0) {
        const hipError_t e = launch_delta_prepare(a, Dk, is_bf16, 0, stream);
        if (e != hipSuccess) return e;
    }
    if (Dk == 64) return is_bf16 ? launch_fwd_t<__bf16, 64, false>(a, Dv, stream) : launch_fwd_t<float, 64, false>(a, Dv, stream);
    return is_bf16 ? launch_fwd_t<__bf16, 128, false>(a, Dv, stream) : launch_fwd_t<float, 128, false>(a, Dv, stream);
}

hipError_t launch_delta_bwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    hipError_t e = launch_delta_prepare(a, Dk, is_bf16, 1, stream);
    if (e != hipSuccess) return e;
    if (Dk == 64) e = is_bf16 ? launch_fwd_t<__bf16, 64, true>(a, Dv, stream) : launch_fwd_t<float, 64, true>(a, Dv, stream);
    else e = is_bf16 ? launch_fwd_t<__bf16, 128, true>(a, Dv, stream) : launch_fwd_t<float, 128, true>(a, Dv, stream);
    if (e != hipSuccess) return e;
    if (Dk == 64) e = is_bf16 ? launch_bwd_t<__bf16, 64>(a, Dv, stream) : launch_bwd_t<float, 64>(a, Dv, stream);
    else e = is_bf16 ? launch_bwd_t<__bf16, 128>(a, Dv, stream) : launch_bwd_t<float, 128>(a, Dv, stream);
    if (e != hipSuccess) return e;
    return launch_delta_grad(a, Dk, Dv, is_bf16, stream);
}

}  // namespace ltn
