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

// first of the four tokens (or features) that a lane holds of row tile rt
__device__ __forceinline__ int token_of(int rt, int grp) { return 32 * (rt >> 1) + 8 * grp + 4 * (rt & 1); }

template <class T> __device__ __forceinline__ void store_frag(T* p, const typename El<T>::F& f) { *(typename El<T>::F*)p = f; }
// four fp32 values as four consecutive elements
__device__ __forceinline__ void store4(__bf16* p, const f32x4& x) { *(bf16x4*)p = to_bf16(x); }
__device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }

// One chunk's tiles in LDS.  FWD: K, T', its second part (bf16), V and, where O is wanted, Q and P.  Backward: K, Q, T, P, dO.
template <class T, int DK, int COLS, bool FULL, bool FWD> struct SweepLds {
    static constexpr int K = 0, T1 = K + Tile<T, DK>::BYTES, V = T1 + Tile<T, kChunk>::BYTES, VEC = V + Tile<T, COLS>::BYTES,
                         T2 = VEC + 1024, Q = T2 + (FWD && sizeof(T) == 2 ? Tile<T, kChunk>::BYTES : 0),
                         P = Q + (FULL ? Tile<T, DK>::BYTES : 0), BYTES = P + (FULL ? Tile<T, kChunk>::BYTES : 0);
    static constexpr int BUFS = 2 * BYTES <= 160 * 1024 ? 2 : 1;
};

// The fetches of a chunk's tiles by W waves.
template <class T, int DK, int COLS, int W, bool FULL, bool FWD> struct SweepFetch {
    typedef SweepLds<T, DK, COLS, FULL, FWD> L;
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
    TileFetch<T, DK, W> k, q;
    TileFetch<T, kChunk, W> t1, t2, p;
    TileFetch<T, COLS, W> v;
    u32x4 vec;
    // at: the chunk's scratch; key_row, val_row: its first token's rows
    __device__ __forceinline__ void fetch(const DeltaArgs& a, size_t at, size_t key_row, size_t val_row, int rows, int Dv, int col0,
                                          char* lds, int w, int lane) {
        k.fetch((const char*)a.k + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, lds + L::K, w, lane);
        t1.fetch((FWD ? a.tq : a.tt) + at * kTile, kChunk * sizeof(T), kChunk, lds + L::T1, w, lane);
        v.fetch((const char*)(FWD ? a.v : a.d_o) + (val_row * Dv + col0) * sizeof(T), Dv * sizeof(T), rows, lds + L::V, w, lane);
        if constexpr (FWD && BF) t2.fetch(a.tl + at * kTile, kChunk * sizeof(T), kChunk, lds + L::T2, w, lane);
        if constexpr (FULL) {
            q.fetch((const char*)a.q + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, lds + L::Q, w, lane);
            p.fetch(a.p + at * kTile, kChunk * sizeof(T), kChunk, lds + L::P, w, lane);
        }
        if (w == 0) {                      // 768 bytes of decays and beta (the last quarter of the kilobyte is not read)
            const char* src = (const char*)(a.vec + at * 3 * kChunk) + (lane < 48 ? lane * 16 : 0);
            if constexpr (BF) dma16(lds_address(lds + L::VEC), src);
            else vec = *(const u32x4*)src;
        }
    }
    __device__ __forceinline__ void put(char* lds, int w, int lane) const {
        if constexpr (!BF) {
            k.put(lds + L::K, w, lane);
            t1.put(lds + L::T1, w, lane);
            v.put(lds + L::V, w, lane);
            if constexpr (FULL) {
                q.put(lds + L::Q, w, lane);
                p.put(lds + L::P, w, lane);
            }
            if (w == 0) *(u32x4*)(lds + L::VEC + lane * 16) = vec;
        }
    }
};

// Forward.  SAVE: Z and the states before chunks are written, for the gradients, and O is not.
template <class T, int DK, int CT, int W, bool SAVE>
__global__ __launch_bounds__(64 * W)
void delta_fwd_kernel(DeltaArgs a, int Dv, int per_chain) {
    constexpr bool BF = sizeof(T) == 2;
    constexpr int COLS = 16 * CT * W, NT = DK / 16;
    typedef typename El<T>::F F;
    typedef SweepLds<T, DK, COLS, !SAVE, true> L;
    constexpr bool TWO = BF && L::BUFS == 2;
    __shared__ __attribute__((aligned(1024))) char lds[(TWO ? 2 : 1) * L::BYTES];

    int chain, split;
    map_workgroup(blockIdx.x, per_chain, a.seqs * a.H, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, grp = lane >> 4;
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
    SweepFetch<T, DK, COLS, W, !SAVE, true> next;
    auto fetch = [&](int chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        next.fetch(a, (size_t)(s.slot + chunk) * a.H + h, key_row + t0, val_row + t0, rows, Dv, wg0,
                   lds + (TWO ? (chunk & 1) * L::BYTES : 0), w, lane);
    };
    if (chunks) fetch(0);
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        const char* const cur = lds + (TWO ? (chunk & 1) * L::BYTES : 0);
        if constexpr (TWO) {
            wait_dma<0>();
            __syncthreads();               // this chunk's tiles are there, the last one's are read
            if (chunk + 1 < chunks) fetch(chunk + 1);
        } else {
            if (BF) wait_dma<0>();
            next.put(lds, w, lane);
            __syncthreads();
            if (!BF && chunk + 1 < chunks) fetch(chunk + 1);
        }
        const char *const K = cur + L::K, *const Tq = cur + L::T1, *const Tl = cur + L::T2, *const V = cur + L::V,
                   *const Q = cur + L::Q, *const P = cur + L::P;
        const float* const vec = (const float*)(cur + L::VEC);           // gam, end, beta
        const float whole = vec[kChunk - 1];

#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int col = c0 + 16 * c;
            F Sh[NT / 2], Sl[BF ? NT / 2 : 1];
#pragma unroll
            for (int p = 0; p < NT / 2; ++p) {
                Sh[p] = frag_of<T>(S[2 * p][c], S[2 * p + 1][c]);
                if constexpr (BF) Sl[p] = rest_of(Sh[p], S[2 * p][c], S[2 * p + 1][c]);
                if constexpr (SAVE) store_frag<T>((T*)a.s0 + (at * Dv + wg0 + col + m) * DK + 32 * p + 8 * grp, Sh[p]);
            }
            f32x4 Z[4], O[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] = O[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < NT / 2; ++p)
#pragma unroll
                for (int rt = 0; rt < 4; ++rt) {
                    const F kf = row_frag<T, DK>(K, paired(rt, m), p, lane);
                    Z[rt] = mma(kf, Sh[p], Z[rt]);
                    if constexpr (BF) Z[rt] = mma(kf, Sl[p], Z[rt]);
                }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
                Z[rt] = col_values<T, COLS>(V, rt, col, lane) - *(const f32x4*)(vec + token_of(rt, grp)) * Z[rt];
            F Xh[2], Xl[BF ? 2 : 1];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                Xh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
                if constexpr (BF) Xl[b] = rest_of(Xh[b], Z[2 * b], Z[2 * b + 1]);
            }
            // O transposed, its rows value columns and its columns tokens: a lane's values are neighbours in memory
            if constexpr (!SAVE) {
#pragma unroll
                for (int p = 0; p < NT / 2; ++p)
#pragma unroll
                    for (int rt = 0; rt < 4; ++rt) O[rt] = mma(Sh[p], row_frag<T, DK>(Q, 16 * rt + m, p, lane), O[rt]);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int rt = 2 * b; rt < 4; ++rt) {
                    const F tf = row_frag<T, kChunk>(Tq, paired(rt, m), b, lane);
                    Z[rt] = mma(tf, Xh[b], Z[rt]);
                    if constexpr (BF) {
                        Z[rt] = mma(tf, Xl[b], Z[rt]);
                        Z[rt] = mma(row_frag<T, kChunk>(Tl, paired(rt, m), b, lane), Xh[b], Z[rt]);
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
                for (int rt = 0; rt < 4; ++rt) {
                    O[rt] *= vec[16 * rt + m] * a.scale;
#pragma unroll
                    for (int b = 0; b <= rt / 2; ++b) O[rt] = mma(Uh[b], row_frag<T, kChunk>(P, 16 * rt + m, b, lane), O[rt]);
                }
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] *= *(const f32x4*)(vec + kChunk + token_of(rt, grp));
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                Uh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
                if constexpr (BF) Ul[b] = rest_of(Uh[b], Z[2 * b], Z[2 * b + 1]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) S[t][c] *= whole;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const F kf = col_frag<T, DK, true>(K, b, t, lane);
                    S[t][c] = mma(kf, Uh[b], S[t][c]);
                    if constexpr (BF) S[t][c] = mma(kf, Ul[b], S[t][c]);
                }
            if constexpr (!SAVE) {
#pragma unroll
                for (int rt = 0; rt < 4; ++rt)
                    if (16 * rt + m < rows) store4((T*)a.o + (val_row + t0 + 16 * rt + m) * Dv + wg0 + col + 4 * grp, O[rt]);
            }
        }
        if constexpr (!TWO) {
            __syncthreads();
            if (BF && chunk + 1 < chunks) fetch(chunk + 1);
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
    constexpr bool BF = sizeof(T) == 2;
    constexpr int COLS = 16 * CT * W, NT = DK / 16;
    typedef typename El<T>::F F;
    typedef SweepLds<T, DK, COLS, true, false> L;
    constexpr bool TWO = BF && L::BUFS == 2;
    __shared__ __attribute__((aligned(1024))) char lds[(TWO ? 2 : 1) * L::BYTES];

    int chain, split;
    map_workgroup(blockIdx.x, per_chain, a.seqs * a.H, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, grp = lane >> 4;
    const int wg0 = split * COLS, c0 = 16 * CT * w;
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first;
    const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first;

    f32x4 S[NT][CT];                       // dS
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) S[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (s.len + kChunk - 1) / kChunk;
    SweepFetch<T, DK, COLS, W, true, false> next;
    auto fetch = [&](int chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        next.fetch(a, (size_t)(s.slot + chunk) * a.H + h, key_row + t0, val_row + t0, rows, Dv, wg0,
                   lds + (TWO ? (chunk & 1) * L::BYTES : 0), w, lane);
    };
    if (chunks) fetch(chunks - 1);
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        const char* const cur = lds + (TWO ? (chunk & 1) * L::BYTES : 0);
        if constexpr (TWO) {
            wait_dma<0>();
            __syncthreads();
            if (chunk) fetch(chunk - 1);
        } else {
            if (BF) wait_dma<0>();
            next.put(lds, w, lane);
            __syncthreads();
            if (!BF && chunk) fetch(chunk - 1);
        }
        const char *const K = cur + L::K, *const Tt = cur + L::T1, *const G = cur + L::V, *const Q = cur + L::Q, *const P = cur + L::P;
        const float* const vec = (const float*)(cur + L::VEC);
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
            for (int b = 0; b < 2; ++b) gf[b] = col_frag<T, COLS, false>(G, b, col / 16, lane);
            f32x4 Y[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Y[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < NT / 2; ++p)
#pragma unroll
                for (int rt = 0; rt < 4; ++rt) Y[rt] = mma(row_frag<T, DK>(K, paired(rt, m), p, lane), Sf[p], Y[rt]);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                Y[rt] *= *(const f32x4*)(vec + kChunk + token_of(rt, grp));
#pragma unroll
                for (int b = rt / 2; b < 2; ++b) Y[rt] = mma(col_frag<T, kChunk, true>(P, b, rt, lane), gf[b], Y[rt]);
            }
            F uf[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) uf[b] = frag_of<T>(Y[2 * b], Y[2 * b + 1]);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
#pragma unroll
                for (int b = rt / 2; b < 2; ++b) Y[rt] = mma(col_frag<T, kChunk, true>(Tt, b, rt, lane), uf[b], Y[rt]);
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
            for (int t = 0; t < NT; ++t) S[t][c] *= whole;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    S[t][c] = mma(col_frag<T, DK, true>(Q, b, t, lane), of[b], S[t][c]);
                    S[t][c] = mma(col_frag<T, DK, true>(K, b, t, lane), xf[b], S[t][c]);
                }
        }
        if constexpr (!TWO) {
            __syncthreads();
            if (BF && chunk) fetch(chunk - 1);
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
