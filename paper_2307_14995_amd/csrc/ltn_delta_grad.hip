// Gated delta rule: the gradients of a chunk of 64 tokens and a head of keys (ltn_delta.h has the formulas), from Z, dV and
// the states that the sweeps left.  The value heads that share the keys follow one another in one workgroup: their dq and
// dk are summed in registers, in a fixed order.  Wave w owns tokens 16 (w % 4) .. +15 and half of the key features; the
// value features come in slabs of VS, so that two workgroups fit a compute unit (62 KB of LDS; 128 registers where a value head
// has its keys alone) and one's loads pass while the other computes.
// Scales of rows and columns (decays, beta) are applied to products' fp32 results, never to an operand.  What is rounded to
// bf16 are dP and E as operands of the products with K and Q; the row and column sums that dg and dbeta take are of dP and E
// in fp32 (a decay's gradient is a small difference of large sums: 1.5e-2 off for keys that are alike, with rounded ones).
// Bound by HBM where the card is full: 178 KB a chunk and head, of which the two states are 64; 4 rows of 8192 tokens, 32 heads
// of 128 features, bf16: 600 us, 4.9 TB/s.  8 rows of 2048, 8 heads on 4 key heads, a workgroup a unit: 94 us (104 where each
// head fetched K, Q and its slabs when it came to them).
#include "ltn_delta.h"

namespace ltn {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

template <class T> __device__ __forceinline__ float dot8(const typename El<T>::F& a, const typename El<T>::F& b) {
    f32x4 a0, a1, b0, b1;
    values_of(a, a0, a1);
    values_of(b, b0, b1);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(a0[i], b0[i], fmaf(a1[i], b1[i], s));
    return s;
}
__device__ __forceinline__ float rounded_product(float a, float b) {     // no part of a fused multiply-add
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ float row_sum16(float x) {      // over the 16 lanes of a row, by rotations within it
#define LTN_ROTATE(n) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x120 + n, 0xf, 0xf, false))
    LTN_ROTATE(8);
    LTN_ROTATE(4);
    LTN_ROTATE(2);
    LTN_ROTATE(1);
#undef LTN_ROTATE
    return x;
}
// four elements in LDS times x; four values to LDS
template <class T> __device__ __forceinline__ float dot4(unsigned at, const f32x4& x) {
    f32x4 v;
    if constexpr (sizeof(T) == 2) v = __builtin_convertvector(lds_read<bf16x4>(at), f32x4);
    else v = lds_read<f32x4>(at);
    return v[0] * x[0] + v[1] * x[1] + v[2] * x[2] + v[3] * x[3];
}
template <class T> __device__ __forceinline__ void write4(unsigned at, const f32x4& x) {
    if constexpr (sizeof(T) == 2) lds_write(at, to_bf16(x));
    else lds_write(at, x);
}
// NT tiles of 16 features of the lane's token
template <int NT> __device__ __forceinline__ void store_row(__bf16* row, const f32x4 (&x)[NT], int grp, bool there) {
    store_strip<NT>(x, (char*)(row + 8 * grp), there);
}
template <int NT> __device__ __forceinline__ void store_row(float* row, const f32x4 (&x)[NT], int grp, bool there) {
    if (there)
#pragma unroll
        for (int t = 0; t < NT; ++t) *(f32x4*)(row + 16 * t + 4 * grp) = x[t];
}

// Two regions: the slab's states, later K and Q; the slab's dO, dV and Z, later dP and E.
template <class T, int DK, int VS> struct GradLds {
    static constexpr int GB = Tile<T, VS>::BYTES, ZB = Tile<T, kChunk>::RB * VS, SB = Tile<T, DK>::RB * VS;
    static constexpr int KB = Tile<T, DK>::BYTES, PB = Tile<T, kChunk>::BYTES;
    static constexpr int A = 2 * (SB > KB ? SB : KB), B = 2 * GB + ZB > 2 * PB ? 2 * GB + ZB : 2 * PB;
    static constexpr int S = 0, D = SB, K = 0, Q = KB, G = A, Y = A + GB, Z = A + 2 * GB, P = A, E = A + PB, BYTES = A + B;
};

// Value heads that share keys, bf16: one workgroup a unit (their sums take the registers), so K and Q stay in LDS and the next slab
// is on its way, into a second buffer, while one is worked on.  P and E lie over the last slab's dO, dV and Z.
template <class T, int DK, int VS> struct GradPipe {
    typedef GradLds<T, DK, VS> L;
    static constexpr int SLAB = L::BYTES, KQ = 2 * L::KB, VECS = KQ + 2 * SLAB, BYTES = VECS + 2 * 2048;
    static_assert(SLAB % 1024 == 0 && L::A >= 2 * L::SB, "tiles of whole kilobytes");
};

// ONE: no other value head shares the keys.
// All products are taken transposed: a lane's results are four features (or columns) of one token, 16 tok + lane % 16.  Of
// dO Z^T and dV Z^T the waves of the first half take one, those of the second the other.
template <class T, int DK, int VS, bool ONE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && ONE ? 4 : 2)
void delta_grad_kernel(DeltaArgs a, int Dv) {
    typedef GradLds<T, DK, VS> L;
    typedef typename El<T>::F F;
    constexpr int NT = DK / 32;
    constexpr bool PIPE = !ONE && sizeof(T) == 2;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    __shared__ __attribute__((aligned(16))) float vec_of_one[PIPE ? 4 : kVec];       // gam, end, beta, G in two parts
    __shared__ __attribute__((aligned(16))) float row_of[2][kChunk], end_of[2][kChunk], col_of[kWaves][kChunk], part[kWaves];
    const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk, group = ONE ? 1 : a.H / a.Hk;
    DeltaSeq s;
    int chunk;
    if (!delta_find(a, slot, s, chunk)) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, grp = lane >> 4;
    const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
    const int tok = w & 3, hf = w >> 2, r = 16 * tok + m, f0 = hf * NT;    // f0: first of the wave's tiles of 16 key features
    const size_t key_row = ((size_t)s.row * a.Hk + hk) * a.N + s.first + t0;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const unsigned base = lds_address(lds);
    RowReader<T, VS> row_v(base, r, lane);
    RowReader<T, kChunk> row_c(base, r, lane);
    ColReader<T, kChunk, false> col_c(base, lane);
    ColReader<T, DK, false> col_k(base, lane), col_s(base, lane);        // of K and Q; of the states
    typedef GradPipe<T, DK, VS> Pipe;
    unsigned slab = base;                  // the slab's buffer; PIPE: behind K and Q, and the other one behind it
    float* vec = PIPE ? (float*)(lds + Pipe::VECS) : vec_of_one;
    auto fetch_slab = [&](int h, int v0, unsigned to, int n) {           // n: which of the heads, for its decays
        const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first + t0, at = (size_t)slot * a.H + h;
        TileFetch<T, VS, kWaves> g, y;
        TileFetch<T, kChunk, kWaves, VS> z;
        TileFetch<T, DK, kWaves, VS> st, d;
        z.fetch((const char*)a.z + (at * Dv + v0) * (kChunk * sizeof(T)), kChunk * sizeof(T), VS, to + L::Z, w, lane);
        y.fetch((const char*)a.dv + (val_row * Dv + v0) * sizeof(T), Dv * sizeof(T), rows, to + L::Y, w, lane);
        g.fetch((const char*)a.d_o + (val_row * Dv + v0) * sizeof(T), Dv * sizeof(T), rows, to + L::G, w, lane);
        st.fetch((const char*)a.s0 + (at * Dv + v0) * (DK * sizeof(T)), DK * sizeof(T), VS, to + L::S, w, lane);
        d.fetch((const char*)a.ds + (at * Dv + v0) * (DK * sizeof(T)), DK * sizeof(T), VS, to + L::D, w, lane);
        if constexpr (PIPE) {
            if (v0 == 0 && w < 2) {        // 1280 bytes of decays and beta: 64 lanes of one wave, 16 of the next
                const int piece = 64 * w + lane;
                dma16(base + Pipe::VECS + (n & 1) * 2048 + w * 1024, piece < 80 ? (const char*)(a.vec + at * kVec) + piece * 16 : (const char*)kZeros);
            }
        } else {
            if constexpr (sizeof(T) == 2) wait_dma<0>();
            z.put(to + L::Z, w, lane);
            y.put(to + L::Y, w, lane);
            g.put(to + L::G, w, lane);
            st.put(to + L::S, w, lane);
            d.put(to + L::D, w, lane);
        }
    };
    auto move_slab = [&](int by) {
        slab += by;
        row_v.move(by);
        row_c.move(by);
        col_c.move(by);
        col_s.move(by);
    };
    if constexpr (PIPE) {
        TileFetch<T, DK, kWaves> kt, qt;
        kt.fetch((const char*)a.k + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, base + L::K, w, lane);
        qt.fetch((const char*)a.q + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, base + L::Q, w, lane);
        move_slab(Pipe::KQ);
        fetch_slab(hk * group, 0, slab, 0);
    }

    f32x4 dq[ONE ? 1 : NT], dk[ONE ? 1 : NT];
    if constexpr (!ONE)
#pragma unroll
        for (int t = 0; t < NT; ++t) dq[t] = dk[t] = zero;

    for (int j = 0; j < group; ++j) {
        const int h = hk * group + j;
        const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first + t0, at = (size_t)slot * a.H + h;
        const float mine = !PIPE && threadIdx.x < kVec ? a.vec[at * kVec + threadIdx.x] : 0.f;
        if constexpr (PIPE) vec = (float*)(lds + Pipe::VECS + (j & 1) * 2048);
        f32x4 pe[4], qs[NT], ks[NT], ke[NT];
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) pe[ct] = zero;
#pragma unroll
        for (int t = 0; t < NT; ++t) qs[t] = ks[t] = ke[t] = zero;
        float sdot = 0.f;
        for (int v0 = 0; v0 < Dv; v0 += VS) {
            if constexpr (PIPE) {
                if (j || v0) move_slab(slab == base + Pipe::KQ ? Pipe::SLAB : -Pipe::SLAB);
                wait_dma<0>();
                __syncthreads();           // this slab is there, and the last one's readers (and those of P and E over it) are done
                const bool more = v0 + VS < Dv;
                if (more || j + 1 < group)
                    fetch_slab(more ? h : h + 1, more ? v0 + VS : 0, slab == base + Pipe::KQ ? slab + Pipe::SLAB : slab - Pipe::SLAB, j + !more);
            } else {
                if (j || v0) __syncthreads();                            // the tiles' last readers are done
                fetch_slab(h, v0, slab, 0);
                if (v0 == 0 && threadIdx.x < kVec) vec[threadIdx.x] = mine;
                __syncthreads();
            }
            col_c.hide_all();
            col_s.hide_all();
            for (int i = threadIdx.x; i < VS * DK / 8; i += kThreads) {  // (both tiles are laid out alike)
                const int o = Tile<T, DK>::at(i / (DK / 8), i % (DK / 8) * 8);
                sdot += dot8<T>(lds_frag<T>(slab + L::S + o), lds_frag<T>(slab + L::D + o));
            }
#pragma unroll
            for (int kb = 0; kb < VS / 32; ++kb) {
                const F gf = row_v.frag(L::G, kb);
                const F yf = row_v.frag(L::Y, kb);
                const F zf = col_c.frag(L::Z, kb, tok);
                const F own = hf ? yf : gf;
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) pe[ct] = mma(col_c.frag(L::Z, kb, ct), own, pe[ct]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const F sf = col_s.frag(L::S, kb, f0 + t), df = col_s.frag(L::D, kb, f0 + t);
                    qs[t] = mma(sf, gf, qs[t]);
                    ks[t] = mma(sf, yf, ks[t]);
                    ke[t] = mma(df, zf, ke[t]);
                }
            }
        }
        __syncthreads();                   // the slab is read: (K, Q,) dP and E take its place
        TileFetch<T, DK, kWaves> kt, qt;
        if constexpr (!PIPE) {
            kt.fetch((const char*)a.k + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, base + L::K, w, lane);
            qt.fetch((const char*)a.q + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, base + L::Q, w, lane);
        }
        {
            const float ghi = vec[3 * kChunk + r], glo = vec[4 * kChunk + r], side = hf ? -1.f : a.scale;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const int c = 16 * ct + 4 * grp;
                asm volatile("" : : : "memory");                         // (what it reads would be read for all four ahead)
                const f32x4 bc = *(const f32x4*)(vec + 2 * kChunk + c), chi = *(const f32x4*)(vec + 3 * kChunk + c),
                            clo = *(const f32x4*)(vec + 4 * kChunk + c);
                f32x4& x = pe[ct];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = side * expf((ghi - chi[i]) + (glo - clo[i])) * pe[ct][i];
                    x[i] = r >= c + i + hf ? y : 0.f;
                }
                write4<T>(slab + (hf ? L::E : L::P) + Tile<T, kChunk>::at(r, c), x * bc);
            }
        }
        const float beta = vec[2 * kChunk + r], gam = vec[r], end = vec[kChunk + r];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            qs[t] = times(qs[t], a.scale * gam);
            ks[t] = times(ks[t], -gam);
            ke[t] = times(ke[t], end);
        }
        if constexpr (!PIPE) {
            if constexpr (sizeof(T) == 2) wait_dma<0>();
            kt.put(base + L::K, w, lane);
            qt.put(base + L::Q, w, lane);
        }
        __syncthreads();
        float sum = 0.f, ends = 0.f;       // of token r: what its row gives dG; k . C
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int o = Tile<T, DK>::at(r, 16 * (f0 + t) + 4 * grp);
            sum += dot4<T>(base + L::Q + o, qs[t]) + dot4<T>(base + L::K + o, ks[t]);
            ends += dot4<T>(base + L::K + o, ke[t]);
            ke[t] = times(ke[t], beta);
        }
        {
            // rows' and columns' sums of dP (.) Q K^T and of E (.) K K^T, from unrounded dP and E: where keys are alike, they
            // cancel to far less than a rounding of their terms
            const RowReader<T, DK> own(base + (hf ? L::K : L::Q), r, lane), other(base + L::K, m, lane);
            f32x4 xk[4];
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) xk[ct] = zero;
#pragma unroll
            for (int kb = 0; kb < DK / 32; ++kb) {
                const F b = own.frag(0, kb);
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) xk[ct] = mma(other.frag(16 * ct * Tile<T, DK>::RB, kb), b, xk[ct]);
            }
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const f32x4 bc = *(const f32x4*)(vec + 2 * kChunk + 16 * ct + 4 * grp);
                f32x4 down;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = r >= 16 * ct + 4 * grp + i + hf ? pe[ct][i] * xk[ct][i] : 0.f;
                    sum += rounded_product(bc[i], y);
                    down[i] = row_sum16(y);
                }
                if (m == 0) *(f32x4*)(col_of[w] + 16 * ct + 4 * grp) = down;
            }
        }
        col_c.hide_all();
        col_k.hide_all();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const F pr = row_c.frag(L::P, kb), er = row_c.frag(L::E, kb);
            const F pc = col_c.frag(L::P, kb, tok), ec = col_c.frag(L::E, kb, tok);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const F kf = col_k.frag(L::K, kb, f0 + t);
                qs[t] = mma(kf, pr, qs[t]);
                ks[t] = mma(kf, er, ks[t]);
                ke[t] = mma(col_k.frag(L::Q, kb, f0 + t), pc, ke[t]);
                ke[t] = mma(kf, ec, ke[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) ks[t] += ke[t];
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        ends += __shfl_xor(ends, 16, 64);
        ends += __shfl_xor(ends, 32, 64);
        if (grp == 0) {
            row_of[hf][r] = sum;
            end_of[hf][r] = ends;
        }
#pragma unroll
        for (int x = 1; x < 64; x *= 2) sdot += __shfl_xor(sdot, x, 64);
        if (lane == 0) part[w] = sdot;
        if constexpr (ONE) {
            store_row<NT>((T*)a.dq + (key_row + r) * DK + 16 * f0, qs, grp, r < rows);
            store_row<NT>((T*)a.dk + (key_row + r) * DK + 16 * f0, ks, grp, r < rows);
        } else {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                dq[t] += qs[t];
                dk[t] += ks[t];
            }
        }
        __syncthreads();
        if (w == 0) {
            const float bt = vec[2 * kChunk + lane], e = end_of[0][lane] + end_of[1][lane];
            float d = e, x = row_of[0][lane] + row_of[1][lane], all = bt * e, states = 0.f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                d += col_of[i][lane];
                states += part[i];
            }
            if (lane < rows) ((T*)a.dbeta)[val_row + lane] = (T)d;
            x -= rounded_product(bt, d);         // (rounded as the rows' terms are: a diagonal's two cancel)
#pragma unroll
            for (int o = 1; o < 64; o *= 2) all += __shfl_xor(all, o, 64);
            if (lane == 63) x += fmaf(vec[kChunk - 1], states, all);
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const float y = __shfl_down(x, o, 64);
                if (lane + o < 64) x += y;
            }
            if (lane < rows) ((T*)a.dg)[val_row + lane] = (T)x;
        }
        // (the next head's sums are written behind barriers that wave 0 takes after this)
    }
    if constexpr (!ONE) {
        store_row<NT>((T*)a.dq + (key_row + r) * DK + 16 * f0, dq, grp, r < rows);
        store_row<NT>((T*)a.dk + (key_row + r) * DK + 16 * f0, dk, grp, r < rows);
    }
}

template <class T, int DK, int VS>
hipError_t launch_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    constexpr int ALONE = GradLds<T, DK, VS>::BYTES, SHARED = sizeof(T) == 2 ? GradPipe<T, DK, VS>::BYTES : ALONE;
    static_assert(SHARED <= 155 * 1024, "LDS");
    const bool one = a.H == a.Hk;
    hipLaunchKernelGGL((one ? delta_grad_kernel<T, DK, VS, true> : delta_grad_kernel<T, DK, VS, false>),
                       dim3((unsigned)((long long)a.slots * a.Hk)), dim3(kThreads), one ? ALONE : SHARED, stream, a, Dv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_grad(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    if (Dk == 64) return is_bf16 ? launch_t<__bf16, 64, 64>(a, Dv, stream) : launch_t<float, 64, 32>(a, Dv, stream);
    return is_bf16 ? launch_t<__bf16, 128, 64>(a, Dv, stream) : launch_t<float, 128, 32>(a, Dv, stream);
}

}  // namespace ltn
