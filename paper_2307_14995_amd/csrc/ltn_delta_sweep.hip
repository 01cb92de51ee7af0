// Gated delta rule: the sweeps over the chunks of a chain (ltn_delta.h has the formulas).  A wave owns 16 columns of the
// state: all Dk rows of them stay in its accumulators from the first chunk to the last, and as the columns of S, X, Z, U,
// O (and of dS, dU, dV) are independent, no wave waits for another's result.  The state's rows and the tokens are dealt
// to the accumulators' rows so (paired()) that one product's results are, lane by lane, the next one's right operand:
// nothing between the products passes through LDS (but in fp32, see below).  What the four waves share are the chunk's
// tiles, the left operands.
//
// bf16: the tiles of the next chunk are fetched into a second buffer by four waves that do nothing else.  (A wave's next
// load waits until the memory path has taken its last one, 57 to 90 cycles; the waves that compute spent two thirds of a
// chunk's 3.7 us on issuing those loads, and one fetching wave still took longer than a chunk.)  The tiles of two chunks
// and some 250 registers a wave make it one workgroup a compute unit.
//
// bf16: S, X, U and, where O is wanted, T' enter the products of the state in two parts of 8 bits of significand each
// (three products of four for T' X): the state that the forward hands on is fp32 and stays as exact as sums of fp32
// products to some 4e-6; in one part each it would be off by 2.4e-3.  O, rounded to bf16 anyway, takes the larger parts
// alone, and so do the gradients, but for the state that they carry along.
//
// fp32 (matrix products at a sixteenth of the bf16 rate, which bound it): while there are workgroups for no more than
// half of the compute units, two waves share 16 columns, each with half of the features, and add their parts of K S and
// Q S through LDS.  Two rows of 700 tokens, 8 heads of 64: forward 75 -> 59 us, the gradients' sweeps 53 -> 40 and 84 -> 66
// by themselves.  (bf16 gains nothing from it: one prompt of 3001 tokens 116 us either way.)
//
// What bounds them, heads of 128 features: 256 or more workgroups, HBM (4 rows of 8192 tokens, 32 heads, bf16: forward 316
// us at 4.6 TB/s, the gradients' two 650 at 5.1); fewer, a chunk's chain of dependent steps, 1.9 to 2.8 us: of the
// forward's 4500 cycles matrix products take 1660 and vector instructions 1990, which one wave a SIMD hardly overlaps
// (asked to interleave them, the compiler ran out of registers: 128 us for 70), and LDS is busy 1580.  One prompt of 3001
// tokens, 47 chunks, 91 us; 8 rows of 2048 tokens, 8 heads: 68 us, and the gradients' two sweeps 90 together (61 and 76 alone).
#include "ltn_delta.h"

namespace ltn {
namespace {

// first of the four tokens (or features) that a lane holds of row tile rt
__device__ __forceinline__ int token_of(int rt, int grp) { return 32 * (rt >> 1) + 8 * grp + 4 * (rt & 1); }

template <class T> __device__ __forceinline__ void store_frag(T* p, const typename El<T>::F& f) { *(typename El<T>::F*)p = f; }
// four fp32 values as four consecutive elements
__device__ __forceinline__ void store4(__bf16* p, const f32x4& x) { *(bf16x4*)p = to_bf16(x); }
__device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }

// A wave's 16 columns of 64 tokens, from a column a lane to a token a lane (16 rows of a tile of a wave's own; a wave's
// accesses to LDS stay in order).
template <class T> struct Turn {
    typedef Tile<T, kChunk> Ti;
    static constexpr int BYTES = 16 * Ti::RB;
    unsigned in, out;
    __device__ __forceinline__ Turn(unsigned lds, int lane, int first) {     // store() numbers row tiles from `first` on
        const int m = lane & 15, grp = lane >> 4;
        in = lds + Ti::chunk(m, sizeof(T) == 2 ? grp : 2 * grp);
        out = sizeof(T) == 2 ? (lds + Ti::at(4 * grp + (m >> 2), 4 * (m & 3))) ^ (first << 5) : lds + Ti::at(4 * grp, m + 16 * first);
    }
    __device__ __forceinline__ void write(int b, const bf16x8& f) const { lds_write(in ^ (b << 6), f); }
    __device__ __forceinline__ void write(int b, const F32Frag& f) const {
        lds_write(in + b * 128, f.a);
        lds_write(in + b * 128 + 16, f.b);
    }
    // (the transposing read takes part of every lane's row: all lanes make it, also those whose token is past the end)
    __device__ __forceinline__ void store(__bf16* p, int rt, bool there) const {
        s16x4 x = lds_read_tr(out ^ (rt << 5));
        asm volatile("" : "+v"(x));
        if (there) *(s16x4*)p = x;
    }
    __device__ __forceinline__ void store(float* p, int rt, bool there) const {
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lds_read<float>(out + 64 * rt + i * Ti::RB);
        if (there) *(f32x4*)p = x;
    }
};

// Nothing is scheduled across it (bf16).  Left to itself the compiler reads an operand from LDS right before its product, to
// save registers, and every product waits for LDS.  So each read is placed where the registers it goes to have just been
// used, a stage or more ahead of its own use.
template <class T> __device__ __forceinline__ void fence() {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
}

// What a wave hands the one that has the other features of its columns: K S (or K dS), and O's other two row tiles.
template <bool SAVE> struct Swap { static constexpr int BYTES = (SAVE ? 4 : 6) * 1024; };

// One chunk's tiles in LDS.  FWD: K, T', V and, where O is wanted, the second part of T' (bf16), Q and P.  Backward: K, Q, T', P, dO.
template <class T, int DK, int COLS, bool FULL, bool FWD> struct SweepLds {
    static constexpr int K = 0, T1 = K + Tile<T, DK>::BYTES, V = T1 + Tile<T, kChunk>::BYTES, VEC = V + Tile<T, COLS>::BYTES,
                         T2 = VEC + 1024, Q = T2 + (FWD && FULL && sizeof(T) == 2 ? Tile<T, kChunk>::BYTES : 0),
                         P = Q + (FULL ? Tile<T, DK>::BYTES : 0), BYTES = P + (FULL ? Tile<T, kChunk>::BYTES : 0);
    static constexpr int BUFS = sizeof(T) == 2 ? 2 : 1, ALL = BUFS * BYTES;                   // of a workgroup
    static_assert(ALL <= 160 * 1024, "LDS");
};

// Waves that compute, and waves that fetch besides them (bf16; fp32: the same, through registers).
constexpr int W = 4, kFetchers = 4;
static_assert(W == kFetchers, "either kind of waves fetches alike");
template <class T> constexpr int kThreadsOf = 64 * (sizeof(T) == 2 ? W + kFetchers : W);

// The fetches of a chunk's tiles.
template <class T, int DK, int COLS, bool FULL, bool FWD> struct SweepFetch {
    typedef SweepLds<T, DK, COLS, FULL, FWD> L;
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr size_t kTile = (size_t)kChunk * kChunk * sizeof(T);
    TileFetch<T, DK, W, kChunk, true> k, q;
    TileFetch<T, kChunk, W, kChunk, true> t1, t2, p;
    TileFetch<T, COLS, W, kChunk, true> v;
    u32x4 vec;
    // at: the chunk's scratch; key_row, val_row: its first token's rows
    __device__ __forceinline__ void fetch(const DeltaArgs& a, size_t at, size_t key_row, size_t val_row, int rows, int Dv, int col0,
                                          unsigned lds, int w, int lane) {
        k.fetch((const char*)a.k + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, lds + L::K, w, lane);
        t1.fetch(a.tq + at * kTile, kChunk * sizeof(T), kChunk, lds + L::T1, w, lane);
        v.fetch((const char*)(FWD ? a.v : a.d_o) + (val_row * Dv + col0) * sizeof(T), Dv * sizeof(T), rows, lds + L::V, w, lane);
        if constexpr (FWD && FULL && BF) t2.fetch(a.tl + at * kTile, kChunk * sizeof(T), kChunk, lds + L::T2, w, lane);
        if constexpr (FULL) {
            q.fetch((const char*)a.q + key_row * (DK * sizeof(T)), DK * sizeof(T), rows, lds + L::Q, w, lane);
            p.fetch(a.p + at * kTile, kChunk * sizeof(T), kChunk, lds + L::P, w, lane);
        }
        if (w == 0) {                      // 768 bytes of decays and beta (what else the kilobyte receives is not read)
            const char* src = (const char*)(a.vec + at * kVec) + (lane < 48 ? lane * 16 : 0);
            if constexpr (BF) dma16(lds + L::VEC, src);
            else vec = *(const u32x4*)src;
        }
    }
    __device__ __forceinline__ void put(unsigned lds, int w, int lane) const {
        if constexpr (!BF) {
            k.put(lds + L::K, w, lane);
            t1.put(lds + L::T1, w, lane);
            v.put(lds + L::V, w, lane);
            if constexpr (FULL) {
                q.put(lds + L::Q, w, lane);
                p.put(lds + L::P, w, lane);
            }
            if (w == 0) lds_write(lds + L::VEC + lane * 16, vec);
        }
    }
};

// Forward.  SAVE: Z and the states before chunks are written, for the gradients, and O is not.
template <class T, int DK, int KS, bool SAVE>
__device__ __forceinline__ void forward_sweep(const DeltaArgs& a, int Dv, int per_chain, int wg) {
    constexpr bool BF = sizeof(T) == 2;
    static_assert(KS == 1 || !BF, "the waves that fetch take no part in the exchange");
    constexpr int COLS = 16 * W / KS, NT = DK / 16 / KS, NP = NT / 2, NO = 4 / KS;
    typedef typename El<T>::F F;
    typedef SweepLds<T, DK, COLS, !SAVE, true> L;
    extern __shared__ __attribute__((aligned(1024))) char lds[];        // (of a size unknown to the compiler, which would else plan for one wave a SIMD and move accumulators to and fro)

    int chain, split;
    map_workgroup(wg, per_chain, a.seqs * a.H, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, grp = lane >> 4;
    const unsigned lds0 = lds_address(lds);
    const int wg0 = split * COLS, c0 = 16 * (w / KS), part = w % KS, f0 = part * (DK / KS);    // the workgroup's and the wave's first column, the wave's first feature
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first;
    const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first;

    const int chunks = (s.len + kChunk - 1) / kChunk;
    SweepFetch<T, DK, COLS, !SAVE, true> next;
    auto fetch = [&](int chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        next.fetch(a, (size_t)(s.slot + chunk) * a.H + h, key_row + t0, val_row + t0, rows, Dv, wg0,
                   lds0 + (BF ? (chunk & 1) * L::BYTES : 0), BF ? w - W : w, lane);
    };
    if (BF && w >= W) {
        if (chunks) fetch(0);
        for (int chunk = 0; chunk < chunks; ++chunk) {
            wait_dma<0>();
            __syncthreads();               // this chunk's tiles are there, the last one's are read
            if (chunk + 1 < chunks) fetch(chunk + 1);
        }
        return;
    }
    f32x4 S[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.kv_in) {
        const float* in = a.kv_in + ((size_t)chain * DK + f0) * Dv + wg0 + c0 + m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[t][i] = in[(size_t)(token_of(t, grp) + i) * Dv];   // (features are dealt as tokens)
    }
    // The state as an operand, and into memory.  Behind a chunk and not before the next: there the stores would wait until the
    // next tiles' loads have been issued, which keep the memory path busy for 1300 cycles and more.
    F Sh[NP], Sl[BF ? NP : 1];
    auto hand_on = [&](size_t at, bool chunk_there) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            Sh[p] = frag_of<T>(S[2 * p], S[2 * p + 1]);
            if constexpr (BF) Sl[p] = rest_of(Sh[p], S[2 * p], S[2 * p + 1]);
        }
        if constexpr (SAVE)
            if (chunk_there)
#pragma unroll
                for (int p = 0; p < NP; ++p) store_frag<T>((T*)a.s0 + (at * Dv + wg0 + c0 + m) * DK + f0 + 32 * p + 8 * grp, Sh[p]);
    };
    if (!BF && chunks) fetch(0);
    if (BF && chunks) hand_on((size_t)s.slot * a.H + h, true);
    PairedRowReader<T, DK> k_row(lds0, lane);
    ColReader<T, DK, true> k_col(lds0, lane);
    PairedRowReader<T, kChunk> t_row(lds0, lane);
    ColReader<T, COLS, false> v_col(lds0, lane);
    constexpr int RD = Tile<T, DK>::RB, RC = Tile<T, kChunk>::RB;
    // Of O a wave ends with row tiles part, part + KS, ..: Q's rows for these and for the others', P's for these
    RowReader<T, DK> q_row(lds0 + 16 * RD * part, m, lane), q_others(lds0 + 16 * RD * (KS - 1 - part), m, lane);
    RowReader<T, kChunk> p_row(lds0 + 16 * RC * part, m, lane);
    if constexpr (KS > 1) {
        k_row.skip(NP * part);
        k_col.skip(NP * part);
        q_row.skip(NP * part);
        q_others.skip(NP * part);
    }
    const unsigned mine = lds0 + L::ALL + w * Swap<SAVE>::BYTES + lane * 16, others = lds0 + L::ALL + (w ^ 1) * Swap<SAVE>::BYTES + lane * 16;
    unsigned vec = lds0 + L::VEC;          // gam, end, beta
    auto vec4 = [&](int which, int rt) { return lds_read<f32x4>(vec + 32 * grp + 4 * (which * kChunk + token_of(rt, 0))); };
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        next.put(lds0, w, lane);
        __syncthreads();
        if (!BF && chunk + 1 < chunks) fetch(chunk + 1);

        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        F rd[4 * (NP)];            // K's rows, then Q's, then K's columns
        F tf[6], tl[BF ? 6 : 1], pf[6];        // T' (in two parts where O is wanted), P: row tiles 0 .. 3 of the first 32 columns, 2, 3 of the second
        f32x4 V[4], gam[4], bt[4], en[4], Z[4], O[4];
        float row_gam[4];
        auto k_cols = [&](int i) { return k_col.frag(L::K, i / NT, i % NT); };
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) rd[i] = k_row.frag(L::K, i % 4, i / 4);
        const float whole = lds_read<float>(vec + 4 * (kChunk - 1));
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            V[rt] = v_col.values(L::V, rt, c0 / 16);
            gam[rt] = vec4(0, rt);
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) tf[i] = t_row.frag(L::T1, i < 4 ? i : i - 2, i / 4);
        fence<T>();
        if constexpr (!BF) hand_on(at, true);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] = mma(rd[4 * p + rt], Sh[p], p ? Z[rt] : zero);
            if constexpr (BF)
#pragma unroll
                for (int rt = 0; rt < 4; ++rt) Z[rt] = mma(rd[4 * p + rt], Sl[p], Z[rt]);
            fence<T>();
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                if constexpr (SAVE) rd[4 * p + rt] = k_cols(4 * p + rt);
                else rd[4 * p + rt] = (rt < NO ? q_row : q_others).frag(L::Q + 16 * KS * (rt % NO) * RD, p);
            }
            fence<T>();
        }
        auto q_state = [&] {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
#pragma unroll
                for (int rt = 0; rt < 4; ++rt) O[rt] = mma(Sh[p], rd[4 * p + rt], p ? O[rt] : zero);
                fence<T>();
#pragma unroll
                for (int rt = 0; rt < 4; ++rt) rd[4 * p + rt] = k_cols(4 * p + rt);
                fence<T>();
            }
        };
        if constexpr (KS > 1) {            // the other features' part of K S, and of this wave's tokens of Q S
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) lds_write(mine + 1024 * rt, Z[rt]);
            if constexpr (!SAVE) {
                q_state();
#pragma unroll
                for (int i = 0; i < NO; ++i) lds_write(mine + 1024 * (4 + i), O[NO + i]);
            }
            __syncthreads();
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Z[rt] += lds_read<f32x4>(others + 1024 * rt);
            if constexpr (!SAVE)
#pragma unroll
                for (int i = 0; i < NO; ++i) O[i] += lds_read<f32x4>(others + 1024 * (4 + i));
        }
        if constexpr (BF && !SAVE)
#pragma unroll
            for (int i = 0; i < 6; ++i) tl[i] = t_row.frag(L::T2, i < 4 ? i : i - 2, i / 4);
        fence<T>();
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] = times(S[t], whole);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) Z[rt] = V[rt] - gam[rt] * Z[rt];
        F Xh[2], Xl[BF ? 2 : 1];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            Xh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
            if constexpr (BF) Xl[b] = rest_of(Xh[b], Z[2 * b], Z[2 * b + 1]);
        }
        fence<T>();
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            bt[rt] = vec4(2, rt);
            en[rt] = vec4(1, rt);
            if (!SAVE && rt < NO) row_gam[rt] = lds_read<float>(vec + 4 * (m + 16 * part) + 64 * KS * rt) * a.scale;
        }
        fence<T>();
#pragma unroll
        for (int i = 0; i < 6; ++i) Z[i < 4 ? i : i - 2] = mma(tf[i], Xh[i / 4], Z[i < 4 ? i : i - 2]);
        if constexpr (BF) {
#pragma unroll
            for (int i = 0; i < 6; ++i) Z[i < 4 ? i : i - 2] = mma(tf[i], Xl[i / 4], Z[i < 4 ? i : i - 2]);
            if constexpr (!SAVE)
#pragma unroll
                for (int i = 0; i < 6; ++i) Z[i < 4 ? i : i - 2] = mma(tl[i], Xh[i / 4], Z[i < 4 ? i : i - 2]);
        }
        fence<T>();
        // O transposed, its rows value columns and its columns tokens: a lane's values are neighbours in memory
        if constexpr (!SAVE) {
#pragma unroll
            for (int i = 0; i < NO * 3 / 2; ++i) pf[i] = p_row.frag(L::P + 16 * KS * (i < NO ? i : i - NO / 2) * RC, i / NO);
            fence<T>();
            if constexpr (KS == 1) q_state();
        }
        if constexpr (SAVE) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
                if (KS == 1 || b == part) store_frag<T>((T*)a.z + (at * Dv + wg0 + c0 + m) * kChunk + 32 * b + 8 * grp, frag_of<T>(Z[2 * b], Z[2 * b + 1]));
        }
        F Uh[2], Ul[BF ? 2 : 1];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) Z[rt] *= bt[rt];              // U
        if constexpr (!SAVE) {
#pragma unroll
            for (int b = 0; b < 2; ++b) Uh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
#pragma unroll
            for (int i = 0; i < NO; ++i) O[i] = times(O[i], row_gam[i]);
#pragma unroll
            for (int i = 0; i < NO * 3 / 2; ++i) O[i < NO ? i : i - NO / 2] = mma(Uh[i / NO], pf[i], O[i < NO ? i : i - NO / 2]);
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) Z[rt] *= en[rt];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            Uh[b] = frag_of<T>(Z[2 * b], Z[2 * b + 1]);
            if constexpr (BF) Ul[b] = rest_of(Uh[b], Z[2 * b], Z[2 * b + 1]);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int t = 0; t < NT; ++t) S[t] = mma(rd[b * NT + t], Uh[b], S[t]);
            if constexpr (BF)
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t] = mma(rd[b * NT + t], Ul[b], S[t]);
        }
        if constexpr (!SAVE) {
            T* const out = (T*)a.o + (val_row + t0 + 16 * part + m) * Dv + wg0 + c0 + 4 * grp;
            if (rows == kChunk) {
#pragma unroll
                for (int i = 0; i < NO; ++i) store4(out + (size_t)(16 * KS * i) * Dv, O[i]);
            } else {
#pragma unroll
                for (int i = 0; i < NO; ++i)
                    if (16 * (KS * i + part) + m < rows) store4(out + (size_t)(16 * KS * i) * Dv, O[i]);
            }
        }
        if constexpr (BF) {                // the other buffer
            hand_on(at + a.H, chunk + 1 < chunks);
            const int by = chunk & 1 ? -L::BYTES : L::BYTES;
            k_row.move(by);
            k_col.move(by);
            t_row.move(by);
            v_col.move(by);
            q_row.move(by);
            q_others.move(by);
            p_row.move(by);
            vec += by;
        } else {
            __syncthreads();
        }
    }
    if (!SAVE && a.kv_out) {
        float* const out = a.kv_out + ((size_t)chain * DK + f0) * Dv + wg0 + c0 + m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) out[(size_t)(token_of(t, grp) + i) * Dv] = S[t][i];
    }
}

// Backward, from the last chunk to the first: dV and the derivatives of the states behind chunks.
template <class T, int DK, int KS>
__device__ __forceinline__ void backward_sweep(const DeltaArgs& a, int Dv, int per_chain, int wg) {
    constexpr bool BF = sizeof(T) == 2;
    static_assert(KS == 1 || !BF, "the waves that fetch take no part in the exchange");
    constexpr int COLS = 16 * W / KS, NT = DK / 16 / KS, NP = NT / 2;
    typedef typename El<T>::F F;
    typedef SweepLds<T, DK, COLS, true, false> L;
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    int chain, split;
    map_workgroup(wg, per_chain, a.seqs * a.H, chain, split);
    const int seq = chain / a.H, h = chain % a.H;
    const DeltaSeq s = delta_seq(a, seq);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, grp = lane >> 4;
    const unsigned lds0 = lds_address(lds);
    const int wg0 = split * COLS, c0 = 16 * (w / KS), part = w % KS, f0 = part * (DK / KS);
    const size_t key_row = ((size_t)s.row * a.Hk + h / (a.H / a.Hk)) * a.N + s.first;
    const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first;

    f32x4 S[NT];                       // dS
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (s.len + kChunk - 1) / kChunk;
    SweepFetch<T, DK, COLS, true, false> next;
    auto fetch = [&](int chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        next.fetch(a, (size_t)(s.slot + chunk) * a.H + h, key_row + t0, val_row + t0, rows, Dv, wg0,
                   lds0 + (BF ? (chunk & 1) * L::BYTES : 0), BF ? w - W : w, lane);
    };
    if (BF && w >= W) {
        if (chunks) fetch(chunks - 1);
        for (int chunk = chunks - 1; chunk >= 0; --chunk) {
            wait_dma<0>();
            __syncthreads();
            if (chunk) fetch(chunk - 1);
        }
        return;
    }
    F Sf[NP];
    auto hand_on = [&](size_t at, bool chunk_there) {      // (as in the forward)
#pragma unroll
        for (int p = 0; p < NP; ++p) Sf[p] = frag_of<T>(S[2 * p], S[2 * p + 1]);
        if (chunk_there)
#pragma unroll
            for (int p = 0; p < NP; ++p) store_frag<T>((T*)a.ds + (at * Dv + wg0 + c0 + m) * DK + f0 + 32 * p + 8 * grp, Sf[p]);
    };
    if (!BF && chunks) fetch(chunks - 1);
    if (BF && chunks) hand_on((size_t)(s.slot + chunks - 1) * a.H + h, true);
    const unsigned first = lds0 + (BF && (chunks - 1) & 1 ? L::BYTES : 0);
    PairedRowReader<T, DK> k_row(first, lane);
    ColReader<T, DK, true> k_col(first, lane);
    ColReader<T, kChunk, true> t_col(first, lane);
    ColReader<T, COLS, false> v_col(first, lane);
    if constexpr (KS > 1) {
        k_row.skip(NP * part);
        k_col.skip(NP * part);
    }
    unsigned vec = first + L::VEC;
    auto vec4 = [&](int which, int rt) { return lds_read<f32x4>(vec + 32 * grp + 4 * (which * kChunk + token_of(rt, 0))); };
    const Turn<T> turn(lds0 + L::ALL + w * Turn<T>::BYTES, lane, part);
    const unsigned swap = lds0 + L::ALL + W * Turn<T>::BYTES + lane * 16, mine = swap + w * Swap<true>::BYTES, others = swap + (w ^ 1) * Swap<true>::BYTES;
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
        const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        const size_t at = (size_t)(s.slot + chunk) * a.H + h;
        next.put(lds0, w, lane);
        __syncthreads();
        if (!BF && chunk) fetch(chunk - 1);

        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        F rd[2 * NT];                  // K's rows, then Q's columns, then K's
        // dO's columns; columns of P and T': row tiles 0 .. 3 of the second 32 rows, 0, 1 of the first
        F gf[2], pf[6], tf[6];
        f32x4 gam[4], en[4], bt[4], Y[4];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) rd[i] = k_row.frag(L::K, i % 4, i / 4);
        const float whole = lds_read<float>(vec + 4 * (kChunk - 1));
#pragma unroll
        for (int b = 0; b < 2; ++b) gf[b] = v_col.frag(L::V, b, c0 / 16);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            en[rt] = vec4(1, rt);
            gam[rt] = vec4(0, rt);
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) pf[i] = t_col.frag(L::P, i < 4, i < 4 ? i : i - 4);
        fence<T>();
        if constexpr (!BF) hand_on(at, true);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Y[rt] = mma(rd[4 * p + rt], Sf[p], p ? Y[rt] : zero);
            fence<T>();
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) rd[4 * p + rt] = k_col.frag(L::Q, (4 * p + rt) / NT, (4 * p + rt) % NT);
            fence<T>();
        }
        if constexpr (KS > 1) {            // the other features' part of K dS
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) lds_write(mine + 1024 * rt, Y[rt]);
            __syncthreads();
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) Y[rt] += lds_read<f32x4>(others + 1024 * rt);
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) tf[i] = t_col.frag(L::T1, i < 4, i < 4 ? i : i - 4);
        fence<T>();
        F of[2];                       // scale gam dO
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x4 o0, o1;
            values_of(gf[b], o0, o1);
            of[b] = frag_of<T>(times(gam[2 * b] * o0, a.scale), times(gam[2 * b + 1] * o1, a.scale));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] = times(S[t], whole);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) Y[rt] *= en[rt];
        fence<T>();
#pragma unroll
        for (int i = 0; i < 6; ++i) Y[i < 4 ? i : i - 4] = mma(pf[i], gf[i < 4], Y[i < 4 ? i : i - 4]);
        fence<T>();
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) bt[rt] = vec4(2, rt);
        fence<T>();
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] = mma(rd[t], of[0], S[t]);
        fence<T>();
#pragma unroll
        for (int t = 0; t < NT; ++t) rd[t] = k_col.frag(L::K, 0, t);
        fence<T>();
        F uf[2];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) Y[rt] *= bt[rt];
#pragma unroll
        for (int b = 0; b < 2; ++b) uf[b] = frag_of<T>(Y[2 * b], Y[2 * b + 1]);
#pragma unroll
        for (int i = 0; i < 6; ++i) Y[i < 4 ? i : i - 4] = mma(tf[i], uf[i < 4], Y[i < 4 ? i : i - 4]);
        fence<T>();
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] = mma(rd[NT + t], of[1], S[t]);
        fence<T>();
#pragma unroll
        for (int t = 0; t < NT; ++t) rd[NT + t] = k_col.frag(L::K, 1, t);
        fence<T>();
        // dV, turned round in LDS for its rows in memory: written a column a lane, read four columns of a token a lane
#pragma unroll
        for (int b = 0; b < 2; ++b) turn.write(b, frag_of<T>(Y[2 * b], Y[2 * b + 1]));
        F xf[2];                       // -gam dV
#pragma unroll
        for (int b = 0; b < 2; ++b) xf[b] = frag_of<T>(-gam[2 * b] * Y[2 * b], -gam[2 * b + 1] * Y[2 * b + 1]);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t) S[t] = mma(rd[b * NT + t], xf[b], S[t]);
        T* const out = (T*)a.dv + (val_row + t0 + 16 * part + m) * Dv + wg0 + c0 + 4 * grp;
        // (of one wave, and in order: no wait but the reads' own)
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 4 / KS; ++i) turn.store(out + (size_t)(16 * KS * i) * Dv, KS * i, 16 * (KS * i + part) + m < rows);
        if constexpr (BF) {
            hand_on(at - a.H, chunk > 0);
            const int by = chunk & 1 ? -L::BYTES : L::BYTES;
            k_row.move(by);
            k_col.move(by);
            t_col.move(by);
            v_col.move(by);
            vec += by;
        } else {
            __syncthreads();
        }
    }
}

template <class T, int DK, int KS>
__global__ __launch_bounds__(kThreadsOf<T>) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1)))
void delta_fwd_kernel(DeltaArgs a, int Dv, int per_chain) {
    forward_sweep<T, DK, KS, false>(a, Dv, per_chain, blockIdx.x);
}

// The gradients' two sweeps do not need each other: the first half of the workgroups go backward, which takes longer, and the
// second half save the states.  Where chains are few, they have the units that one sweep alone would leave idle.
template <class T, int DK, int KS>
__global__ __launch_bounds__(kThreadsOf<T>) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1)))
void delta_bwd_kernel(DeltaArgs a, int Dv, int per_chain) {
    const int half = gridDim.x / 2, wg = blockIdx.x;
    if (wg < half) backward_sweep<T, DK, KS>(a, Dv, per_chain, wg);
    else forward_sweep<T, DK, KS, true>(a, Dv, per_chain, wg - half);
}

template <class T, int DK, int KS>
hipError_t launch_fwd_ks(const DeltaArgs& a, int Dv, hipStream_t stream) {
    constexpr int COLS = 16 * W / KS, LDS = SweepLds<T, DK, COLS, true, true>::ALL + (KS > 1 ? W * Swap<false>::BYTES : 0);
    static_assert(LDS <= 160 * 1024, "LDS");
    hipLaunchKernelGGL((delta_fwd_kernel<T, DK, KS>), dim3((unsigned)((long long)a.seqs * a.H * (Dv / COLS))), dim3(kThreadsOf<T>), LDS, stream, a, Dv, Dv / COLS);
    return hipGetLastError();
}
template <class T, int DK, int KS>
hipError_t launch_bwd_ks(const DeltaArgs& a, int Dv, hipStream_t stream) {
    constexpr int COLS = 16 * W / KS, LDS = SweepLds<T, DK, COLS, true, false>::ALL + W * (Turn<T>::BYTES + (KS > 1 ? Swap<true>::BYTES : 0));
    static_assert(LDS <= 160 * 1024 && LDS >= SweepLds<T, DK, COLS, false, true>::ALL + (KS > 1 ? W * Swap<true>::BYTES : 0), "LDS");
    hipLaunchKernelGGL((delta_bwd_kernel<T, DK, KS>), dim3((unsigned)(2 * (long long)a.seqs * a.H * (Dv / COLS))), dim3(kThreadsOf<T>), LDS, stream, a, Dv, Dv / COLS);
    return hipGetLastError();
}
// fp32, while each of twice as many workgroups (of both sweeps, in the gradients) has a compute unit of its own: two waves
// share 16 columns.  Forward of sequences of 700 tokens, heads of 128 features, a wave a column and half a wave: 32 workgroups
// 123 and 94 us, 128 (the last that share) 140 and 111, 256 164 and 212, 512 333 and 437.  Gradients, whole calls: 2 x 16
// of 64 features 112 and 95 us, 2 x 128 214 and 233; 2 x 32 of 128 features 192 and 147, 2 x 128 299 and 305.
bool shared_columns(const DeltaArgs& a, int Dv, int sweeps) { return (long long)a.seqs * a.H * (Dv / (16 * W)) * 2 * sweeps <= 256; }
template <class T, int DK>
hipError_t launch_fwd_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    if constexpr (sizeof(T) == 4)
        if (shared_columns(a, Dv, 1)) return launch_fwd_ks<T, DK, 2>(a, Dv, stream);
    return launch_fwd_ks<T, DK, 1>(a, Dv, stream);
}
template <class T, int DK>
hipError_t launch_bwd_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    if constexpr (sizeof(T) == 4)
        if (shared_columns(a, Dv, 2)) return launch_bwd_ks<T, DK, 2>(a, Dv, stream);
    return launch_bwd_ks<T, DK, 1>(a, Dv, stream);
}

}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    if (a.slots > 0) {
        const hipError_t e = launch_delta_prepare(a, Dk, is_bf16, stream);
        if (e != hipSuccess) return e;
    }
    if (Dk == 64) return is_bf16 ? launch_fwd_t<__bf16, 64>(a, Dv, stream) : launch_fwd_t<float, 64>(a, Dv, stream);
    return is_bf16 ? launch_fwd_t<__bf16, 128>(a, Dv, stream) : launch_fwd_t<float, 128>(a, Dv, stream);
}

hipError_t launch_delta_bwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    hipError_t e = launch_delta_prepare(a, Dk, is_bf16, stream);
    if (e != hipSuccess) return e;
    if (Dk == 64) e = is_bf16 ? launch_bwd_t<__bf16, 64>(a, Dv, stream) : launch_bwd_t<float, 64>(a, Dv, stream);
    else e = is_bf16 ? launch_bwd_t<__bf16, 128>(a, Dv, stream) : launch_bwd_t<float, 128>(a, Dv, stream);
    if (e != hipSuccess) return e;
    return launch_delta_grad(a, Dk, Dv, is_bf16, stream);
}

}  // namespace ltn
