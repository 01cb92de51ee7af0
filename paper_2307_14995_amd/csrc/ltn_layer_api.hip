// C-ABI layer of the gated delta rule and of the norms around a block: argument validation (host only, before any launch)
// and dispatch.  See include/ltn_attn.h for the contract.
#include "../../include/ltn_attn.h"
#include "ltn_args.h"
#include "ltn_delta.h"
#include "ltn_kernels.h"

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

template <class... P> bool any_null(P... p) { return (... || (p == nullptr)); }
template <class... P> bool all_aligned16(P... p) { return (... && aligned16(p)); }

// Sizes of a delta call in elements; `rows` sequences' states.
struct DeltaDims {
    long long chains, states, slots;
    size_t qk, vo, gates, state;           // bytes of a [.., Hk, N, Dk], a [.., H, N, Dv], an fp32 [.., H, N], the states
};

ltn_status check_delta(int Bt, int Hk, int H, long long N, int Dk, int Dv, bool packed, int seqs, ltn_dtype dtype, DeltaDims* d) {
    if (Bt < 0 || Hk < 0 || H < 0 || N < 0 || Dk <= 0 || Dv <= 0 || (packed && (seqs < 0 || Bt != 1))) return LTN_ERR_SHAPE;
    if (dtype != LTN_F32 && dtype != LTN_BF16) return LTN_ERR_UNSUPPORTED;
    if ((Dk != 64 && Dk != 128) || (Dv != 64 && Dv != 128)) return LTN_ERR_UNSUPPORTED;
    if (H > 0 && (Hk == 0 || H % Hk)) return LTN_ERR_SHAPE;
    if (N > 0x7fffffffLL - 64) return LTN_ERR_SHAPE;
    const long long rows = packed ? seqs : Bt;
    d->chains = rows * H;
    d->slots = ltn::delta_slots(rows, N, packed);
    // (a launch has a workgroup per chunk and head, or up to four per chain)
    if (rows * H > 0x1fffffffLL || d->slots > 0x7fffffffLL / (H ? H : 1)) return LTN_ERR_SHAPE;
    const size_t e = esize_of(dtype), tokens = (size_t)Bt * (size_t)N;
    d->qk = tokens * Hk * Dk * e;
    d->vo = tokens * H * Dv * e;
    d->gates = tokens * H * sizeof(float);
    d->state = (size_t)d->chains * Dk * Dv * sizeof(float);
    return LTN_OK;
}

// A launch has less than 2^32 threads in its grid: the sweeps up to 2048 a chain, "grad" 512 a chunk and head.
bool launches(const DeltaDims& d, int H) { return d.chains < (1 << 21) && d.slots * H < (1 << 23); }

// Hands out the workspace's arrays; returns its size.
size_t lay_out(ltn::DeltaArgs& a, char* base, int Dk, int Dv, bool bf16, bool bwd) {
    const ltn::DeltaScratch s = ltn::delta_scratch(Dk, Dv, bf16);
    const size_t n = (size_t)a.slots * a.H;
    char* p = base;
    auto take = [&](size_t bytes) {
        char* const at = p;
        p += n * bytes;
        return at;
    };
    a.tq = take(s.tile);
    if (bf16 && !bwd) a.tl = take(s.tile);
    a.p = take(s.tile);
    a.vec = reinterpret_cast<float*>(take(s.vec));
    if (bwd) {
        a.z = take(s.z);
        a.s0 = take(s.state);
        a.ds = take(s.state);
    }
    return (size_t)(p - base);
}

}  // namespace

size_t ltn_delta_workspace_bytes(int Bt, int H, long long N, int Dk, int Dv, int seqs, ltn_dtype dtype, int call) {
    if (Bt <= 0 || H <= 0 || N <= 0 || seqs < 0 || call < 0 || call > 1) return 0;
    DeltaDims d;
    if (check_delta(Bt, H, H, N, Dk, Dv, seqs > 0, seqs, dtype, &d) != LTN_OK || !launches(d, H)) return 0;
    return (size_t)d.slots * H * ltn::delta_bytes(Dk, Dv, dtype == LTN_BF16, call == 1);
}

ltn_status ltn_delta_fwd(const void* q, const void* k, const void* v, void* o, const float* g, const float* beta,
                         const int* cu, const float* kv_in, float* kv_out, float scale,
                         int Bt, int Hk, int H, long long N, int Dk, int Dv, int seqs, ltn_dtype dtype,
                         void* workspace, size_t workspace_bytes, void* stream) {
    DeltaDims d;
    const ltn_status cs = check_delta(Bt, Hk, H, N, Dk, Dv, cu != nullptr, seqs, dtype, &d);
    if (cs != LTN_OK) return cs;
    if (!launches(d, H)) return LTN_ERR_SHAPE;
    const bool empty = Bt == 0 || H == 0 || N == 0;
    if (!empty && any_null(q, k, v, (const void*)o, (const void*)g, (const void*)beta)) return LTN_ERR_NULL;
    const size_t need = ltn_delta_workspace_bytes(Bt, H, N, Dk, Dv, cu ? seqs : 0, dtype, 0);
    if (workspace_bytes < need) return LTN_ERR_SHAPE;
    if (need && !workspace) return LTN_ERR_NULL;
    if (!all_aligned16(q, k, v, o, kv_in, kv_out, workspace) || !aligned4(g) || !aligned4(beta) || !aligned4(cu)) return LTN_ERR_ALIGN;
    const Span ins[7] = {{q, d.qk}, {k, d.qk}, {v, d.vo}, {g, d.gates}, {beta, d.gates},
                         {cu, ((size_t)seqs + 1) * sizeof(int)}, {kv_in == kv_out ? nullptr : kv_in, d.state}};
    const Span outs[3] = {{o, d.vo}, {kv_out, d.state}, {workspace, need}};
    if (outputs_alias(outs, 3, ins, 7)) return LTN_ERR_UNSUPPORTED;
    if (d.chains == 0 || (empty && !kv_out)) return LTN_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (empty) return ltn::launch_state_copy(kv_in, kv_out, (size_t)d.chains * Dk * Dv, st) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
    ltn::DeltaArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.o = o;
    a.g = g;
    a.beta = beta;
    a.kv_in = kv_in;
    a.kv_out = kv_out;
    a.cu = cu;
    a.Hk = Hk;
    a.H = H;
    a.seqs = cu ? seqs : Bt;
    a.N = N;
    a.scale = scale;
    a.slots = (int)d.slots;
    lay_out(a, static_cast<char*>(workspace), Dk, Dv, dtype == LTN_BF16, false);
    return ltn::launch_delta_fwd(a, Dk, Dv, dtype == LTN_BF16, st) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
}

ltn_status ltn_delta_bwd(const void* q, const void* k, const void* v, const void* d_o,
                         void* dq, void* dk, void* dv, void* dg, void* dbeta, const float* g, const float* beta,
                         const int* cu, float scale, int Bt, int Hk, int H, long long N, int Dk, int Dv, int seqs,
                         ltn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream) {
    DeltaDims d;
    const ltn_status cs = check_delta(Bt, Hk, H, N, Dk, Dv, cu != nullptr, seqs, dtype, &d);
    if (cs != LTN_OK) return cs;
    if (!launches(d, H)) return LTN_ERR_SHAPE;
    const bool empty = Bt == 0 || H == 0 || N == 0;
    if (!empty && any_null(q, k, v, d_o, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)dg, (const void*)dbeta,
                           (const void*)g, (const void*)beta))
        return LTN_ERR_NULL;
    const size_t need = ltn_delta_workspace_bytes(Bt, H, N, Dk, Dv, cu ? seqs : 0, dtype, 1);
    if (workspace_bytes < need) return LTN_ERR_SHAPE;
    if (need && !workspace) return LTN_ERR_NULL;
    if (!all_aligned16(q, k, v, d_o, dq, dk, dv, workspace) || !aligned4(dg) || !aligned4(dbeta) || !aligned4(g) ||
        !aligned4(beta) || !aligned4(cu))
        return LTN_ERR_ALIGN;
    const size_t small = d.gates / sizeof(float) * esize_of(dtype);
    const Span ins[7] = {{q, d.qk}, {k, d.qk}, {v, d.vo}, {d_o, d.vo}, {g, d.gates}, {beta, d.gates}, {cu, ((size_t)seqs + 1) * sizeof(int)}};
    const Span outs[6] = {{dq, d.qk}, {dk, d.qk}, {dv, d.vo}, {dg, small}, {dbeta, small}, {workspace, need}};
    if (outputs_alias(outs, 6, ins, 7)) return LTN_ERR_UNSUPPORTED;
    if (empty || d.chains == 0) return LTN_OK;
    ltn::DeltaArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.d_o = d_o;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.dg = dg;
    a.dbeta = dbeta;
    a.g = g;
    a.beta = beta;
    a.cu = cu;
    a.Hk = Hk;
    a.H = H;
    a.seqs = cu ? seqs : Bt;
    a.N = N;
    a.scale = scale;
    a.slots = (int)d.slots;
    lay_out(a, static_cast<char*>(workspace), Dk, Dv, dtype == LTN_BF16, true);
    return ltn::launch_delta_bwd(a, Dk, Dv, dtype == LTN_BF16, static_cast<hipStream_t>(stream)) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
}

ltn_status ltn_delta_decode_steps(const void* q, const void* k, const void* v, void* o, float* kv,
                                  const float* g, const float* beta, float scale,
                                  int Bt, int Hk, int H, int S, int Dk, int Dv, ltn_dtype dtype, void* stream) {
    DeltaDims d;
    const ltn_status cs = check_delta(Bt, Hk, H, S, Dk, Dv, false, 0, dtype, &d);
    if (cs != LTN_OK) return cs;
    const bool empty = Bt == 0 || H == 0 || S == 0;
    if (!empty && any_null(q, k, v, (const void*)o, (const void*)kv, (const void*)g, (const void*)beta)) return LTN_ERR_NULL;
    if (!all_aligned16(q, k, v, o, kv) || !aligned4(g) || !aligned4(beta)) return LTN_ERR_ALIGN;
    const Span ins[5] = {{q, d.qk}, {k, d.qk}, {v, d.vo}, {g, d.gates}, {beta, d.gates}};
    const Span outs[2] = {{o, d.vo}, {kv, d.state}};
    if (outputs_alias(outs, 2, ins, 5)) return LTN_ERR_UNSUPPORTED;
    if (empty) return LTN_OK;
    return ltn::launch_delta_decode(q, k, v, o, kv, g, beta, scale, Bt, Hk, H, S, Dk, Dv, dtype == LTN_BF16,
                                    static_cast<hipStream_t>(stream)) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
}

// ---------------------------------------------------------------------------------------
// The norms around a block.
// ---------------------------------------------------------------------------------------

static ltn_status check_block_norm(const void* gate, float eps, long long rows, long long gates, int C, ltn_dtype dtype) {
    if (rows < 0 || C <= 0 || !(eps >= 0.0f)) return LTN_ERR_SHAPE;
    if (gate && (gates <= 0 || rows % gates)) return LTN_ERR_SHAPE;
    if (dtype != LTN_F32 && dtype != LTN_BF16) return LTN_ERR_UNSUPPORTED;
    if (C % 8 || C > 8192) return LTN_ERR_UNSUPPORTED;
    if (rows > 0x7fffffffLL) return LTN_ERR_SHAPE;
    return LTN_OK;
}

size_t ltn_block_norm_workspace_bytes(long long rows, int C) {
    if (rows <= 0 || C <= 0 || C % 8 || C > 8192 || rows > 0x7fffffffLL) return 0;
    return ltn::block_norm_part_floats(rows, C) * sizeof(float);
}

ltn_status ltn_block_norm_fwd(const void* x, const void* y, const void* gate, const float* w_after, const float* w_before,
                              void* x_out, void* h, float scale, float eps, int after,
                              long long rows, long long gates, int C, ltn_dtype dtype, void* stream) {
    const ltn_status cs = check_block_norm(gate, eps, rows, gates, C, dtype);
    if (cs != LTN_OK) return cs;
    if (!after && w_after) return LTN_ERR_UNSUPPORTED;
    if (rows && any_null(x, y, (const void*)x_out, (const void*)h)) return LTN_ERR_NULL;
    if (!all_aligned16(x, y, gate, w_after, w_before, x_out, h)) return LTN_ERR_ALIGN;
    const size_t tb = (size_t)rows * C * esize_of(dtype), wb = (size_t)C * sizeof(float);
    const Span ins[5] = {{x == x_out ? nullptr : x, tb}, {y, tb}, {gate, gate ? (size_t)gates * C * esize_of(dtype) : 0}, {w_after, wb}, {w_before, wb}};
    const Span outs[2] = {{x_out, tb}, {h, tb}};
    if (outputs_alias(outs, 2, ins, 5)) return LTN_ERR_UNSUPPORTED;
    return ltn::launch_block_norm(x, y, gate, w_after, w_before, nullptr, nullptr, x_out, h, nullptr, nullptr, nullptr, nullptr,
                                  scale, eps, after != 0, rows, gates, C, dtype == LTN_BF16, 0,
                                  static_cast<hipStream_t>(stream)) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
}

ltn_status ltn_block_norm_bwd(const void* x, const void* y, const void* gate, const float* w_after, const float* w_before,
                              const void* d_x_out, const void* d_h, void* d_x, void* d_y, void* d_gate,
                              float* d_w_after, float* d_w_before, float scale, float eps, int after,
                              long long rows, long long gates, int C, ltn_dtype dtype,
                              void* workspace, size_t workspace_bytes, void* stream) {
    const ltn_status cs = check_block_norm(gate, eps, rows, gates, C, dtype);
    if (cs != LTN_OK) return cs;
    if (!after && w_after) return LTN_ERR_UNSUPPORTED;
    if ((rows && any_null(x, y, d_h, (const void*)d_x, (const void*)d_y)) || !gate != !d_gate || !w_after != !d_w_after ||
        !w_before != !d_w_before)
        return LTN_ERR_NULL;
    const size_t need = ltn_block_norm_workspace_bytes(rows, C);
    if (workspace_bytes < need) return LTN_ERR_SHAPE;
    if (need && !workspace) return LTN_ERR_NULL;
    if (!all_aligned16(x, y, gate, w_after, w_before, d_x_out, d_h) || !all_aligned16(d_x, d_y, d_gate, d_w_after, d_w_before, workspace))
        return LTN_ERR_ALIGN;
    const size_t tb = (size_t)rows * C * esize_of(dtype), wb = (size_t)C * sizeof(float), gb = gate ? (size_t)gates * C * esize_of(dtype) : 0;
    const Span ins[7] = {{x, tb}, {y, tb}, {gate, gb}, {w_after, wb}, {w_before, wb}, {d_x_out, tb}, {d_h, tb}};
    const Span outs[6] = {{d_x, tb}, {d_y, tb}, {d_gate, gb}, {d_w_after, wb}, {d_w_before, wb}, {workspace, need}};
    if (outputs_alias(outs, 6, ins, 7)) return LTN_ERR_UNSUPPORTED;
    return ltn::launch_block_norm(x, y, gate, w_after, w_before, d_x_out, d_h, d_x, d_y, d_gate, d_w_after, d_w_before,
                                  static_cast<float*>(workspace), scale, eps, after != 0, rows, gates, C, dtype == LTN_BF16, 1,
                                  static_cast<hipStream_t>(stream)) == hipSuccess ? LTN_OK : LTN_ERR_LAUNCH;
}
