// C ABI of the workers' local gradients (declared in include/lossy_local.h):
// argument checks around the HIP kernels.
#include "lossy_local.h"

#include <hip/hip_runtime.h>

#include "errors.h"
#include "local.h"

using namespace lossy;

static_assert(LL_ACT_GROUP == kActGroup, "checkpoint groups");

namespace {

constexpr int64_t kMaxInt = 0x7FFFFFFFll;
constexpr int32_t kMaxN = 1024;

int check_batch(int32_t n, int64_t t) {
    if (n < 1 || n > kMaxN) return fail(LL_EINVAL, "n=%d outside [1, %d]", n, kMaxN);
    if (t < 0) return fail(LL_EINVAL, "t=%lld is negative", (long long)t);
    if (t > kMaxInt / n)
        return fail(LL_EINVAL, "n * t = %d * %lld exceeds 2^31 - 1", n, (long long)t);
    return LL_OK;
}

int check_width(const char* name, int64_t x) {
    if (x < 1 || x > kMaxInt)
        return fail(LL_EINVAL, "%s=%lld outside [1, 2^31)", name, (long long)x);
    return LL_OK;
}

int check_aligned(const char* name, const void* p, size_t a) {
    if (reinterpret_cast<uintptr_t>(p) % a)
        return fail(LL_EALIGN, "%s is not %zu-byte aligned", name, a);
    return LL_OK;
}

// Strided rows of `width` elements; only looked at where there are tokens.
int check_act(const char* name, const void* p, int64_t ld, int64_t width, size_t esize) {
    if (!p) return fail(LL_EINVAL, "%s is NULL", name);
    if (ld < width)
        return fail(LL_EINVAL, "%s: ld=%lld < width %lld", name, (long long)ld, (long long)width);
    if (ld > (int64_t)1 << 40) return fail(LL_EINVAL, "%s: ld=%lld", name, (long long)ld);
    return check_aligned(name, p, esize);
}

int check_lengths(const int32_t* lengths) { return check_aligned("lengths", lengths, 4); }

int check_tokens(int32_t itype, const void* tokens, int64_t ld_t, int64_t t) {
    if (itype != LL_I32 && itype != LL_I64)
        return fail(LL_EINVAL, "itype: unknown integer type %d", itype);
    if (t == 0) return LL_OK;
    return check_act("tokens", tokens, ld_t, t, itype == LL_I64 ? 8 : 4);
}

// `rows` rows of h elements at `offset` inside every row of [n][ld].
int check_rows_at(const char* name, int32_t dtype, const void* p, int64_t ld, int64_t offset,
                  int64_t rows, int64_t h) {
    int r;
    if ((r = check_dtype(name, dtype))) return r;
    if (offset < 0) return fail(LL_EINVAL, "offset=%lld is negative", (long long)offset);
    const int64_t size = rows * h;  // both below 2^31
    if (ld < size || offset > ld - size)
        return fail(LL_EINVAL, "%s: offset=%lld + %lld * %lld elements exceed ld=%lld", name,
                    (long long)offset, (long long)rows, (long long)h, (long long)ld);
    return check_rows(name, p, ld, size, elem_bytes(dtype));
}

int check_pack(const uint8_t* q, int64_t ld_q, const uint8_t* s, int64_t ld_s, int64_t h) {
    int r = check_act("q", q, ld_q, h, 1);
    if (r) return r;
    return check_act("s", s, ld_s, (h + kActGroup - 1) / kActGroup, 1);
}

int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return LL_OK;
    if (!ws || have < need)
        return fail(LL_EINVAL, "workspace of %zu bytes is smaller than %zu", ws ? have : 0, need);
    return check_aligned("workspace", ws, 16);
}

TokenView token_view(int32_t itype, const void* tokens, int64_t ld_t, int64_t first, int64_t v) {
    return TokenView{tokens, ld_t, first, v, itype == LL_I64};
}

ActView act_view(int32_t dtype, const void* p, int64_t ld) {
    return ActView{const_cast<void*>(p), ld, dtype == LL_BF16};
}

RowView row_view(int32_t dtype, const void* p, int64_t ld, int64_t offset) {
    return RowView{const_cast<void*>(p), ld, offset, dtype == LL_BF16};
}

PackView pack_view(const uint8_t* q, int64_t ld_q, const uint8_t* s, int64_t ld_s) {
    return PackView{const_cast<uint8_t*>(q), ld_q, const_cast<uint8_t*>(s), ld_s};
}

// The launchers refuse a grid that does not fit as hipErrorInvalidConfiguration,
// before any launch.
int launched(hipError_t e, const char* fn) {
    if (e == hipErrorInvalidConfiguration) return fail(LL_EINVAL, "%s: too many workgroups", fn);
    return hip_check(e, fn);
}

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int ll_embed(int32_t n, int64_t t, int64_t h, int64_t v, int64_t first, int32_t itype,
             const void* tokens, int64_t ld_t, const int32_t* lengths, int32_t rdtype,
             const void* replicas, int64_t ld_r, int64_t offset, float scale, int32_t odtype,
             void* out, int64_t ld_o, void* stream) {
    int r;
    if ((r = check_batch(n, t))) return r;
    if ((r = check_width("h", h))) return r;
    if ((r = check_width("v", v))) return r;
    if ((r = check_tokens(itype, tokens, ld_t, t))) return r;
    if ((r = check_lengths(lengths))) return r;
    if ((r = check_rows_at("replicas", rdtype, replicas, ld_r, offset, v, h))) return r;
    if ((r = check_dtype("odtype", odtype))) return r;
    if (t == 0) return ok();
    if ((r = check_act("out", out, ld_o, h, elem_bytes(odtype)))) return r;
    EmbedParams p;
    p.n = n;
    p.t = t;
    p.h = h;
    p.lengths = lengths;
    p.tok = token_view(itype, tokens, ld_t, first, v);
    p.table = row_view(rdtype, replicas, ld_r, offset);
    p.scale = scale;
    p.out = act_view(odtype, out, ld_o);
    return launched(launch_embed(p, as_stream(stream)), "ll_embed");
}

size_t ll_embed_grad_workspace_bytes(int32_t n, int64_t t, int64_t h, int64_t v) {
    if (check_batch(n, t) || check_width("h", h) || check_width("v", v)) return 0;
    return embed_grad_workspace(n, t, h, v);
}

int ll_embed_grad(int32_t n, int64_t t, int64_t h, int64_t v, int64_t first, int32_t itype,
                  const void* tokens, int64_t ld_t, const int32_t* lengths, int32_t ydtype,
                  const void* dy, int64_t ld_y, float scale, int32_t gdtype, void* grads,
                  int64_t ld_g, int64_t offset, int32_t accumulate, void* workspace,
                  size_t ws_bytes, void* stream) {
    int r;
    if ((r = check_batch(n, t))) return r;
    if ((r = check_width("h", h))) return r;
    if ((r = check_width("v", v))) return r;
    if ((r = check_tokens(itype, tokens, ld_t, t))) return r;
    if ((r = check_lengths(lengths))) return r;
    if ((r = check_rows_at("grads", gdtype, grads, ld_g, offset, v, h))) return r;
    if ((r = check_dtype("ydtype", ydtype))) return r;
    if (t > 0 && (r = check_act("dy", dy, ld_y, h, elem_bytes(ydtype)))) return r;
    if ((r = check_workspace(workspace, ws_bytes, embed_grad_workspace(n, t, h, v)))) return r;
    EmbedGradParams p;
    p.n = n;
    p.t = t;
    p.h = h;
    p.lengths = lengths;
    p.tok = token_view(itype, tokens, ld_t, first, v);
    p.dy = act_view(ydtype, dy, ld_y);
    p.scale = scale;
    p.grads = row_view(gdtype, grads, ld_g, offset);
    p.accumulate = accumulate != 0;
    return launched(launch_embed_grad(p, workspace, as_stream(stream)), "ll_embed_grad");
}

int ll_act_pack(int32_t n, int64_t t, int64_t h, const int32_t* lengths, int32_t xdtype,
                const void* x, int64_t ld_x, uint8_t* q, int64_t ld_q, uint8_t* s, int64_t ld_s,
                void* stream) {
    int r;
    if ((r = check_batch(n, t))) return r;
    if ((r = check_width("h", h))) return r;
    if ((r = check_lengths(lengths))) return r;
    if ((r = check_dtype("xdtype", xdtype))) return r;
    if (t == 0) return ok();
    if ((r = check_act("x", x, ld_x, h, elem_bytes(xdtype)))) return r;
    if ((r = check_pack(q, ld_q, s, ld_s, h))) return r;
    PackParams p{n, t, h, lengths, act_view(xdtype, x, ld_x), pack_view(q, ld_q, s, ld_s)};
    return launched(launch_act_pack(p, as_stream(stream)), "ll_act_pack");
}

int ll_act_unpack(int32_t n, int64_t t, int64_t h, const int32_t* lengths, const uint8_t* q,
                  int64_t ld_q, const uint8_t* s, int64_t ld_s, int32_t odtype, void* out,
                  int64_t ld_o, void* stream) {
    int r;
    if ((r = check_batch(n, t))) return r;
    if ((r = check_width("h", h))) return r;
    if ((r = check_lengths(lengths))) return r;
    if ((r = check_dtype("odtype", odtype))) return r;
    if (t == 0) return ok();
    if ((r = check_pack(q, ld_q, s, ld_s, h))) return r;
    if ((r = check_act("out", out, ld_o, h, elem_bytes(odtype)))) return r;
    PackParams p{n, t, h, lengths, act_view(odtype, out, ld_o), pack_view(q, ld_q, s, ld_s)};
    return launched(launch_act_unpack(p, as_stream(stream)), "ll_act_unpack");
}

size_t ll_act_wgrad_workspace_bytes(int32_t n, int64_t t, int64_t o, int64_t h) {
    if (check_batch(n, t) || check_width("o", o) || check_width("h", h)) return 0;
    return act_wgrad_workspace(n, t, o, h);
}

int ll_act_wgrad(int32_t n, int64_t t, int64_t o, int64_t h, const int32_t* lengths,
                 int32_t ydtype, const void* dy, int64_t ld_y, const uint8_t* q, int64_t ld_q,
                 const uint8_t* s, int64_t ld_s, float scale, int32_t gdtype, void* grads,
                 int64_t ld_g, int64_t offset, int32_t accumulate, void* workspace,
                 size_t ws_bytes, void* stream) {
    int r;
    if ((r = check_batch(n, t))) return r;
    if ((r = check_width("o", o))) return r;
    if ((r = check_width("h", h))) return r;
    if ((r = check_lengths(lengths))) return r;
    if ((r = check_rows_at("grads", gdtype, grads, ld_g, offset, o, h))) return r;
    if ((r = check_dtype("ydtype", ydtype))) return r;
    if (t > 0) {
        if ((r = check_act("dy", dy, ld_y, o, elem_bytes(ydtype)))) return r;
        if ((r = check_pack(q, ld_q, s, ld_s, h))) return r;
        // the kernel addresses 32 rows with 31-bit byte offsets
        const int64_t most = 1 << 24;
        if (ld_y >= most || ld_q >= most || ld_s >= most)
            return fail(LL_EINVAL, "dy, q, s: ld=%lld, %lld, %lld not below 2^24", (long long)ld_y,
                        (long long)ld_q, (long long)ld_s);
    }
    if ((r = check_workspace(workspace, ws_bytes, act_wgrad_workspace(n, t, o, h)))) return r;
    WgradParams p;
    p.n = n;
    p.t = t;
    p.o = o;
    p.h = h;
    p.lengths = lengths;
    p.dy = act_view(ydtype, dy, ld_y);
    p.x = pack_view(q, ld_q, s, ld_s);
    p.scale = scale;
    p.grads = row_view(gdtype, grads, ld_g, offset);
    p.accumulate = accumulate != 0;
    return launched(launch_act_wgrad(p, workspace, as_stream(stream)), "ll_act_wgrad");
}

}  // extern "C"
