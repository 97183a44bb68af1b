// Argument marshalling of the serving calls (mla.py, layer.py) in native code.
//
// A decode step is three calls whose kernels together take 14 to 20 us at small sizes; checking the tensors,
// asking for the stream and converting some twenty arguments each in Python took 6 to 8 us per call, so that
// the host set the pace below about 25 us per step.  The functions here read the tensors' fields directly and
// call the C entry point they are given.  They accept what mla.py's checks let through, as far as it is plain torch
// tensors, integers and floats: inputs of the expected types and shapes, tables of int32, and outputs of the
// expected element size with room for the result (their own shape is the caller's, and in mla.py's calls their type).  For anything else
// they return None without having called anything, and mla.py goes through its own checks, which raise.
// No arithmetic, no allocation, no state beyond the entry points' addresses; the interpreter lock is released
// around the call as ctypes does.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include "mla_gfx950.h"
#include "mla_layer_gfx950.h"
#include "mla_masked_gfx950.h"

namespace {

decltype(&mla_absorb_q) p_absorb_q;
decltype(&mla_out_proj) p_out_proj;
decltype(&mla_decode_paged_multi) p_decode;
decltype(&mla_merge_out_proj_multi) p_merge_out_proj;
decltype(&mla_merge_partials) p_merge_partials;
decltype(&mla_cache_append) p_append;
decltype(&mla_rms_norm) p_rms_norm;
decltype(&mla_quantize_rows) p_quantize;
decltype(&mla_gemm_fp8) p_gemm_fp8;
decltype(&mla_rope_queries) p_rope;
decltype(&mla_cache_store) p_store;
decltype(&mla_decode_paged_tree) p_tree;
decltype(&mla_decode_paged_window) p_window;
decltype(&mla_cache_move) p_move;

struct No {};   // the arguments are not of the plain kind

// a contiguous tensor on the GPU
const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) throw No();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) throw No();
    return t;
}

long integer(PyObject* o)
{
    if (!PyLong_CheckExact(o)) throw No();
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v < INT32_MIN || v > INT32_MAX) throw No();
    return v;
}
float real(PyObject* o)
{
    if (!PyFloat_CheckExact(o)) throw No();
    return (float)PyFloat_AS_DOUBLE(o);
}
int dim(int64_t v)
{
    if (v > INT32_MAX) throw No();
    return (int)v;
}
mla_dtype io_type(const at::Tensor& t)
{
    if (t.scalar_type() == at::kFloat) return MLA_F32;
    if (t.scalar_type() == at::kBFloat16) return MLA_BF16;
    throw No();
}
mla_dtype cache_type(const at::Tensor& t)
{
    if (t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e4m3fn) return MLA_FP8_E4M3;
    return io_type(t);
}
void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }
void require(bool ok)
{
    if (!ok) throw No();
}

// an output (or scratch) with room for n elements of `size` bytes
void* room(PyObject* o, int64_t n, size_t size)
{
    const at::Tensor& t = tensor(o);
    require((size_t)t.element_size() == size && t.numel() >= n);
    return t.data_ptr();
}
void* room_or_null(PyObject* o, int64_t n, size_t size) { return o == Py_None ? nullptr : room(o, n, size); }
size_t size_of(mla_dtype io) { return io == MLA_F32 ? 4 : 2; }

// f(): the status of the call it makes
template <typename F> PyObject* guarded(F f)
{
    try {
        return PyLong_FromLong(f());
    } catch (...) {       // No, or what a tensor without storage throws: the caller's own checks find it again
        Py_RETURN_NONE;
    }
}
template <typename F> int unlocked(F f)
{
    PyThreadState* s = PyEval_SaveThread();
    const int r = f();
    PyEval_RestoreThread(s);
    return r;
}

// (x [B, H, K], W [H, K, N], out)
template <typename P> PyObject* projection(P p, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 3);
        const at::Tensor &x = tensor(a[0]), &W = tensor(a[1]);
        require(x.dim() == 3 && W.dim() == 3 && W.size(0) == x.size(1) && W.size(1) == x.size(2) && W.scalar_type() == x.scalar_type());
        const int B = dim(x.size(0)), H = dim(x.size(1)), K = dim(x.size(2)), N = dim(W.size(2));
        const mla_dtype io = io_type(x);
        void *px = x.data_ptr(), *pw = W.data_ptr(), *po = room(a[2], (int64_t)B * H * N, size_of(io)), *s = stream_of(x);
        return unlocked([&] { return p(px, pw, po, B, H, K, N, io, s); });
    });
}
PyObject* absorb_q(PyObject*, PyObject* const* a, Py_ssize_t n) { return projection(p_absorb_q, a, n); }
PyObject* out_proj(PyObject*, PyObject* const* a, Py_ssize_t n) { return projection(p_out_proj, a, n); }

// (dimensions of q_abs, q_abs, q_rope | None, kv_cache, page_table, seq_lens, scale, num_splits, kv_scale | None, workspace,
//  out | None, lse | None, flags); q_abs [B, H, d_c] or [B, T, H, d_c]
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 13);
        const int k = (int)integer(*a++);
        const at::Tensor &q = tensor(a[0]), &kv = tensor(a[2]), &table = tensor(a[3]), &lens = tensor(a[4]), &ws = tensor(a[8]);
        require((k == 3 || k == 4) && q.dim() == k && kv.dim() == 3);
        const int64_t B = q.size(0), T = k == 4 ? q.size(1) : 1, H = q.size(k - 2), d_c = q.size(k - 1);
        const int64_t pages = kv.size(0), page = kv.size(1), d_rope = kv.size(2) - d_c;
        require(d_rope >= 0);
        void* pr = nullptr;
        if (a[1] != Py_None) {
            const at::Tensor& r = tensor(a[1]);
            if (d_rope) {
                require(r.dim() == k && r.size(0) == B && r.size(k - 2) == H && r.size(k - 1) == d_rope && (k == 3 || r.size(1) == T) &&
                        r.scalar_type() == q.scalar_type());
            }
            pr = r.data_ptr();
        } else {
            require(d_rope == 0);
        }
        require(table.scalar_type() == at::kInt && lens.scalar_type() == at::kInt && table.dim() == 2 && table.size(0) == B &&
                lens.dim() == 1 && lens.size(0) == B);
        const float* ps = nullptr;
        if (a[7] != Py_None) {
            const at::Tensor& s = tensor(a[7]);
            require(s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == pages && s.size(1) == page);
            ps = static_cast<const float*>(s.data_ptr());
        }
        const mla_dtype io = io_type(q), cache = cache_type(kv);
        void *pq = q.data_ptr(), *pkv = kv.data_ptr(), *pws = ws.data_ptr();
        void *po = room_or_null(a[9], q.numel(), size_of(io)), *pl = room_or_null(a[10], B * T * H, 4);
        const auto* pt = static_cast<const int32_t*>(table.data_ptr());
        const auto* pn = static_cast<const int32_t*>(lens.data_ptr());
        const size_t bytes = ws.nbytes();
        const float scale = real(a[5]);
        const int splits = (int)integer(a[6]), flags = (int)integer(a[11]);
        const int b = dim(B), t = dim(T), h = dim(H), dc = dim(d_c), dr = dim(d_rope), pg = dim(page), np = dim(pages), mp = dim(table.size(1));
        void* s = stream_of(q);
        return unlocked([&] {
            return p_decode(pq, pr, pkv, ps, pt, pn, po, static_cast<float*>(pl), pws, bytes, b, t, h, dc, dr, pg, np, mp, splits, scale, io,
                            cache, (unsigned)flags, s);
        });
    });
}

// (workspace, W_UV, o_lat, lse | None, out, B, q_len, num_splits, flags)
PyObject* merge_out_proj(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 9);
        const at::Tensor &ws = tensor(a[0]), &W = tensor(a[1]);
        require(W.dim() == 3);
        const int B = (int)integer(a[5]), T = (int)integer(a[6]), S = (int)integer(a[7]), flags = (int)integer(a[8]);
        const int H = dim(W.size(0)), d_c = dim(W.size(1)), d_head = dim(W.size(2));
        const mla_dtype io = io_type(W);
        require(B >= 0 && B <= 65535 && T >= 0 && T <= 65535 && (int64_t)B * T <= 65535 && H <= 65535);   // (no more is taken: the products below fit)
        const int64_t rows = (int64_t)B * T * H;
        void *pws = ws.data_ptr(), *pw = W.data_ptr(), *po = room(a[2], rows * d_c, size_of(io)), *pl = room_or_null(a[3], rows, 4),
             *pout = room(a[4], rows * d_head, size_of(io));
        const size_t bytes = ws.nbytes();
        void* s = stream_of(ws);
        return unlocked([&] {
            return p_merge_out_proj(pws, bytes, pw, po, static_cast<float*>(pl), pout, B, T, H, d_c, d_head, S, io, (unsigned)flags, s);
        });
    });
}

// (workspace, out, lse | None, B, H, d_c, num_splits, flags)
PyObject* merge_partials(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 8);
        const at::Tensor &ws = tensor(a[0]), &out = tensor(a[1]);
        const int B = (int)integer(a[3]), H = (int)integer(a[4]), d_c = (int)integer(a[5]), S = (int)integer(a[6]), flags = (int)integer(a[7]);
        const mla_dtype io = io_type(out);
        require(B >= 0 && B <= 65535 && H >= 0 && H <= 65535 && d_c >= 0);
        void *pws = ws.data_ptr(), *po = room(a[1], (int64_t)B * H * d_c, size_of(io)), *pl = room_or_null(a[2], (int64_t)B * H, 4);
        const size_t bytes = ws.nbytes();
        void* s = stream_of(ws);
        return unlocked([&] { return p_merge_partials(pws, bytes, po, static_cast<float*>(pl), B, H, d_c, S, io, (unsigned)flags, s); });
    });
}

// (x, W_DKVR, kv_cache, kv_scale | None, page_table, positions, workspace, d_c, rope_base)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 9);
        const at::Tensor &x = tensor(a[0]), &W = tensor(a[1]), &kv = tensor(a[2]), &table = tensor(a[4]), &pos = tensor(a[5]), &ws = tensor(a[6]);
        require(x.dim() == 2 && W.dim() == 2 && kv.dim() == 3 && table.dim() == 2);
        require(W.size(0) == x.size(1) && W.size(1) == kv.size(2) && W.scalar_type() == x.scalar_type());
        require(table.scalar_type() == at::kInt && table.size(0) >= x.size(0) && pos.scalar_type() == at::kInt && pos.numel() >= x.size(0));
        const int d_c = (int)integer(a[7]);
        void *px = x.data_ptr(), *pw = W.data_ptr(), *pkv = kv.data_ptr(), *ps = room_or_null(a[3], kv.size(0) * kv.size(1), 4),
             *pws = ws.data_ptr();
        const auto* pt = static_cast<const int32_t*>(table.data_ptr());
        const auto* pp = static_cast<const int32_t*>(pos.data_ptr());
        const int B = dim(x.size(0)), D = dim(x.size(1)), d_rope = dim(W.size(1)) - d_c, page = dim(kv.size(1)), pages = dim(kv.size(0)),
                  mp = dim(table.size(1));
        const float base = real(a[8]);
        const mla_dtype io = io_type(x), cache = cache_type(kv);
        const size_t bytes = (size_t)ws.numel();
        void* s = stream_of(x);
        return unlocked([&] {
            return p_append(px, pw, pkv, static_cast<float*>(ps), pt, pp, pws, bytes, B, D, d_c, d_rope, page, pages, mp, base, io, cache, s);
        });
    });
}

// ---- the operators around the attention (layer.py)

// a tensor on the GPU whose last axis is dense
const at::Tensor& dense_rows(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) throw No();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() < 1 || (t.stride(-1) != 1 && t.size(-1) != 1)) throw No();
    return t;
}
bool is_codes(const at::Tensor& t) { return t.scalar_type() == at::kFloat8_e4m3fn || t.scalar_type() == at::kByte; }
int64_t scale_blocks(int64_t n) { return (n + 127) / 128; }

// Outputs of these calls are of the type that is written there, not only of its size (values of x's type, codes, fp32 scales).
void* values_or_null(PyObject* o, int64_t n, const at::Tensor& x)
{
    void* p = room_or_null(o, n, (size_t)x.element_size());
    require(!p || THPVariable_Unpack(o).scalar_type() == x.scalar_type());
    return p;
}
uint8_t* codes_or_null(PyObject* o, int64_t n)
{
    void* p = room_or_null(o, n, 1);
    require(!p || is_codes(THPVariable_Unpack(o)));
    return static_cast<uint8_t*>(p);
}
float* scales_or_null(PyObject* o, int64_t n)
{
    void* p = room_or_null(o, n, 4);
    require(!p || THPVariable_Unpack(o).scalar_type() == at::kFloat);
    return static_cast<float*>(p);
}

// distance of the rows of x [T, D]
int64_t row_pitch(const at::Tensor& x) { return x.size(0) > 1 ? x.stride(0) : x.size(1); }

// (x [T, D], weight | None, eps, residual | None, residual_out | None, out | None, codes | None, scales | None)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 8);
        const at::Tensor& x = dense_rows(a[0]);
        require(x.dim() == 2 && (a[3] == Py_None) == (a[4] == Py_None) && (a[6] == Py_None) == (a[7] == Py_None));
        const int64_t T = x.size(0), D = x.size(1);
        const mla_dtype io = io_type(x);
        const void *pw = nullptr, *pr = nullptr;
        if (a[1] != Py_None) {
            const at::Tensor& w = tensor(a[1]);
            require(w.dim() == 1 && w.size(0) == D && w.scalar_type() == x.scalar_type());
            pw = w.data_ptr();
        }
        if (a[3] != Py_None) {
            const at::Tensor& r = tensor(a[3]);
            require(r.dim() == 2 && r.size(0) == T && r.size(1) == D && r.scalar_type() == x.scalar_type());
            pr = r.data_ptr();
        }
        void *pro = values_or_null(a[4], T * D, x), *py = values_or_null(a[5], T * D, x), *px = x.data_ptr(), *s = stream_of(x);
        uint8_t* pc = codes_or_null(a[6], T * D);
        float* ps = scales_or_null(a[7], T * scale_blocks(D));
        const int t = dim(T), d = dim(D);
        const int64_t pitch = row_pitch(x);
        const float eps = real(a[2]);
        return unlocked([&] { return p_rms_norm(px, pr, pw, pro, py, pc, ps, t, d, pitch, eps, io, s); });
    });
}

// (x [T, D], codes, scales)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 3 && a[1] != Py_None && a[2] != Py_None);
        const at::Tensor& x = dense_rows(a[0]);
        require(x.dim() == 2);
        const int64_t T = x.size(0), D = x.size(1);
        const mla_dtype io = io_type(x);
        void *px = x.data_ptr(), *s = stream_of(x);
        uint8_t* pc = codes_or_null(a[1], T * D);
        float* ps = scales_or_null(a[2], T * scale_blocks(D));
        const int t = dim(T), d = dim(D);
        const int64_t pitch = row_pitch(x);
        return unlocked([&] { return p_quantize(px, pc, ps, t, d, pitch, io, s); });
    });
}

// (a [M, K], a_scales, w [N, K], w_scales, out, workspace | None, flags)
PyObject* gemm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 7);
        const at::Tensor &x = tensor(a[0]), &xs = tensor(a[1]), &w = tensor(a[2]), &ws = tensor(a[3]), &out = tensor(a[4]);
        require(x.dim() == 2 && w.dim() == 2 && is_codes(x) && is_codes(w) && x.size(1) == w.size(1));
        const int M = dim(x.size(0)), N = dim(w.size(0)), K = dim(x.size(1));
        require(xs.scalar_type() == at::kFloat && xs.dim() == 2 && xs.size(0) == scale_blocks(K) && xs.size(1) == M);
        require(ws.scalar_type() == at::kFloat && ws.dim() == 2 && ws.size(0) == scale_blocks(N) && ws.size(1) == scale_blocks(K));
        const mla_dtype io = io_type(out);
        require(out.numel() >= (int64_t)M * N);
        void *px = x.data_ptr(), *pxs = xs.data_ptr(), *pw = w.data_ptr(), *pws = ws.data_ptr(), *po = out.data_ptr(), *pk = nullptr, *s = stream_of(x);
        size_t bytes = 0;
        const int flags = (int)integer(a[6]);
        if (a[5] != Py_None) {
            const at::Tensor& k = tensor(a[5]);
            pk = k.data_ptr();
            bytes = k.nbytes();
        }
        return unlocked([&] {
            return p_gemm_fp8(static_cast<uint8_t*>(px), static_cast<float*>(pxs), static_cast<uint8_t*>(pw), static_cast<float*>(pws), po, pk, bytes, M,
                              N, K, io, (unsigned)flags, s);
        });
    });
}

// (q [T, H, d_nope + d_rope], positions, freq, gain, layout, q_nope | None, q_rope)
PyObject* rope_queries(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 7);
        const at::Tensor &q = dense_rows(a[0]), &pos = tensor(a[1]), &freq = tensor(a[2]);
        require(q.dim() == 3 && pos.scalar_type() == at::kInt && freq.scalar_type() == at::kDouble && freq.dim() == 1);
        const int64_t T = q.size(0), H = q.size(1), width = q.size(2), d_rope = 2 * freq.size(0), d_nope = width - d_rope;
        require(d_nope >= 0 && (H == 1 || q.stride(1) == width) && pos.dim() == 1 && pos.size(0) == T);
        const mla_dtype io = io_type(q);
        void *pn = values_or_null(a[5], T * H * d_nope, q), *pr = values_or_null(a[6], T * H * d_rope, q);
        require(pr && (pn || d_nope == 0));
        void *pq = q.data_ptr(), *s = stream_of(q);
        const auto* pp = static_cast<const int32_t*>(pos.data_ptr());
        const auto* pf = static_cast<const double*>(freq.data_ptr());
        const int t = dim(T), h = dim(H), dn = dim(d_nope), dr = dim(d_rope), layout = (int)integer(a[4]);
        const int64_t pitch = T > 1 ? q.stride(0) : H * width;
        const float gain = real(a[3]);
        return unlocked([&] { return p_rope(pq, pp, pf, pn, pr, t, h, dn, dr, pitch, gain, layout, io, s); });
    });
}

// (rows [B, new, d_c + d_rope], positions, freq, kv_cache, page_table, d_c, gain, layout, norm_weight | None, eps, kv_scale | None)
PyObject* cache_store(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 11);
        const at::Tensor &x = dense_rows(a[0]), &pos = tensor(a[1]), &freq = tensor(a[2]), &kv = tensor(a[3]), &table = tensor(a[4]);
        require(x.dim() == 3 && kv.dim() == 3 && table.dim() == 2 && x.size(2) == kv.size(2));
        const int64_t B = x.size(0), T = x.size(1), row = x.size(2), d_c = integer(a[5]), d_rope = row - d_c;
        require(d_c > 0 && d_rope >= 0 && pos.scalar_type() == at::kInt && pos.dim() == 2 && pos.size(0) == B && pos.size(1) == T);
        require(freq.scalar_type() == at::kDouble && freq.dim() == 1 && 2 * freq.size(0) == d_rope && table.scalar_type() == at::kInt && table.size(0) == B);
        const int64_t pitch = T > 1 ? x.stride(1) : B > 1 ? x.stride(0) : row;
        require(B == 1 || T == 1 || x.stride(0) == T * pitch);
        const mla_dtype io = io_type(x), cache = cache_type(kv);
        const void* pw = nullptr;
        if (a[8] != Py_None) {
            const at::Tensor& w = tensor(a[8]);
            require(w.dim() == 1 && w.size(0) == d_c && w.scalar_type() == x.scalar_type());
            pw = w.data_ptr();
        }
        float* ps = nullptr;
        if (a[10] != Py_None) {
            const at::Tensor& s = tensor(a[10]);
            require(s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == kv.size(0) && s.size(1) == kv.size(1));
            ps = static_cast<float*>(s.data_ptr());
        }
        void *px = x.data_ptr(), *pkv = kv.data_ptr(), *s = stream_of(x);
        const auto* pp = static_cast<const int32_t*>(pos.data_ptr());
        const auto* pf = static_cast<const double*>(freq.data_ptr());
        const auto* pt = static_cast<const int32_t*>(table.data_ptr());
        const int b = dim(B), t = dim(T), dc = dim(d_c), dr = dim(d_rope), page = dim(kv.size(1)), pages = dim(kv.size(0)), mp = dim(table.size(1)),
                  layout = (int)integer(a[7]);
        const float gain = real(a[6]), eps = real(a[9]);
        return unlocked([&] { return p_store(px, pp, pf, pw, pkv, ps, pt, b, t, dc, dr, pitch, page, pages, mp, gain, layout, eps, io, cache, s); });
    });
}

// the tensors of a masked call lie together, on the current device (elsewhere the binding makes theirs the current one)
void together(const at::Tensor& first, PyObject* const* others, int n)
{
    require(first.device().index() == c10::hip::current_device());
    for (int i = 0; i < n; ++i)
        if (others[i] != Py_None) require(THPVariable_CheckExact(others[i]) && THPVariable_Unpack(others[i]).device() == first.device());
}

// (q_abs [B, T, H, d_c], q_rope | None, kv_cache, page_table, lens, kv_scale | None, workspace, out, lse | None, tree_mask | None, window, sinks,
//  scale, flags)
PyObject* decode_masked(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 14);
        const at::Tensor &q = tensor(a[0]), &kv = tensor(a[2]), &table = tensor(a[3]), &lens = tensor(a[4]), &ws = tensor(a[6]);
        together(q, a + 1, 9);
        require(q.dim() == 4 && kv.dim() == 3 && table.dim() == 2 && lens.dim() == 1);
        const int64_t B = q.size(0), T = q.size(1), H = q.size(2), d_c = q.size(3), pages = kv.size(0), page = kv.size(1), d_rope = kv.size(2) - d_c;
        require(d_rope >= 0);
        void* pr = nullptr;
        if (d_rope) {
            const at::Tensor& r = tensor(a[1]);
            require(r.dim() == 4 && r.size(0) == B && r.size(1) == T && r.size(2) == H && r.size(3) == d_rope && r.scalar_type() == q.scalar_type());
            pr = r.data_ptr();
        } else {
            require(a[1] == Py_None);
        }
        require(table.scalar_type() == at::kInt && lens.scalar_type() == at::kInt && table.size(0) == B && lens.size(0) == B);
        const float* ps = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor& s = tensor(a[5]);
            require(s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == pages && s.size(1) == page);
            ps = static_cast<const float*>(s.data_ptr());
        }
        const mla_dtype io = io_type(q), cache = cache_type(kv);
        const at::Tensor& out = tensor(a[7]);
        require(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        float* pl = nullptr;
        if (a[8] != Py_None) {
            const at::Tensor& l = tensor(a[8]);
            require(l.scalar_type() == at::kFloat && l.dim() == 3 && l.size(0) == B && l.size(1) == T && l.size(2) == H);
            pl = static_cast<float*>(l.data_ptr());
        }
        void *pq = q.data_ptr(), *pkv = kv.data_ptr(), *pws = ws.data_ptr(), *po = out.data_ptr(), *s = stream_of(q);
        const auto* pt = static_cast<const int32_t*>(table.data_ptr());
        const auto* pn = static_cast<const int32_t*>(lens.data_ptr());
        const size_t bytes = ws.nbytes();
        const int b = dim(B), t = dim(T), h = dim(H), dc = dim(d_c), dr = dim(d_rope), pg = dim(page), np = dim(pages), mp = dim(table.size(1)),
                  window = (int)integer(a[10]), sinks = (int)integer(a[11]), flags = (int)integer(a[13]);
        const float scale = real(a[12]);
        if (a[9] == Py_None)
            return unlocked([&] {
                return p_window(pq, pr, pkv, ps, pt, pn, po, pl, pws, bytes, b, t, h, dc, dr, pg, np, mp, window, sinks, scale, io, cache, (unsigned)flags, s);
            });
        const at::Tensor& m = tensor(a[9]);
        require(m.scalar_type() == at::kLong && ((m.dim() == 2 && m.size(0) == B && m.size(1) == T) || (m.dim() == 1 && m.size(0) == T)));
        const auto* pm = static_cast<const uint64_t*>(m.data_ptr());
        const int64_t pitch = m.dim() == 2 ? T : 0;
        return unlocked([&] {
            return p_tree(pq, pr, pkv, ps, pt, pn, pm, pitch, po, pl, pws, bytes, b, t, h, dc, dr, pg, np, mp, scale, io, cache, (unsigned)flags, s);
        });
    });
}

// (kv_cache, kv_scale | None, page_table, src, dst)
PyObject* cache_move(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        require(n == 5);
        const at::Tensor &kv = tensor(a[0]), &table = tensor(a[2]), &src = tensor(a[3]), &dst = tensor(a[4]);
        together(kv, a + 1, 4);
        require(kv.dim() == 3 && table.dim() == 2 && src.dim() == 2 && dst.sizes() == src.sizes() && table.size(0) == src.size(0));
        require(table.scalar_type() == at::kInt && src.scalar_type() == at::kInt && dst.scalar_type() == at::kInt);
        float* ps = nullptr;
        require((a[1] != Py_None) == (cache_type(kv) == MLA_FP8_E4M3));
        if (a[1] != Py_None) {
            const at::Tensor& s = tensor(a[1]);
            require(s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == kv.size(0) && s.size(1) == kv.size(1));
            ps = static_cast<float*>(s.data_ptr());
        }
        void *pkv = kv.data_ptr(), *s = stream_of(kv);
        const auto* pt = static_cast<const int32_t*>(table.data_ptr());
        const auto* p0 = static_cast<const int32_t*>(src.data_ptr());
        const auto* p1 = static_cast<const int32_t*>(dst.data_ptr());
        const int b = dim(src.size(0)), m = dim(src.size(1)), row = dim(kv.size(2) * kv.element_size()), page = dim(kv.size(1)), pages = dim(kv.size(0)),
                  mp = dim(table.size(1));
        return unlocked([&] { return p_move(pkv, ps, pt, p0, p1, b, m, row, page, pages, mp, s); });
    });
}

// (addresses of the fourteen entry points, in the order above)
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long p[14];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKKK", p, p + 1, p + 2, p + 3, p + 4, p + 5, p + 6, p + 7, p + 8, p + 9, p + 10, p + 11, p + 12, p + 13)) return nullptr;
    p_absorb_q = reinterpret_cast<decltype(p_absorb_q)>(p[0]);
    p_out_proj = reinterpret_cast<decltype(p_out_proj)>(p[1]);
    p_decode = reinterpret_cast<decltype(p_decode)>(p[2]);
    p_merge_out_proj = reinterpret_cast<decltype(p_merge_out_proj)>(p[3]);
    p_merge_partials = reinterpret_cast<decltype(p_merge_partials)>(p[4]);
    p_append = reinterpret_cast<decltype(p_append)>(p[5]);
    p_rms_norm = reinterpret_cast<decltype(p_rms_norm)>(p[6]);
    p_quantize = reinterpret_cast<decltype(p_quantize)>(p[7]);
    p_gemm_fp8 = reinterpret_cast<decltype(p_gemm_fp8)>(p[8]);
    p_rope = reinterpret_cast<decltype(p_rope)>(p[9]);
    p_store = reinterpret_cast<decltype(p_store)>(p[10]);
    p_tree = reinterpret_cast<decltype(p_tree)>(p[11]);
    p_window = reinterpret_cast<decltype(p_window)>(p[12]);
    p_move = reinterpret_cast<decltype(p_move)>(p[13]);
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(absorb_q), FAST(out_proj), FAST(decode), FAST(merge_out_proj), FAST(merge_partials), FAST(cache_append),
                         FAST(rms_norm), FAST(quantize_rows), FAST(gemm_fp8), FAST(rope_queries), FAST(cache_store),
                         FAST(decode_masked), FAST(cache_move),
                         {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module_def); }
