// Argument marshalling of the Python binding in native code: turns tensors (anything with data_ptr(), stride(), shape and
// dtype), (address, leading dimension[, dtype]) sequences and None into the structures of the C ABI (include/tp_linear.h) and makes
// the call.  Nothing is computed, kept or checked here beyond that; the library answers for the arguments.
//
// Why: the smallest calls are shorter on the GPU than they were on the host.  A forward of 256 x 1024 x 4096 on a 2 x 2 grid spent
// 6.7 us in Python and ctypes before a call that takes 5.4 with its launch.
//
// The functions come from the loaded library by address (bind()), so this module links against nothing.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <new>
#include <vector>

#include "tp_linear.h"

namespace {

PyObject *s_data_ptr, *s_stride, *s_shape, *s_dtype, *s_numel, *s_element_size;      // interned names
PyObject *s_get_device, *s_is_contiguous;
PyObject* g_tensor;                                                                  // torch.Tensor, or None
PyObject *g_i32, *g_i64, *g_u64, *g_f32, *g_bf16;                                    // torch.int32, torch.int64, torch.uint64, torch.float32, torch.bfloat16
int (*g_current_device)(int*);                                                       // hipGetDevice, or null: its answer is not compared

decltype(&tp_block_map) f_block_map;
decltype(&tp_linear_fwd_ex) f_fwd;
decltype(&tp_linear_fwd_static) f_static;
decltype(&tp_linear_bwd_ex) f_bwd;
decltype(&tp_linear_bwd_partials_ex) f_partials;
decltype(&tp_bias_act) f_bias_act;
decltype(&tp_dgelu) f_dgelu;
decltype(&tp_bias_grad) f_bias_grad;
decltype(&tp_dropout_fwd) f_dropout_fwd;
decltype(&tp_dropout_bwd) f_dropout_bwd;
decltype(&tp_adapter_fwd) f_adapter_fwd;
decltype(&tp_adapter_bwd) f_adapter_bwd;

// Every helper returns false with a Python exception set.
struct Ref {                                       // an owned reference
    PyObject* p;
    explicit Ref(PyObject* q) : p(q) {}
    ~Ref() { Py_XDECREF(p); }
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
    explicit operator bool() const { return p != nullptr; }
};

bool to_i64(PyObject* o, int64_t* out) {           // int(o)
    if (PyLong_CheckExact(o)) {
        *out = (int64_t)PyLong_AsUnsignedLongLongMask(o);
        return !(*out == -1 && PyErr_Occurred());
    }
    Ref l(PyNumber_Long(o));
    if (!l) return false;
    *out = (int64_t)PyLong_AsUnsignedLongLongMask(l.p);
    return !(*out == -1 && PyErr_Occurred());
}
bool to_int(PyObject* o, int* out) {
    int64_t v;
    if (!to_i64(o, &v)) return false;
    *out = (int)v;
    return true;
}
bool call0(PyObject* o, PyObject* name, int64_t* out) {
    Ref r(PyObject_CallMethodNoArgs(o, name));
    return r && to_i64(r.p, out);
}
bool is_sequence(PyObject* o) { return PyTuple_Check(o) || PyList_Check(o); }
// a tensor has data_ptr; what has none is taken as a sequence.  (torch's own types are known without asking.)
bool is_tensor(PyObject* o, bool* yes) {
    if (is_sequence(o)) { *yes = false; return true; }
    if (g_tensor && (PyObject*)Py_TYPE(o) == g_tensor) { *yes = true; return true; }
    Ref a(PyObject_GetAttr(o, s_data_ptr));
    if (!a && !PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
    *yes = (bool)a;
    if (!a) PyErr_Clear();
    return true;
}
bool item(PyObject* o, Py_ssize_t i, int64_t* out) {
    if (PyTuple_CheckExact(o) && i < PyTuple_GET_SIZE(o)) return to_i64(PyTuple_GET_ITEM(o, i), out);
    Ref v(PySequence_GetItem(o, i));
    return v && to_i64(v.p, out);
}
// leading dimension: row stride of a 2-D tensor with unit column stride; a 1-D tensor is one row
bool tensor_ld(PyObject* t, int64_t* ld) {
    Ref st(PyObject_CallMethodNoArgs(t, s_stride));
    if (!st) return false;
    const Py_ssize_t n = PySequence_Size(st.p);
    if (n < 0) return false;
    if (n == 2) {
        int64_t cs;
        if (!item(st.p, 1, &cs)) return false;
        bool ok = cs == 1;
        if (!ok) {
            Ref sh(PyObject_GetAttr(t, s_shape));
            int64_t cols;
            if (!sh || !item(sh.p, 1, &cols)) return false;
            ok = cols <= 1;
        }
        if (ok) return item(st.p, 0, ld);
    } else if (n == 1) {
        Ref sh(PyObject_GetAttr(t, s_shape));
        return sh && item(sh.p, 0, ld);
    }
    PyErr_SetString(PyExc_ValueError, "blocks must be 2-D with unit column stride");
    return false;
}
bool to_cblk(PyObject* o, tp_cblk_t* b) {
    int64_t ptr = 0, ld = 0;
    if (o != Py_None) {
        bool tensor;
        if (!is_tensor(o, &tensor)) return false;
        if (tensor ? !(call0(o, s_data_ptr, &ptr) && tensor_ld(o, &ld)) : !(item(o, 0, &ptr) && item(o, 1, &ld))) return false;
    }
    b->ptr = reinterpret_cast<const void*>(ptr);
    b->ld = ld;
    return true;
}
bool to_oblk(PyObject* o, tp_oblk_t* b) {
    int64_t ptr = 0, ld = 0;
    int dtype = 0;
    if (o != Py_None) {
        bool tensor;
        if (!is_tensor(o, &tensor)) return false;
        if (tensor) {
            if (!call0(o, s_data_ptr, &ptr) || !tensor_ld(o, &ld)) return false;
            Ref dt(PyObject_GetAttr(o, s_dtype));
            if (!dt) return false;
            dtype = dt.p == g_f32 ? TP_F32 : dt.p == g_bf16 ? TP_BF16 : 99;       // 99: the library answers TP_ERR_DTYPE
        } else {
            int64_t d;
            if (!item(o, 0, &ptr) || !item(o, 1, &ld) || !item(o, 2, &d)) return false;
            dtype = (int)d;
        }
    }
    b->ptr = reinterpret_cast<void*>(ptr);
    b->ld = ld;
    b->dtype = dtype;
    return true;
}
bool to_ptr(PyObject* o, void** out) {             // None, a tensor or an address
    int64_t v = 0;
    if (o != Py_None) {
        if (PyLong_Check(o)) {
            if (!to_i64(o, &v)) return false;
        } else {
            bool tensor;
            if (!is_tensor(o, &tensor)) return false;
            if (tensor ? !call0(o, s_data_ptr, &v) : !to_i64(o, &v)) return false;
        }
    }
    *out = reinterpret_cast<void*>(v);
    return true;
}
struct Workspace { void* ptr; size_t bytes; };     // None, a tensor or (address, bytes)
bool to_ws(PyObject* o, Workspace* w) {
    int64_t ptr = 0, n = 0, each = 1;
    if (o != Py_None) {
        bool tensor;
        if (!is_tensor(o, &tensor)) return false;
        if (tensor ? !(call0(o, s_data_ptr, &ptr) && call0(o, s_numel, &n) && call0(o, s_element_size, &each)) : !(item(o, 0, &ptr) && item(o, 1, &n)))
            return false;
    }
    w->ptr = reinterpret_cast<void*>(ptr);
    w->bytes = (size_t)(n * each);
    return true;
}
bool to_dims(PyObject* o, tp_dims_t* d) {
    Ref s(PySequence_Fast(o, "dims must be (M, H, F)"));
    if (!s) return false;
    if (PySequence_Fast_GET_SIZE(s.p) != 3) {
        PyErr_SetString(PyExc_ValueError, "dims must be (M, H, F)");
        return false;
    }
    PyObject** it = PySequence_Fast_ITEMS(s.p);
    return to_i64(it[0], &d->M) && to_i64(it[1], &d->H) && to_i64(it[2], &d->F);
}
// A list of blocks, with empty ones up to TP_MAX_STEPS (the library reads no more); None: a null pointer.
template <class B, bool (*CONVERT)(PyObject*, B*)> struct Blocks {
    B fixed[TP_MAX_STEPS] = {};
    std::vector<B> more;
    const B* ptr = nullptr;
    bool fill(PyObject* o) {
        if (o == Py_None) return true;
        if (PyObject_Size(o) < 0) return false;    // (an iterator's blocks may be gone before the call)
        Ref s(PySequence_Fast(o, "blocks must be a sequence"));
        if (!s) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(s.p);
        B* to = fixed;
        if (n > TP_MAX_STEPS) {
            try { more.resize((size_t)n); } catch (const std::bad_alloc&) { PyErr_NoMemory(); return false; }
            to = more.data();
        }
        for (Py_ssize_t i = 0; i < n; ++i)
            if (!CONVERT(PySequence_Fast_GET_ITEM(s.p, i), to + i)) return false;
        ptr = to;
        return true;
    }
};
using CBlocks = Blocks<tp_cblk_t, to_cblk>;
using OBlocks = Blocks<tp_oblk_t, to_oblk>;
struct MaybeBlock {                                // None: a null pointer
    tp_cblk_t b;
    const tp_cblk_t* ptr = nullptr;
    bool fill(PyObject* o) {
        if (o == Py_None) return true;
        if (!to_cblk(o, &b)) return false;
        ptr = &b;
        return true;
    }
};
template <class T> bool to_struct(PyObject* o, const T** out) {      // the address of a structure, 0 or None: none
    void* p;
    if (!to_ptr(o, &p)) return false;
    *out = static_cast<const T*>(p);
    return true;
}
bool count(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, have);
    return false;
}
// The call itself runs without the interpreter lock: a launch waits when the stream's queue is full.
template <class F> PyObject* answer(F&& call) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// fwd(grid, dims, n_steps, x_blocks, w_blocks, bias, epi, y, preact, workspace, stream, opts)
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid; const tp_plan_opts_t* opts;
    tp_dims_t dims; int steps, epi; CBlocks x, w; void *bias, *stream; tp_oblk_t y, pre; Workspace ws;
    if (!count(n, 12) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &steps) || !x.fill(a[3]) || !w.fill(a[4]) ||
        !to_ptr(a[5], &bias) || !to_int(a[6], &epi) || !to_oblk(a[7], &y) || !to_oblk(a[8], &pre) || !to_ws(a[9], &ws) ||
        !to_ptr(a[10], &stream) || !to_struct(a[11], &opts))
        return nullptr;
    return answer([&] { return f_fwd(grid, &dims, steps, x.ptr, w.ptr, bias, epi, y, pre, ws.ptr, ws.bytes, stream, opts); });
}
// fwd_static(grid, dims, n_steps, x_blocks, w_blocks, bias, epi, y, preact, stream)
PyObject* fwd_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid;
    tp_dims_t dims; int steps, epi; CBlocks x, w; void *bias, *stream; tp_oblk_t y, pre;
    if (!count(n, 10) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &steps) || !x.fill(a[3]) || !w.fill(a[4]) ||
        !to_ptr(a[5], &bias) || !to_int(a[6], &epi) || !to_oblk(a[7], &y) || !to_oblk(a[8], &pre) || !to_ptr(a[9], &stream))
        return nullptr;
    return answer([&] { return f_static(grid, &dims, steps, x.ptr, w.ptr, bias, epi, y, pre, stream); });
}
// bwd(grid, dims, n_dx, n_dw, dy_own, preact_own, da_row_blocks, w_blocks_dx, x_blocks_dw, da_col_blocks, own_slot_dx, own_slot_dw,
//     dgelu_preact, dx, dw, da_own_out, db, workspace, stream, opts)
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid; const tp_plan_opts_t* opts;
    tp_dims_t dims; int ndx, ndw, sdx, sdw; MaybeBlock dy, pre, dg; CBlocks rows, w, x, cols; tp_oblk_t dx, dw, da; void *db, *stream; Workspace ws;
    if (!count(n, 20) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &ndx) || !to_int(a[3], &ndw) || !dy.fill(a[4]) ||
        !pre.fill(a[5]) || !rows.fill(a[6]) || !w.fill(a[7]) || !x.fill(a[8]) || !cols.fill(a[9]) || !to_int(a[10], &sdx) ||
        !to_int(a[11], &sdw) || !dg.fill(a[12]) || !to_oblk(a[13], &dx) || !to_oblk(a[14], &dw) || !to_oblk(a[15], &da) || !to_ptr(a[16], &db) ||
        !to_ws(a[17], &ws) || !to_ptr(a[18], &stream) || !to_struct(a[19], &opts))
        return nullptr;
    return answer([&] {
        return f_bwd(grid, &dims, ndx, ndw, dy.ptr, pre.ptr, rows.ptr, w.ptr, x.ptr, cols.ptr, sdx, sdw, dg.ptr, dx, dw, da, db, ws.ptr, ws.bytes,
                     stream, opts);
    });
}
// bwd_partials(grid, dims, n_dx, n_dw, da_own, w_blocks_dx, dx_partials, x_blocks_dw, dw_partials, workspace, stream, opts)
PyObject* bwd_partials(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid; const tp_plan_opts_t* opts;
    tp_dims_t dims; int ndx, ndw; MaybeBlock da; CBlocks w, x; OBlocks dx, dw; void* stream; Workspace ws;
    if (!count(n, 12) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &ndx) || !to_int(a[3], &ndw) || !da.fill(a[4]) ||
        !w.fill(a[5]) || !dx.fill(a[6]) || !x.fill(a[7]) || !dw.fill(a[8]) || !to_ws(a[9], &ws) || !to_ptr(a[10], &stream) ||
        !to_struct(a[11], &opts))
        return nullptr;
    return answer([&] { return f_partials(grid, &dims, ndx, ndw, da.ptr, w.ptr, dx.ptr, x.ptr, dw.ptr, ws.ptr, ws.bytes, stream, opts); });
}
// bias_act(c, bias, epi, y, preact, rows, cols, stream)
PyObject* bias_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    tp_cblk_t c; tp_oblk_t y, pre; void *bias, *stream; int epi; int64_t rows, cols;
    if (!count(n, 8) || !to_cblk(a[0], &c) || !to_ptr(a[1], &bias) || !to_int(a[2], &epi) || !to_oblk(a[3], &y) || !to_oblk(a[4], &pre) ||
        !to_i64(a[5], &rows) || !to_i64(a[6], &cols) || !to_ptr(a[7], &stream))
        return nullptr;
    return answer([&] { return f_bias_act(c.ptr, c.ld, bias, epi, y, pre, rows, cols, stream); });
}
// dgelu(dy, preact, da, rows, cols, stream)
PyObject* dgelu(PyObject*, PyObject* const* a, Py_ssize_t n) {
    tp_cblk_t dy, pre, da; void* stream; int64_t rows, cols;
    if (!count(n, 6) || !to_cblk(a[0], &dy) || !to_cblk(a[1], &pre) || !to_cblk(a[2], &da) || !to_i64(a[3], &rows) || !to_i64(a[4], &cols) ||
        !to_ptr(a[5], &stream))
        return nullptr;
    return answer([&] { return f_dgelu(dy.ptr, dy.ld, pre.ptr, pre.ld, const_cast<void*>(da.ptr), da.ld, rows, cols, stream); });
}
// bias_grad(da, db, rows, cols, workspace, stream)
PyObject* bias_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    tp_cblk_t da; void *db, *stream; int64_t rows, cols; Workspace ws;
    if (!count(n, 6) || !to_cblk(a[0], &da) || !to_ptr(a[1], &db) || !to_i64(a[2], &rows) || !to_i64(a[3], &cols) || !to_ws(a[4], &ws) ||
        !to_ptr(a[5], &stream))
        return nullptr;
    return answer([&] { return f_bias_grad(da.ptr, da.ld, rows, cols, db, ws.ptr, ws.bytes, stream); });
}
// The calls below also look at what the C functions cannot see of a tensor: its type, where only one fits, that it holds all that the call's extents
// say (a kernel goes by those), and that all of a call's tensors are on the current device (a kernel that follows a host address ends the process).
struct Devices {
    int64_t seen = -1;
    bool add(PyObject* t) {
        int64_t d;
        if (!call0(t, s_get_device, &d)) return false;
        if (d < 0) { PyErr_SetString(PyExc_ValueError, "a tensor of the call is not on the GPU"); return false; }
        if (seen >= 0) {
            if (d == seen) return true;
        } else {
            seen = d;
            int now;
            if (!g_current_device || (g_current_device(&now) == 0 && d == now)) return true;
        }
        PyErr_SetString(PyExc_ValueError, "the call's tensors are not all on the current device");
        return false;
    }
};
// None, an address or sequence (taken as it is), or a tensor on the current device, of type `want` if that is given
bool look(PyObject* o, PyObject* want, Devices* at) {
    if (o == Py_None || PyLong_Check(o)) return true;
    bool tensor;
    if (!is_tensor(o, &tensor)) return false;
    if (!tensor) return true;
    if (!at->add(o)) return false;
    if (!want || want == Py_None) return true;
    Ref dt(PyObject_GetAttr(o, s_dtype));
    if (!dt) return false;
    if (dt.p == want) return true;
    PyErr_Format(PyExc_TypeError, "%R expected, got %R", want, dt.p);
    return false;
}

bool numel(PyObject* o, int64_t* n) { return call0(o, s_numel, n); }
// a tensor (others are taken as they are) has at least `want` elements (`have` if that is known), one behind the other
bool flat(PyObject* t, int64_t want, const char* what, int64_t have = -1) {
    bool tensor;
    if (t == Py_None || PyLong_Check(t)) return true;
    if (!is_tensor(t, &tensor)) return false;
    if (!tensor) return true;
    if (have < 0 && !numel(t, &have)) return false;
    Ref c(PyObject_CallMethodNoArgs(t, s_is_contiguous));
    if (!c) return false;
    if (have >= want && c.p == Py_True) return true;
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous tensor of at least %lld elements", what, (long long)want);
    return false;
}
// a bias or its gradient
bool to_flat(PyObject* o, PyObject* type, Devices* at, int64_t want, const char* what, void** p) { return look(o, type, at) && flat(o, want, what) && to_ptr(o, p); }

// What a tensor has to hold; nothing with no rows or columns (of what the call does not use, or the library refuses)
struct Extents { int64_t rows = 0, cols = 0; const char* what = ""; };
bool holds(const Extents& e, int64_t rows, int64_t cols) {
    if (e.rows <= 0 || e.cols <= 0 || (rows >= e.rows && cols >= e.cols)) return true;
    PyErr_Format(PyExc_ValueError, "%s must have at least %lld rows of %lld columns, got %lld of %lld", e.what, (long long)e.rows, (long long)e.cols,
                 (long long)rows, (long long)cols);
    return false;
}
// element i of a tensor's shape or strides (tuples, of a type of their own)
bool extent(PyObject* o, Py_ssize_t i, int64_t* out) { return PyTuple_Check(o) && i < PyTuple_GET_SIZE(o) ? to_i64(PyTuple_GET_ITEM(o, i), out) : item(o, i, out); }
// the leading dimension of a tensor as tensor_ld() takes it, with these extents
bool tensor_ld(PyObject* t, const Extents& e, int64_t* ld) {
    Ref st(PyObject_CallMethodNoArgs(t, s_stride)), sh(PyObject_GetAttr(t, s_shape));
    if (!st || !sh) return false;
    const Py_ssize_t n = PySequence_Size(st.p);
    if (n < 0) return false;
    int64_t rows = 1, cols, unit;
    if (n == 2) {
        if (!extent(sh.p, 0, &rows) || !extent(sh.p, 1, &cols) || !extent(st.p, 0, ld) || !extent(st.p, 1, &unit)) return false;
        if (unit == 1 || cols <= 1) return holds(e, rows, cols);
    } else if (n == 1) {
        if (!extent(sh.p, 0, &cols) || !extent(st.p, 0, &unit)) return false;
        *ld = cols;
        if (unit == 1 || cols <= 1) return holds(e, rows, cols);
    }
    PyErr_SetString(PyExc_ValueError, "blocks must be 2-D with unit column stride");
    return false;
}
// A block: None, a sequence as to_oblk() and to_cblk() take it, or a tensor on the current device of type `want` (null: fp32 or bf16, else 99)
bool to_block(PyObject* o, PyObject* want, Devices* at, const Extents& e, tp_oblk_t* b) {
    bool tensor = false;
    if (o == Py_None) return to_oblk(o, b);
    if (!is_tensor(o, &tensor)) return false;
    if (!tensor) {
        if (!want) return to_oblk(o, b);
        tp_cblk_t c;
        if (!to_cblk(o, &c)) return false;
        *b = tp_oblk_t{const_cast<void*>(c.ptr), c.ld, 0};
        return true;
    }
    int64_t ptr = 0, ld = 0;
    if (!at->add(o) || !call0(o, s_data_ptr, &ptr) || !tensor_ld(o, e, &ld)) return false;
    Ref dt(PyObject_GetAttr(o, s_dtype));
    if (!dt) return false;
    if (want && want != Py_None && dt.p != want) {
        PyErr_Format(PyExc_TypeError, "%R expected, got %R", want, dt.p);
        return false;
    }
    *b = tp_oblk_t{reinterpret_cast<void*>(ptr), ld, dt.p == g_f32 ? TP_F32 : dt.p == g_bf16 ? TP_BF16 : 99};
    return true;
}
bool to_input(PyObject* o, Devices* at, const Extents& e, tp_cblk_t* b) {           // bf16
    tp_oblk_t q;
    if (!to_block(o, g_bf16, at, e, &q)) return false;
    *b = tp_cblk_t{q.ptr, q.ld};
    return true;
}
struct Inputs {                                                  // a list of them, with empty ones up to TP_MAX_STEPS; None: a null pointer
    tp_cblk_t blocks[TP_MAX_STEPS] = {};
    const tp_cblk_t* ptr = nullptr;
    bool fill(PyObject* o, Devices* at, const Extents& e, int used) {      // (the first `used` are read)
        if (o == Py_None) return true;
        if (PyObject_Size(o) < 0) return false;
        Ref s(PySequence_Fast(o, "blocks must be a sequence"));
        if (!s) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(s.p);
        if (n > TP_MAX_STEPS) { PyErr_SetString(PyExc_ValueError, "too many blocks"); return false; }
        for (Py_ssize_t i = 0; i < n; ++i)
            if (!to_input(PySequence_Fast_GET_ITEM(s.p, i), at, i < used ? e : Extents{}, blocks + i)) return false;
        ptr = blocks;
        return true;
    }
};
struct MaybeInput {
    tp_cblk_t b;
    const tp_cblk_t* ptr = nullptr;
    bool fill(PyObject* o, Devices* at, const Extents& e) {
        if (o == Py_None) return true;
        if (!to_input(o, at, e, &b)) return false;
        ptr = &b;
        return true;
    }
};

// A mask: a sequence (p, seed, offset, offset_dev, row0, col0)
bool to_dropout(PyObject* o, tp_dropout_t* d, Devices* at) {
    Ref s(PySequence_Fast(o, "dropout must be a Dropout"));
    if (!s) return false;
    if (PySequence_Fast_GET_SIZE(s.p) != 6) {
        PyErr_SetString(PyExc_ValueError, "dropout must be a Dropout: (p, seed, offset, offset_dev, row0, col0)");
        return false;
    }
    PyObject** it = PySequence_Fast_ITEMS(s.p);
    d->p = PyFloat_AsDouble(it[0]);
    if (d->p == -1.0 && PyErr_Occurred()) return false;
    int64_t seed, offset;
    void* dev;
    if (!to_i64(it[1], &seed) || !to_i64(it[2], &offset) || !look(it[3], nullptr, at) || !flat(it[3], 1, "offset_dev") || !to_ptr(it[3], &dev) ||
        !to_i64(it[4], &d->row0) || !to_i64(it[5], &d->col0))
        return false;
    if (it[3] != Py_None && !PyLong_Check(it[3])) {
        bool tensor;
        if (!is_tensor(it[3], &tensor)) return false;
        Ref dt(tensor ? PyObject_GetAttr(it[3], s_dtype) : nullptr);
        if (tensor && !dt) return false;
        if (tensor && dt.p != g_i64 && dt.p != g_u64) { PyErr_SetString(PyExc_TypeError, "offset_dev must be a 64-bit integer"); return false; }
    }
    d->seed = (uint64_t)seed;
    d->offset = (uint64_t)offset;
    d->offset_dev = static_cast<const uint64_t*>(dev);
    return true;
}
// dropout_fwd(dropout, x, bias, epi, residual, y, preact, rows, cols, stream)
PyObject* dropout_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    tp_dropout_t d; tp_oblk_t x, y, pre; tp_cblk_t res; void *bias, *stream; int epi; int64_t rows, cols; Devices at;
    if (!count(n, 10) || !to_i64(a[7], &rows) || !to_i64(a[8], &cols) || !to_dropout(a[0], &d, &at) || !to_block(a[1], nullptr, &at, {rows, cols, "x"}, &x) ||
        !to_flat(a[2], g_bf16, &at, cols, "bias", &bias) || !to_int(a[3], &epi) || !to_input(a[4], &at, {rows, cols, "residual"}, &res) ||
        !to_block(a[5], nullptr, &at, {rows, cols, "y"}, &y) || !to_block(a[6], nullptr, &at, {rows, cols, "preact"}, &pre) || !to_ptr(a[9], &stream))
        return nullptr;
    return answer([&] { return f_dropout_fwd(&d, x.ptr, x.ld, x.dtype, bias, epi, res, y, pre, rows, cols, stream); });
}
// dropout_bwd(dropout, dy, preact, dx, db, rows, cols, workspace, stream)
PyObject* dropout_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    tp_dropout_t d; tp_cblk_t dy, pre, dx; void *db, *stream; int64_t rows, cols; Workspace ws; Devices at;
    if (!count(n, 9) || !to_i64(a[5], &rows) || !to_i64(a[6], &cols) || !to_flat(a[4], g_f32, &at, cols, "db", &db) || !look(a[7], nullptr, &at) ||
        !to_dropout(a[0], &d, &at) || !to_input(a[1], &at, {rows, cols, "dy"}, &dy) || !to_input(a[2], &at, {rows, cols, "preact"}, &pre) ||
        !to_input(a[3], &at, {rows, cols, "dx"}, &dx) || !to_ws(a[7], &ws) || !to_ptr(a[8], &stream))
        return nullptr;
    return answer([&] {
        return f_dropout_bwd(&d, dy.ptr, dy.ld, pre.ptr, pre.ld, const_cast<void*>(dx.ptr), dx.ld, db, rows, cols, ws.ptr, ws.bytes, stream);
    });
}
// A call's adapters: a sequence (offsets, ids, n_adapters, rank, scale, n_segments); n_segments None: as many as ids, a tensor, has
bool to_adapters(PyObject* o, tp_adapters_t* a, Devices* at) {
    Ref s(PySequence_Fast(o, "adapters must be an Adapters"));
    if (!s) return false;
    if (PySequence_Fast_GET_SIZE(s.p) != 6) {
        PyErr_SetString(PyExc_ValueError, "adapters must be an Adapters: (offsets, ids, n_adapters, rank, scale, n_segments)");
        return false;
    }
    PyObject** it = PySequence_Fast_ITEMS(s.p);
    void *offsets, *ids, *scale;
    int pool, rank;
    int64_t n = 0, counted = -1;
    if (!look(it[0], g_i32, at) || !look(it[1], g_i32, at) || !look(it[4], g_f32, at) || !to_ptr(it[0], &offsets) || !to_ptr(it[1], &ids) ||
        !to_int(it[2], &pool) || !to_int(it[3], &rank) || !to_ptr(it[4], &scale) || (it[5] != Py_None && !to_i64(it[5], &n)))
        return false;
    if (it[5] == Py_None && it[1] != Py_None) {
        if (PyLong_Check(it[1])) {
            PyErr_SetString(PyExc_ValueError, "n_segments is needed where ids is an address");
            return false;
        }
        if (!numel(it[1], &n)) return false;
        counted = n;
    }
    if (n < 0 || n > INT32_MAX - 1) n = -1;                              // (the library answers)
    if (!flat(it[0], n > 0 ? n + 1 : 0, "offsets") || !flat(it[1], n > 0 ? n : 0, "ids", counted) || !flat(it[4], pool, "scale")) return false;
    *a = tp_adapters_t{static_cast<const int32_t*>(offsets), static_cast<const int32_t*>(ids), static_cast<const float*>(scale), (int32_t)n, pool, rank};
    return true;
}
// A factor: a tensor [n_adapters, rank, cols] with unit column stride, (address, leading dimension, stride) or None
template <class F> bool to_factor(PyObject* o, F* f, const tp_adapters_t& a, PyObject* type, Devices* at, int64_t cols, const char* what) {
    int64_t ptr = 0, ld = 0, stride = 0;
    if (o != Py_None) {
        bool tensor;
        if (!is_tensor(o, &tensor)) return false;
        if (!tensor) {
            if (!item(o, 0, &ptr) || !item(o, 1, &ld) || !item(o, 2, &stride)) return false;
        } else {
            if (!look(o, type, at) || !call0(o, s_data_ptr, &ptr)) return false;
            Ref st(PyObject_CallMethodNoArgs(o, s_stride)), sh(PyObject_GetAttr(o, s_shape));
            if (!st || !sh) return false;
            int64_t n, r, have, unit;
            if (PySequence_Size(st.p) != 3 || !extent(sh.p, 0, &n) || !extent(sh.p, 1, &r) || !extent(sh.p, 2, &have) ||
                !extent(st.p, 0, &stride) || !extent(st.p, 1, &ld) || !extent(st.p, 2, &unit)) {
                if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a factor must be [n_adapters, rank, cols]");
                return false;
            }
            if (n != a.n_adapters || r != a.rank || unit != 1) {
                PyErr_SetString(PyExc_ValueError, "a factor must be [n_adapters, rank, cols] with unit column stride");
                return false;
            }
            if (have < cols) {
                PyErr_Format(PyExc_ValueError, "%s must have at least %lld columns, got %lld", what, (long long)cols, (long long)have);
                return false;
            }
            if (n == 1) stride = 0;                                      // (never used; torch puts anything there)
        }
    }
    f->ptr = reinterpret_cast<decltype(f->ptr)>(ptr);
    f->ld = ld;
    f->stride = stride;
    return true;
}
struct Factors {
    tp_factor_t at_[TP_MAX_STEPS] = {};
    const tp_factor_t* ptr = nullptr;
    bool fill(PyObject* o, const tp_adapters_t& a, Devices* at, int64_t cols, const char* what, int used) {
        if (o == Py_None) return true;
        if (PyObject_Size(o) < 0) return false;
        Ref s(PySequence_Fast(o, "factors must be a sequence"));
        if (!s) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(s.p);
        if (n > TP_MAX_STEPS) { PyErr_SetString(PyExc_ValueError, "too many factors"); return false; }
        for (Py_ssize_t i = 0; i < n; ++i)
            if (!to_factor(PySequence_Fast_GET_ITEM(s.p, i), at_ + i, a, g_bf16, at, i < used ? cols : 0, what)) return false;
        ptr = at_;
        return true;
    }
};
// V: fp32 [rows, rank], one row behind the other
bool to_v(PyObject* o, float** v, Devices* at, int64_t rows, int rank) {
    void* p;
    if (!to_flat(o, g_f32, at, rank > 0 ? rows * rank : 0, "v", &p)) return false;
    *v = static_cast<float*>(p);
    return true;
}
struct MaybeDropout {
    tp_dropout_t d;
    const tp_dropout_t* ptr = nullptr;
    bool fill(PyObject* o, Devices* at) {
        if (o == Py_None) return true;
        if (!to_dropout(o, &d, at)) return false;
        ptr = &d;
        return true;
    }
};
// Extents of the rank's share in one pass; zeros where the library will refuse it
struct Share { int64_t m = 0, n = 0, k = 0; };
Share share(const tp_grid_t* grid, const tp_dims_t* dims, int pass) {
    Share s;
    if (f_block_map(grid, dims, pass, nullptr, &s.m, &s.n, &s.k, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) != TP_OK ||
        s.m > INT32_MAX || s.n > INT32_MAX || s.k > INT32_MAX)
        return Share{};
    return s;
}
// adapter_fwd(grid, dims, n_steps, adapters, x_blocks, a_blocks, b, dropout, c, bias, epi, y, preact, v, workspace, stream)
PyObject* adapter_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid; tp_dims_t dims; int steps, epi; tp_adapters_t ad; Inputs x; Factors f; tp_factor_t b; MaybeDropout drop; tp_oblk_t c, y, pre;
    void *bias, *stream; float* v; Workspace ws; Devices at;
    if (!count(n, 16) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &steps) || !to_adapters(a[3], &ad, &at)) return nullptr;
    const Share s = share(grid, &dims, TP_PASS_FWD);
    if (!x.fill(a[4], &at, {s.m, s.k, "a block of X"}, steps) || !f.fill(a[5], ad, &at, s.k, "a chunk of A", steps) ||
        !to_factor(a[6], &b, ad, g_bf16, &at, s.n, "b") || !drop.fill(a[7], &at) || !to_block(a[8], nullptr, &at, {s.m, s.n, "c"}, &c) ||
        !to_int(a[10], &epi) || !to_flat(a[9], g_bf16, &at, epi == TP_EPI_NONE ? 0 : s.n, "bias", &bias) ||
        !to_block(a[11], nullptr, &at, {s.m, s.n, "y"}, &y) || !to_block(a[12], nullptr, &at, {s.m, s.n, "preact"}, &pre) || !to_v(a[13], &v, &at, s.m, ad.rank) ||
        !look(a[14], nullptr, &at) || !to_ws(a[14], &ws) || !to_ptr(a[15], &stream))
        return nullptr;
    return answer([&] {
        return f_adapter_fwd(grid, &dims, steps, &ad, x.ptr, f.ptr, a[6] == Py_None ? nullptr : &b, drop.ptr, c, bias, epi, y, pre, v, ws.ptr, ws.bytes, stream);
    });
}
// adapter_bwd(grid, dims, n_steps, adapters, dy_blocks, b_blocks, a, dropout, dx_base, dx, x_own, da, dy_own, v, db, accumulate, workspace, stream)
PyObject* adapter_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    const tp_grid_t* grid; tp_dims_t dims; int steps, accumulate; tp_adapters_t ad; Inputs dy; Factors f; tp_factor_t fa; MaybeDropout drop;
    tp_oblk_t base, dx; MaybeInput x, own; tp_factor_out_t da, db; float* v; void* stream; Workspace ws; Devices at;
    if (!count(n, 18) || !to_struct(a[0], &grid) || !to_dims(a[1], &dims) || !to_int(a[2], &steps) || !to_adapters(a[3], &ad, &at)) return nullptr;
    const Share s = share(grid, &dims, TP_PASS_DX), fs = share(grid, &dims, TP_PASS_FWD);
    const bool wants_dx = a[9] != Py_None, wants_da = a[11] != Py_None, wants_db = a[14] != Py_None;       // (what is not used may be any block)
    const int used = wants_dx || wants_da ? steps : 0;
    if (!dy.fill(a[4], &at, {s.m, s.k, "a block of dY"}, used) || !f.fill(a[5], ad, &at, s.k, "a chunk of B", used) ||
        !to_factor(a[6], &fa, ad, g_bf16, &at, wants_dx ? s.n : 0, "a") || !drop.fill(a[7], &at) ||
        !to_block(a[8], nullptr, &at, {wants_dx ? s.m : 0, s.n, "dx_base"}, &base) || !to_block(a[9], nullptr, &at, {s.m, s.n, "dx"}, &dx) ||
        !x.fill(a[10], &at, {wants_da ? s.m : 0, s.n, "x_own"}) || !to_factor(a[11], &da, ad, g_f32, &at, s.n, "da") ||
        !own.fill(a[12], &at, {wants_db ? fs.m : 0, fs.n, "dy_own"}) || !to_v(a[13], &v, &at, wants_db ? fs.m : 0, ad.rank) ||
        !to_factor(a[14], &db, ad, g_f32, &at, fs.n, "db") || !to_int(a[15], &accumulate) || !look(a[16], nullptr, &at) || !to_ws(a[16], &ws) || !to_ptr(a[17], &stream))
        return nullptr;
    return answer([&] {
        return f_adapter_bwd(grid, &dims, steps, &ad, dy.ptr, f.ptr, a[6] == Py_None ? nullptr : &fa, drop.ptr, base, dx, x.ptr, da, own.ptr, v, db, accumulate,
                             ws.ptr, ws.bytes, stream);
    });
}
// bind(addresses of the first seven functions in the order above, torch.float32, torch.bfloat16)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* f[7];
    if (!count(n, 9)) return nullptr;
    for (int i = 0; i < 7; ++i)
        if (!to_ptr(a[i], &f[i])) return nullptr;
    f_fwd = reinterpret_cast<decltype(f_fwd)>(f[0]);
    f_static = reinterpret_cast<decltype(f_static)>(f[1]);
    f_bwd = reinterpret_cast<decltype(f_bwd)>(f[2]);
    f_partials = reinterpret_cast<decltype(f_partials)>(f[3]);
    f_bias_act = reinterpret_cast<decltype(f_bias_act)>(f[4]);
    f_dgelu = reinterpret_cast<decltype(f_dgelu)>(f[5]);
    f_bias_grad = reinterpret_cast<decltype(f_bias_grad)>(f[6]);
    Py_INCREF(a[7]); Py_XSETREF(g_f32, a[7]);
    Py_INCREF(a[8]); Py_XSETREF(g_bf16, a[8]);
    Py_RETURN_NONE;
}

// bind_ops(addresses of the functions behind those and of tp_block_map, torch.int32, torch.int64, torch.uint64, torch.Tensor, the address of hipGetDevice or None)
PyObject* bind_ops(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void *f[5], *get_device;
    if (!count(n, 10)) return nullptr;
    for (int i = 0; i < 5; ++i)
        if (!to_ptr(a[i], &f[i])) return nullptr;
    if (!to_ptr(a[9], &get_device)) return nullptr;
    Py_INCREF(a[5]); Py_XSETREF(g_i32, a[5]);
    Py_INCREF(a[6]); Py_XSETREF(g_i64, a[6]);
    Py_INCREF(a[7]); Py_XSETREF(g_u64, a[7]);
    Py_INCREF(a[8]); Py_XSETREF(g_tensor, a[8]);
    g_current_device = reinterpret_cast<decltype(g_current_device)>(get_device);
    f_block_map = reinterpret_cast<decltype(f_block_map)>(f[4]);
    f_adapter_fwd = reinterpret_cast<decltype(f_adapter_fwd)>(f[2]);
    f_adapter_bwd = reinterpret_cast<decltype(f_adapter_bwd)>(f[3]);
    f_dropout_fwd = reinterpret_cast<decltype(f_dropout_fwd)>(f[0]);
    f_dropout_bwd = reinterpret_cast<decltype(f_dropout_bwd)>(f[1]);
    Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"fwd", FAST(fwd)}, {"fwd_static", FAST(fwd_static)}, {"bwd", FAST(bwd)}, {"bwd_partials", FAST(bwd_partials)},
                         {"bias_act", FAST(bias_act)}, {"dgelu", FAST(dgelu)}, {"bias_grad", FAST(bias_grad)}, {"bind", FAST(bind)},
                         {"dropout_fwd", FAST(dropout_fwd)}, {"dropout_bwd", FAST(dropout_bwd)}, {"adapter_fwd", FAST(adapter_fwd)},
                         {"adapter_bwd", FAST(adapter_bwd)}, {"bind_ops", FAST(bind_ops)},
                         {nullptr, nullptr, 0, nullptr}};
// (Set up in its exec slot: a second load of the file makes a module of its own.  A module set up in one go would fill the one that stands under
// this name in sys.modules, which may be another copy's.)
int exec(PyObject*) {
    struct { PyObject** to; const char* name; } names[] = {{&s_data_ptr, "data_ptr"}, {&s_stride, "stride"}, {&s_shape, "shape"},
                                                           {&s_dtype, "dtype"}, {&s_numel, "numel"}, {&s_element_size, "element_size"},
                                                           {&s_get_device, "get_device"}, {&s_is_contiguous, "is_contiguous"}};
    for (auto& x : names)
        if (!*x.to && !(*x.to = PyUnicode_InternFromString(x.name))) return -1;
    return 0;
}
PyModuleDef_Slot slots[] = {{Py_mod_exec, reinterpret_cast<void*>(exec)}, {0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tpcall", "argument marshalling of the libtplinear binding", 0, methods, slots, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tpcall(void) { return PyModuleDef_Init(&module); }
