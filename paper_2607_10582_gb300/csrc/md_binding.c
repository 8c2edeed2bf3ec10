/* Argument marshalling of the per-step calls for the Python binding.
 *
 * Through ctypes a call spends most of its host time converting arguments and
 * reading array addresses: more than the GPU takes for a short step or for one
 * layer of a small batch.  Here a call converts its arguments with the C API
 * and calls the library directly.  On a Grace core, a decode step and its
 * observation: 448 tokens 26.0 -> 15.8 us, 1,700 tokens 32.9 -> 18.8 us; 28
 * layer calls 176 -> 143 us.
 *
 * Device buffers are None, an address, or an object with data_ptr() (a torch
 * tensor).  Host arrays are taken in place when they are C-contiguous of the
 * exact type; for anything else a call returns None and the caller converts
 * the array first.  The GIL is released around the library's calls, as ctypes
 * does. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include "../../include/memdecay.h"

static PyObject *s_data_ptr, *s_is_cuda, *s_is_contiguous, *s_cdata;
static md_status (*f_decode_step)(md_ctx *, int, const void *, const void *, const void *, const uint8_t *, void *);
static md_status (*f_decode_step_host)(md_ctx *, int, const void *, const void *, const void *, const uint8_t *,
                                       void *);
static md_status (*f_decode_layer)(md_ctx *, int, int, const void *, const void *, const void *, const uint8_t *,
                                   void *);
static md_status (*f_evict)(md_ctx *, int, const int32_t *, int32_t *, int32_t *);
static md_status (*f_get_state)(md_ctx *, int, void *, size_t);
static md_status (*f_norm_rope)(const md_norm_rope_args *);
static md_status (*f_page_bounds)(const void *, const int32_t *, const int32_t *, const int32_t *, void *, int, int, int,
                                  int, int, int, void *);
static md_status (*f_page_scores)(const void *, const void *, const int32_t *, const int32_t *, float *, int, int, int,
                                  int, int, int, int, void *);
static md_status (*f_page_top)(const float *, const int32_t *, int32_t *, int, int, int, int, int, int, int, int, void *);
static md_status (*f_attend_pages)(const void *, const void *, const int32_t *, const int32_t *, const int32_t *, void *,
                                   float *, int, int, int, int, int, int, int, int, void *);
static md_status (*f_write_cache8)(const md_cache8_args *);
static md_status (*f_read_cache8)(const md_cache8_args *);
static md_status (*f_attend_cache)(const md_attend_cache_args *);

static PyObject *load(PyObject *self, PyObject *path) {
  const char *s = PyUnicode_AsUTF8(path);
  if (!s) return NULL;
  void *h = dlopen(s, RTLD_NOW | RTLD_LOCAL);
  if (!h) {
    PyErr_SetString(PyExc_OSError, dlerror());
    return NULL;
  }
  *(void **)&f_decode_step = dlsym(h, "md_decode_step");
  *(void **)&f_decode_step_host = dlsym(h, "md_decode_step_host");
  *(void **)&f_decode_layer = dlsym(h, "md_decode_layer");
  *(void **)&f_evict = dlsym(h, "md_evict");
  *(void **)&f_get_state = dlsym(h, "md_get_state");
  *(void **)&f_norm_rope = dlsym(h, "md_norm_rope");
  *(void **)&f_page_bounds = dlsym(h, "md_page_bounds");
  *(void **)&f_page_scores = dlsym(h, "md_page_scores");
  *(void **)&f_page_top = dlsym(h, "md_page_top");
  *(void **)&f_attend_pages = dlsym(h, "md_attend_pages");
  *(void **)&f_write_cache8 = dlsym(h, "md_write_cache8");
  *(void **)&f_read_cache8 = dlsym(h, "md_read_cache8");
  *(void **)&f_attend_cache = dlsym(h, "md_attend_cache");
  if (!f_decode_step || !f_decode_step_host || !f_decode_layer || !f_evict || !f_get_state || !f_norm_rope ||
      !f_page_bounds || !f_page_scores || !f_page_top || !f_attend_pages || !f_write_cache8 || !f_read_cache8 ||
      !f_attend_cache) {
    PyErr_SetString(PyExc_OSError, "libmemdecay.so lacks an entry point");
    return NULL;
  }
  Py_RETURN_NONE;
}

/* Device address of a buffer argument; -1 with an exception set on failure. */
static int dev_ptr(PyObject *o, void **out) {
  if (o == Py_None) {
    *out = NULL;
    return 0;
  }
  if (PyLong_Check(o)) {
    *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
    return PyErr_Occurred() ? -1 : 0;
  }
  PyObject *v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!v) return -1;
  *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(v);
  Py_DECREF(v);
  return PyErr_Occurred() ? -1 : 0;
}

/* Address of a contiguous CPU tensor: 1, 0 if it is something else or not
 * contiguous (no exception: the caller reports it), -1 with an exception. */
static int host_ptr(PyObject *o, void **out) {
  PyObject *v = PyObject_GetAttr(o, s_is_cuda);
  if (!v) {
    PyErr_Clear();
    return 0;
  }
  const int cuda = v != Py_False;
  Py_DECREF(v);
  if (cuda) return 0;
  v = PyObject_CallMethodNoArgs(o, s_is_contiguous);
  if (!v) return -1;
  const int dense = v == Py_True;
  Py_DECREF(v);
  if (!dense) return 0;
  return dev_ptr(o, out) ? -1 : 1;
}

/* A one-dimensional C-contiguous buffer of items with this format: 1 and the
 * view (to be released), 0 if it is something else, never an exception.  Not a
 * byte string: the caller's conversion reads its bytes as text. */
static int host_view(PyObject *o, char format, Py_ssize_t item, int writable, Py_buffer *view) {
  if (PyBytes_Check(o)) return 0;
  if (PyObject_GetBuffer(o, view, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT | (writable ? PyBUF_WRITABLE : 0)) != 0) {
    PyErr_Clear();
    return 0;
  }
  const char *f = view->format ? view->format : "B";
  if (view->ndim == 1 && view->itemsize == item && f[0] == format && f[1] == 0) return 1;
  PyBuffer_Release(view);
  return 0;
}

/* The labels of a step: one per sequence of the batch at least. */
static int label_view(PyObject *o, int batch, Py_buffer *view) {
  if (!host_view(o, 'B', 1, 0, view)) return 0;
  if (view->shape[0] >= batch) return 1;
  PyBuffer_Release(view);
  return 0;
}

static int as_int(PyObject *o, int *out) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) return -1;
  *out = (int)v;
  return 0;
}

static int arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 0;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return -1;
}

/* decode_step(handle, batch, q, k_new, v_new, new_regions, out) -> status, or
 * None when new_regions must be converted */
static PyObject *decode_step(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *h, *q, *k, *v, *out;
  int batch, st;
  Py_buffer regs;
  if (arity(n, 7) || dev_ptr(a[0], &h) || as_int(a[1], &batch) || dev_ptr(a[2], &q) || dev_ptr(a[3], &k) ||
      dev_ptr(a[4], &v) || dev_ptr(a[6], &out))
    return NULL;
  if (!label_view(a[5], batch, &regs)) Py_RETURN_NONE;
  Py_BEGIN_ALLOW_THREADS
  st = f_decode_step((md_ctx *)h, batch, q, k, v, (const uint8_t *)regs.buf, out);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&regs);
  return PyLong_FromLong(st);
}

/* decode_step_host(handle, batch, q, k_new, v_new, new_regions, out): host
 * buffers are contiguous CPU tensors */
static PyObject *decode_step_host(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *h, *x[4];
  int batch, st;
  Py_buffer regs;
  if (arity(n, 7) || dev_ptr(a[0], &h) || as_int(a[1], &batch)) return NULL;
  for (int i = 0; i < 4; ++i) {
    const int ok = host_ptr(a[i < 3 ? 2 + i : 6], &x[i]);
    if (ok < 0) return NULL;
    if (ok == 0) Py_RETURN_NONE;
  }
  if (!label_view(a[5], batch, &regs)) Py_RETURN_NONE;
  Py_BEGIN_ALLOW_THREADS
  st = f_decode_step_host((md_ctx *)h, batch, x[0], x[1], x[2], (const uint8_t *)regs.buf, x[3]);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&regs);
  return PyLong_FromLong(st);
}

/* decode_layer(handle, layer, batch, q, k_new, v_new, new_regions, out) */
static PyObject *decode_layer(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *h, *q, *k, *v, *out;
  int layer, batch, st;
  Py_buffer regs;
  if (arity(n, 8) || dev_ptr(a[0], &h) || as_int(a[1], &layer) || as_int(a[2], &batch) || dev_ptr(a[3], &q) ||
      dev_ptr(a[4], &k) || dev_ptr(a[5], &v) || dev_ptr(a[7], &out))
    return NULL;
  if (!label_view(a[6], layer == 0 ? batch : 0, &regs)) Py_RETURN_NONE;   // later layers read none
  Py_BEGIN_ALLOW_THREADS
  st = f_decode_layer((md_ctx *)h, layer, batch, q, k, v, (const uint8_t *)regs.buf, out);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&regs);
  return PyLong_FromLong(st);
}

/* evict(handle, budgets, n_evicted, evicted_ids) -> status; budgets and
 * n_evicted are int32 arrays of one length, or None is returned */
static PyObject *evict(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *h, *ids;
  int st;
  Py_buffer bud, ev;
  if (arity(n, 4) || dev_ptr(a[0], &h) || dev_ptr(a[3], &ids)) return NULL;
  if (!host_view(a[1], 'i', 4, 0, &bud)) Py_RETURN_NONE;
  if (!host_view(a[2], 'i', 4, 1, &ev)) {
    PyBuffer_Release(&bud);
    Py_RETURN_NONE;
  }
  if (bud.shape[0] != ev.shape[0]) {
    PyBuffer_Release(&bud);
    PyBuffer_Release(&ev);
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  st = f_evict((md_ctx *)h, (int)bud.shape[0], (const int32_t *)bud.buf, (int32_t *)ev.buf, (int32_t *)ids);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&bud);
  PyBuffer_Release(&ev);
  return PyLong_FromLong(st);
}

/* get_state(handle, what, dst, bytes) -> status */
static PyObject *get_state(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *h, *dst;
  int what, st;
  if (arity(n, 4) || dev_ptr(a[0], &h) || as_int(a[1], &what) || dev_ptr(a[2], &dst)) return NULL;
  const long long bytes = PyLong_AsLongLong(a[3]);
  if (bytes == -1 && PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  st = f_get_state((md_ctx *)h, what, dst, (size_t)bytes);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* ---- calls without a handle: whatever they do not take as it is (another type,
 * shape, layout or device, an argument missing) they leave to the caller, by
 * None, who converts it or says what is wrong ---- */

/* A tensor's address, type, shape, strides and device come from torch's C interface
 * (exported by its libraries, the same across versions), which takes the address of
 * a pointer to the tensor's implementation: one attribute of the Python object.
 * Against reading the object's attributes, on a Grace core, a call: norm_rope of one
 * token (ten tensors) 6.4 -> 4.0 us, bounds of 32 pages 4.4 -> 3.5, scores of one row
 * 4.7 -> 3.5, attention of one row over one layer 5.9 -> 4.9. */
enum { T_BF16, T_F16, T_F32, T_I16, T_I32, T_E4M3, T_U8, T_OTHER };
#define MAX_DIMS 6

static struct {
  PyObject *tensor, *parameter;      /* torch.Tensor, torch.nn.Parameter; tensor NULL: not loaded */
  int32_t types[T_OTHER], cuda;
  int32_t (*get_data_ptr)(void *, void **);
  int32_t (*get_dim)(void *, int64_t *);
  int32_t (*get_sizes)(void *, int64_t **);
  int32_t (*get_strides)(void *, int64_t **);
  int32_t (*get_dtype)(void *, int32_t *);
  int32_t (*get_device_type)(void *, int32_t *);
  int32_t (*get_device_index)(void *, int32_t *);
  int32_t (*current_device)(int32_t *);
  int32_t (*current_stream)(int32_t, void **);
} torch_c;

/* load_torch(Tensor, Parameter, path of libtorch_cpu, of libtorch_cuda) -> whether
 * the calls below take tensors; the libraries are the ones torch has loaded */
static PyObject *load_torch(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  if (arity(n, 4)) return NULL;
  const char *cpu = PyUnicode_AsUTF8(a[2]), *cuda = cpu ? PyUnicode_AsUTF8(a[3]) : NULL;
  if (!cuda) return NULL;
  void *l = dlopen(cpu, RTLD_NOW | RTLD_NOLOAD), *g = dlopen(cuda, RTLD_NOW | RTLD_NOLOAD);
  if (!l || !g) Py_RETURN_FALSE;
  static const char *const kinds[T_OTHER] = {"aoti_torch_dtype_bfloat16", "aoti_torch_dtype_float16",
                                             "aoti_torch_dtype_float32", "aoti_torch_dtype_int16",
                                             "aoti_torch_dtype_int32", "aoti_torch_dtype_float8_e4m3fn",
                                             "aoti_torch_dtype_uint8"};
  int32_t (*kind)(void);
  for (int i = 0; i < T_OTHER; ++i) {
    *(void **)&kind = dlsym(l, kinds[i]);
    if (!kind) Py_RETURN_FALSE;
    torch_c.types[i] = kind();
  }
  *(void **)&kind = dlsym(l, "aoti_torch_device_type_cuda");
  if (!kind) Py_RETURN_FALSE;
  torch_c.cuda = kind();
  *(void **)&torch_c.get_data_ptr = dlsym(l, "aoti_torch_get_data_ptr");
  *(void **)&torch_c.get_dim = dlsym(l, "aoti_torch_get_dim");
  *(void **)&torch_c.get_sizes = dlsym(l, "aoti_torch_get_sizes");
  *(void **)&torch_c.get_strides = dlsym(l, "aoti_torch_get_strides");
  *(void **)&torch_c.get_dtype = dlsym(l, "aoti_torch_get_dtype");
  *(void **)&torch_c.get_device_type = dlsym(l, "aoti_torch_get_device_type");
  *(void **)&torch_c.get_device_index = dlsym(l, "aoti_torch_get_device_index");
  *(void **)&torch_c.current_device = dlsym(l, "aoti_torch_get_current_device_index");
  *(void **)&torch_c.current_stream = dlsym(g, "aoti_torch_get_current_cuda_stream");
  if (!torch_c.get_data_ptr || !torch_c.get_dim || !torch_c.get_sizes || !torch_c.get_strides || !torch_c.get_dtype ||
      !torch_c.get_device_type || !torch_c.get_device_index || !torch_c.current_device || !torch_c.current_stream)
    Py_RETURN_FALSE;
  Py_XSETREF(torch_c.parameter, Py_NewRef(a[1]));
  Py_XSETREF(torch_c.tensor, Py_NewRef(a[0]));
  Py_RETURN_TRUE;
}

typedef struct {
  void *p;
  int dims, type;
  int32_t device;
  int64_t n[MAX_DIMS], stride[MAX_DIMS];
} tensor;

/* A tensor on a GPU (not of a subclass, which may be something else): 1, or 0 (an
 * exception may be set). */
static int device_tensor(PyObject *o, tensor *t) {
  if (!torch_c.tensor || ((PyObject *)Py_TYPE(o) != torch_c.tensor && (PyObject *)Py_TYPE(o) != torch_c.parameter)) return 0;
  PyObject *v = PyObject_GetAttr(o, s_cdata);
  if (!v) return 0;
  void *impl = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (!impl) return 0;
  int32_t kind, type;
  int64_t dims, *n, *stride;
  if (torch_c.get_device_type(&impl, &kind) || kind != torch_c.cuda || torch_c.get_device_index(&impl, &t->device) ||
      torch_c.get_dtype(&impl, &type) || torch_c.get_dim(&impl, &dims) || dims > MAX_DIMS ||
      torch_c.get_sizes(&impl, &n) || torch_c.get_strides(&impl, &stride) || torch_c.get_data_ptr(&impl, &t->p))
    return 0;
  t->dims = (int)dims;
  for (int i = 0; i < dims; ++i) {
    t->n[i] = n[i];
    t->stride[i] = stride[i];
  }
  for (t->type = 0; t->type < T_OTHER && torch_c.types[t->type] != type; ++t->type) {
  }
  return 1;
}

static int two_bytes(const tensor *t) { return t->type == T_BF16 || t->type == T_I16; }

/* A contiguous one. */
static int dense_tensor(PyObject *o, tensor *t) {
  if (!device_tensor(o, t)) return 0;
  int64_t want = 1;
  for (int i = t->dims - 1; i >= 0; --i) {
    if (t->n[i] == 0) return 1;
    if (t->n[i] > 1 && t->stride[i] != want) return 0;
    want *= t->n[i];
  }
  return 1;
}

static int has_shape(const tensor *t, int dims, long long a, long long b, long long c, long long d, long long e) {
  const long long want[5] = {a, b, c, d, e};
  if (t->dims != dims) return 0;
  for (int i = 0; i < dims; ++i)
    if (t->n[i] != want[i]) return 0;
  return 1;
}

/* The stream of a call whose tensors lie on `device`, which has to be the current
 * one: an address, or None for the current stream. */
static int call_stream(int32_t device, PyObject *o, void **out) {
  int32_t now;
  if (torch_c.current_device(&now) || now != device) return 0;
  return o == Py_None ? torch_c.current_stream(device, out) == 0 : dev_ptr(o, out) == 0;
}

static PyObject *leave(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

/* int32 counts, one per sequence at least */
static int count_view(PyObject *o, long long batch, Py_buffer *view) {
  if (!host_view(o, 'i', 4, 0, view)) return 0;
  if (view->shape[0] >= batch) return 1;
  PyBuffer_Release(view);
  return 0;
}

/* Rows [tokens][heads][128] with their strides over tokens and heads. */
static int row_tensor(PyObject *o, tensor *t, int64_t *token, int64_t *head) {
  if (!device_tensor(o, t) || t->dims != 3 || t->n[2] != MD_HEAD_DIM || t->stride[2] != 1) return 0;
  *token = t->n[0] > 1 ? t->stride[0] : 0;
  *head = t->n[1] > 1 ? t->stride[1] : 0;
  return 1;
}

/* norm_rope(q, k, v, q_out, k_out, v_out, positions, table, q_weight, k_weight,
 * eps, axes, interleaved, stream) */
static PyObject *norm_rope(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  if (arity(n, 14)) return NULL;
  md_norm_rope_args r = {0};
  tensor x[3], y[3], t;
  int64_t *in[3][2] = {{&r.q_token, &r.q_head}, {&r.k_token, &r.k_head}, {&r.v_token, &r.v_head}};
  int64_t *out[3][2] = {{&r.q_out_token, &r.q_out_head}, {&r.k_out_token, &r.k_out_head}, {&r.v_out_token, &r.v_out_head}};
  if (a[0] == Py_None && a[1] == Py_None) return leave();
  const int first = a[0] != Py_None ? 0 : 1;
  for (int i = first; i < 3; ++i) {
    if (a[i] == Py_None) continue;
    if (!row_tensor(a[i], &x[i], in[i][0], in[i][1]) || !row_tensor(a[3 + i], &y[i], out[i][0], out[i][1]))
      return leave();
    if (x[i].device != x[first].device || y[i].device != x[first].device || x[i].type != x[first].type ||
        x[i].n[0] != x[first].n[0] || !two_bytes(&y[i]) || y[i].n[0] != x[i].n[0] ||
        y[i].n[1] != x[i].n[1])
      return leave();
  }
  const int hq = a[0] != Py_None, hk = a[1] != Py_None, hv = a[2] != Py_None;
  if (x[first].type > T_F32 || x[first].n[0] > INT32_MAX || (hv && (!hk || x[2].n[1] != x[1].n[1]))) return leave();
  r.n_tokens = (int)x[first].n[0];
  r.type = x[first].type == T_BF16 ? MD_TYPE_BF16 : x[first].type == T_F16 ? MD_TYPE_F16 : MD_TYPE_F32;
  if (hq) r.q = x[0].p, r.q_out = y[0].p, r.num_q_heads = (int)x[0].n[1];
  if (hk) r.k = x[1].p, r.k_out = y[1].p, r.num_kv_heads = (int)x[1].n[1];
  if (hv) r.v = x[2].p, r.v_out = y[2].p;
  for (int i = 0; i < 2; ++i) {
    if (a[8 + i] == Py_None || a[i] == Py_None) continue;
    if (!dense_tensor(a[8 + i], &t) || t.type != T_F32 || !has_shape(&t, 1, MD_HEAD_DIM, 0, 0, 0, 0) ||
        t.device != x[first].device)
      return leave();
    *(i ? &r.k_weight : &r.q_weight) = (const float *)t.p;
  }
  Py_buffer axes = {0};
  const double eps = PyFloat_AsDouble(a[10]);
  if (PyErr_Occurred() || !call_stream(x[first].device, a[13], &r.stream)) return leave();
  r.eps = (float)eps;
  r.interleaved = PyObject_IsTrue(a[12]);
  if (r.interleaved < 0) return leave();
  if (a[7] != Py_None) {
    if (!dense_tensor(a[7], &t) || t.type != T_F32 || t.dims != 3 || t.n[2] != 2 || t.n[0] > INT32_MAX ||
        t.n[1] > MD_HEAD_DIM / 2 || t.device != x[first].device)
      return leave();
    r.table = (const float *)t.p;
    r.table_len = (int)t.n[0];
    r.rotary_dim = 2 * (int)t.n[1];
    if (!dense_tensor(a[6], &t) || t.type != T_I32 || t.dims < 1 || t.dims > 2 || t.n[t.dims - 1] != r.n_tokens ||
        (t.dims == 2 && t.n[0] > MD_MAX_AXES) || t.device != x[first].device)
      return leave();
    r.positions = (const int32_t *)t.p;
    r.num_axes = t.dims == 2 ? (int)t.n[0] : 1;
    if (a[11] != Py_None) {
      if (!host_view(a[11], 'B', 1, 0, &axes)) return leave();
      if (axes.shape[0] < r.rotary_dim / 2) {
        PyBuffer_Release(&axes);
        return leave();
      }
      r.axis_host = (const uint8_t *)axes.buf;
    }
  }
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_norm_rope(&r);
  Py_END_ALLOW_THREADS
  if (r.axis_host) PyBuffer_Release(&axes);
  return PyLong_FromLong(st);
}

/* A pool [L][pages][Hkv][2][page_size][128]. */
static int pool_tensor(PyObject *o, tensor *t) {
  return dense_tensor(o, t) && t->dims == 6 && two_bytes(t) && t->n[3] == 2 && t->n[5] == MD_HEAD_DIM &&
         t->n[0] < 256 && t->n[1] < INT32_MAX && t->n[2] < INT32_MAX;
}
static int block_table_tensor(PyObject *o, tensor *t) {
  return dense_tensor(o, t) && t->dims == 2 && t->type == T_I32 && t->n[0] <= MD_MAX_BATCH && t->n[1] < INT32_MAX;
}

/* page_bounds(pool, block_table, n_tokens, first_pages, bounds, stream) */
static PyObject *page_bounds(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  tensor pool, table, bounds;
  void *s;
  Py_buffer count, first = {0};
  if (arity(n, 6)) return NULL;
  if (!pool_tensor(a[0], &pool) || !block_table_tensor(a[1], &table) || !dense_tensor(a[4], &bounds) ||
      !two_bytes(&bounds) || !has_shape(&bounds, 5, pool.n[0], pool.n[1], pool.n[2], 2, MD_HEAD_DIM) ||
      table.device != pool.device || bounds.device != pool.device || !call_stream(pool.device, a[5], &s) ||
      !count_view(a[2], table.n[0], &count))
    return leave();
  if (a[3] != Py_None && !count_view(a[3], table.n[0], &first)) {
    PyBuffer_Release(&count);
    return leave();
  }
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_page_bounds(pool.p, table.p, count.buf, a[3] == Py_None ? NULL : first.buf, bounds.p, (int)table.n[0],
                               (int)pool.n[0], (int)pool.n[2], (int)pool.n[4], (int)table.n[1], (int)pool.n[1], s);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&count);
  if (a[3] != Py_None) PyBuffer_Release(&first);
  return PyLong_FromLong(st);
}

/* page_scores(q, bounds, block_table, n_tokens, scores, page_size, stream) */
static PyObject *page_scores(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  tensor q, bounds, table, scores;
  void *s;
  int ps;
  Py_buffer count;
  if (arity(n, 7)) return NULL;
  if (!dense_tensor(a[0], &q) || !two_bytes(&q) || q.dims != 4 || q.n[2] > INT32_MAX || !dense_tensor(a[1], &bounds) ||
      !two_bytes(&bounds) || bounds.dims != 5 || bounds.n[0] > 255 || bounds.n[1] > INT32_MAX ||
      bounds.n[2] > INT32_MAX || bounds.n[3] != 2 || bounds.n[4] != MD_HEAD_DIM || !block_table_tensor(a[2], &table) ||
      !has_shape(&q, 4, table.n[0], bounds.n[0], q.n[2], MD_HEAD_DIM, 0) || !dense_tensor(a[4], &scores) ||
      scores.type != T_F32 || !has_shape(&scores, 4, table.n[0], bounds.n[0], bounds.n[2], table.n[1], 0) ||
      as_int(a[5], &ps) || bounds.device != q.device || table.device != q.device || scores.device != q.device ||
      !call_stream(q.device, a[6], &s) || !count_view(a[3], table.n[0], &count))
    return leave();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_page_scores(q.p, bounds.p, table.p, count.buf, scores.p, (int)table.n[0], (int)bounds.n[0],
                               (int)q.n[2], (int)bounds.n[2], ps, (int)table.n[1], (int)bounds.n[1], s);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&count);
  return PyLong_FromLong(st);
}

/* page_top(scores, n_tokens, page_ids, page_size, first, last, stream) */
static PyObject *page_top(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  tensor scores, ids;
  void *s;
  int ps, first, last;
  Py_buffer count;
  if (arity(n, 7)) return NULL;
  if (!dense_tensor(a[0], &scores) || scores.type != T_F32 || scores.dims != 4 || scores.n[0] > MD_MAX_BATCH ||
      scores.n[1] > 255 || scores.n[2] > INT32_MAX || scores.n[3] > INT32_MAX || !dense_tensor(a[2], &ids) ||
      ids.type != T_I32 || ids.dims != 4 || ids.n[3] > INT32_MAX ||
      !has_shape(&ids, 4, scores.n[0], scores.n[1], scores.n[2], ids.n[3], 0) || as_int(a[3], &ps) ||
      as_int(a[4], &first) || as_int(a[5], &last) || ids.device != scores.device ||
      !call_stream(scores.device, a[6], &s) || !count_view(a[1], scores.n[0], &count))
    return leave();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_page_top(scores.p, count.buf, ids.p, (int)scores.n[0], (int)scores.n[1], (int)scores.n[2], ps,
                            (int)scores.n[3], (int)ids.n[3], first, last, s);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&count);
  return PyLong_FromLong(st);
}

/* attend_pages(q, pool, block_table, n_tokens, page_ids, out, mass, stream) */
static PyObject *attend_pages(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  tensor q, pool, table, ids, out, mass = {0};
  void *s;
  Py_buffer count;
  if (arity(n, 8)) return NULL;
  if (!dense_tensor(a[0], &q) || !two_bytes(&q) || q.dims != 4 || q.n[2] > INT32_MAX || !pool_tensor(a[1], &pool) ||
      !block_table_tensor(a[2], &table) || !has_shape(&q, 4, table.n[0], pool.n[0], q.n[2], MD_HEAD_DIM, 0) ||
      !dense_tensor(a[4], &ids) || ids.type != T_I32 || ids.dims != 4 || ids.n[3] > MD_MAX_TOP_TOKENS ||
      !has_shape(&ids, 4, table.n[0], pool.n[0], pool.n[2], ids.n[3], 0) || !dense_tensor(a[5], &out) ||
      !two_bytes(&out) || !has_shape(&out, 4, q.n[0], q.n[1], q.n[2], q.n[3], 0))
    return leave();
  if (a[6] != Py_None &&
      (!dense_tensor(a[6], &mass) || mass.type != T_F32 ||
       !has_shape(&mass, 4, table.n[0], pool.n[0], pool.n[2], ids.n[3] * pool.n[4], 0)))
    return leave();
  if (pool.device != q.device || table.device != q.device || ids.device != q.device || out.device != q.device ||
      (mass.p && mass.device != q.device) || !call_stream(q.device, a[7], &s) || !count_view(a[3], table.n[0], &count))
    return leave();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_attend_pages(q.p, pool.p, table.p, count.buf, ids.p, out.p, mass.p, (int)table.n[0], (int)pool.n[0],
                                (int)q.n[2], (int)pool.n[2], (int)pool.n[4], (int)table.n[1], (int)pool.n[1],
                                (int)ids.n[3], s);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&count);
  return PyLong_FromLong(st);
}

static int one_byte(const tensor *t) { return t->type == T_E4M3 || t->type == T_U8; }

/* A pool in eight bits, [L][pages][Hkv][2][page_size][128], and its scales. */
static int pool8_tensor(PyObject *o, tensor *t) {
  return dense_tensor(o, t) && t->dims == 6 && one_byte(t) && t->n[3] == 2 && t->n[5] == MD_HEAD_DIM &&
         t->n[0] < 256 && t->n[1] < INT32_MAX && t->n[2] < INT32_MAX && t->n[4] < INT32_MAX;
}
static int scale_tensor(PyObject *o, tensor *t, const tensor *pool) {
  return dense_tensor(o, t) && t->type == T_F32 &&
         has_shape(t, 5, pool->n[0], pool->n[1], pool->n[2], 2, pool->n[4] / MD_SCALE_TOKENS) && t->device == pool->device;
}

/* (k, v, pool, scales, block_table, first, count, stream) of md_write_cache8 and md_read_cache8 */
static PyObject *cache8(PyObject *const *a, Py_ssize_t n, md_status (*f)(const md_cache8_args *)) {
  if (arity(n, 8)) return NULL;
  md_cache8_args r = {0};
  tensor x[2], pool, scales, table;
  int64_t *stride[2][3] = {{&r.k_row, &r.k_layer, &r.k_head}, {&r.v_row, &r.v_layer, &r.v_head}};
  if (!pool8_tensor(a[2], &pool) || !scale_tensor(a[3], &scales, &pool) || !block_table_tensor(a[4], &table) ||
      table.device != pool.device)
    return leave();
  for (int i = 0; i < 2; ++i) {
    if (!device_tensor(a[i], &x[i]) || x[i].dims != 4 || x[i].type > T_F32 || x[i].type != x[0].type ||
        x[i].device != pool.device || x[i].n[0] != x[0].n[0] || x[i].n[1] != pool.n[0] || x[i].n[2] != pool.n[2] ||
        x[i].n[3] != MD_HEAD_DIM || x[i].stride[3] != 1)
      return leave();
    for (int d = 0; d < 3; ++d) {
      if (f == f_read_cache8 && x[i].n[d] > 1 && x[i].stride[d] == 0) return leave();   // rows on one another
      *stride[i][d] = x[i].n[d] > 1 ? x[i].stride[d] : 0;
    }
  }
  Py_buffer first, count;
  if (!call_stream(pool.device, a[7], &r.stream) || !count_view(a[5], table.n[0], &first)) return leave();
  if (!count_view(a[6], table.n[0], &count)) {
    PyBuffer_Release(&first);
    return leave();
  }
  long long rows = 0;
  int whole = 1, st = 0;
  for (int64_t b = 0; b < table.n[0]; ++b) {
    const int32_t c = ((const int32_t *)count.buf)[b];
    whole &= c >= 0;
    rows += c;
  }
  if (whole && rows <= x[0].n[0]) {
    r.batch = (int)table.n[0];
    r.num_layers = (int)pool.n[0];
    r.num_kv_heads = (int)pool.n[2];
    r.page_size = (int)pool.n[4];
    r.max_pages_per_seq = (int)table.n[1];
    r.num_phys_pages = (int)pool.n[1];
    r.type = x[0].type == T_BF16 ? MD_TYPE_BF16 : x[0].type == T_F16 ? MD_TYPE_F16 : MD_TYPE_F32;
    r.first_host = first.buf;
    r.count_host = count.buf;
    r.k = x[0].p;
    r.v = x[1].p;
    r.pool_dev = pool.p;
    r.scales_dev = scales.p;
    r.block_table_dev = table.p;
    Py_BEGIN_ALLOW_THREADS
    st = f(&r);
    Py_END_ALLOW_THREADS
  }
  PyBuffer_Release(&first);
  PyBuffer_Release(&count);
  if (!whole || rows > x[0].n[0]) return leave();
  return PyLong_FromLong(st);
}
static PyObject *write_cache8(PyObject *self, PyObject *const *a, Py_ssize_t n) { return cache8(a, n, f_write_cache8); }
static PyObject *read_cache8(PyObject *self, PyObject *const *a, Py_ssize_t n) { return cache8(a, n, f_read_cache8); }

/* A whole number from `least` to INT32_MAX. */
static int count_arg(PyObject *o, int least, int *out) {
  if (!PyLong_Check(o)) return 0;
  const long long v = PyLong_AsLongLong(o);
  if (PyErr_Occurred() || v < least || v > INT32_MAX) return 0;
  *out = (int)v;
  return 1;
}

/* attend_cache(q, pool, block_table, n_tokens, out, scales, window, sinks, lse, workspace, stream) */
static PyObject *attend_cache(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  if (arity(n, 11)) return NULL;
  md_attend_cache_args r = {0};
  tensor q, pool, table, out, t;
  const int wide = a[5] == Py_None;
  if (!(wide ? pool_tensor(a[1], &pool) : pool8_tensor(a[1], &pool)) || !block_table_tensor(a[2], &table) ||
      !dense_tensor(a[0], &q) || !two_bytes(&q) || q.dims != 4 || q.n[2] > INT32_MAX || pool.n[4] > INT32_MAX ||
      !has_shape(&q, 4, table.n[0], pool.n[0], q.n[2], MD_HEAD_DIM, 0) || !dense_tensor(a[4], &out) ||
      !two_bytes(&out) || !has_shape(&out, 4, q.n[0], q.n[1], q.n[2], MD_HEAD_DIM, 0) || q.device != pool.device ||
      table.device != pool.device || out.device != pool.device)
    return leave();
  r.type = MD_TYPE_BF16;
  if (!wide) {
    if (!scale_tensor(a[5], &t, &pool)) return leave();
    r.scales_dev = t.p;
    r.type = MD_TYPE_E4M3;
  }
  r.window = -1;
  if ((a[6] != Py_None && !count_arg(a[6], 0, &r.window)) || !count_arg(a[7], 0, &r.sinks)) return leave();
  if (a[8] != Py_None) {
    if (!dense_tensor(a[8], &t) || t.type != T_F32 || !has_shape(&t, 3, q.n[0], q.n[1], q.n[2], 0, 0) ||
        t.device != pool.device)
      return leave();
    r.lse_dev = t.p;
  }
  if (a[9] != Py_None) {
    if (!dense_tensor(a[9], &t) || t.type != T_U8 || t.dims != 1 || t.device != pool.device) return leave();
    r.workspace_dev = t.p;
    r.workspace_bytes = (size_t)t.n[0];
  }
  Py_buffer count;
  if (!call_stream(pool.device, a[10], &r.stream) || !count_view(a[3], table.n[0], &count)) return leave();
  r.batch = (int)table.n[0];
  r.num_layers = (int)pool.n[0];
  r.num_q_heads = (int)q.n[2];
  r.num_kv_heads = (int)pool.n[2];
  r.page_size = (int)pool.n[4];
  r.max_pages_per_seq = (int)table.n[1];
  r.num_phys_pages = (int)pool.n[1];
  r.q_dev = q.p;
  r.pool_dev = pool.p;
  r.block_table_dev = table.p;
  r.n_tokens_host = count.buf;
  r.out_dev = out.p;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f_attend_cache(&r);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&count);
  return PyLong_FromLong(st);
}

static PyMethodDef methods[] = {
    {"load", load, METH_O, "load(path): binds the calls to libmemdecay.so"},
    {"decode_step", (PyCFunction)(void (*)(void))decode_step, METH_FASTCALL, "md_decode_step"},
    {"decode_step_host", (PyCFunction)(void (*)(void))decode_step_host, METH_FASTCALL, "md_decode_step_host"},
    {"decode_layer", (PyCFunction)(void (*)(void))decode_layer, METH_FASTCALL, "md_decode_layer"},
    {"evict", (PyCFunction)(void (*)(void))evict, METH_FASTCALL, "md_evict"},
    {"get_state", (PyCFunction)(void (*)(void))get_state, METH_FASTCALL, "md_get_state"},
    {"load_torch", (PyCFunction)(void (*)(void))load_torch, METH_FASTCALL, "load_torch(Tensor, Parameter, libtorch_cpu, libtorch_cuda)"},
    {"norm_rope", (PyCFunction)(void (*)(void))norm_rope, METH_FASTCALL, "md_norm_rope"},
    {"page_bounds", (PyCFunction)(void (*)(void))page_bounds, METH_FASTCALL, "md_page_bounds"},
    {"page_scores", (PyCFunction)(void (*)(void))page_scores, METH_FASTCALL, "md_page_scores"},
    {"page_top", (PyCFunction)(void (*)(void))page_top, METH_FASTCALL, "md_page_top"},
    {"attend_pages", (PyCFunction)(void (*)(void))attend_pages, METH_FASTCALL, "md_attend_pages"},
    {"write_cache8", (PyCFunction)(void (*)(void))write_cache8, METH_FASTCALL, "md_write_cache8"},
    {"read_cache8", (PyCFunction)(void (*)(void))read_cache8, METH_FASTCALL, "md_read_cache8"},
    {"attend_cache", (PyCFunction)(void (*)(void))attend_cache, METH_FASTCALL, "md_attend_cache"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_cdata = PyUnicode_InternFromString("_cdata");
  return s_data_ptr && s_is_cuda && s_is_contiguous && s_cdata ? PyModule_Create(&module) : NULL;
}
