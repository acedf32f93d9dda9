// The calls of the replay path for Python, argument marshalling only: numbers, tensors (device pointers) and streams in, the
// status code and what the call reports out.  Loaded by apex.py, which documents the calls; the library itself is opened
// there too, and its entry points are looked up here by name.
//
// What a call costs the host beside its launches, and why this is not done with ctypes: a call with eight tensors took 4 us
// for their checks and addresses and for ctypes' conversion of the arguments, which is more than its launch (2.4 us).
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <tuple>
#include <utility>
#include <vector>

#include "apex_replay.h"

namespace {

PyObject *g_address = nullptr;                                  // apex._ptr: address of what is no torch.Tensor
PyObject *g_plain = nullptr;                                    // apex._plain: what an argument that is no number stands for
PyObject *g_current_device = nullptr, *g_current_stream = nullptr;  // torch's raw handle of the current stream

struct Failed {};  // a Python error is set

// A reference that is given back when it goes out of scope.
struct Ref {
  PyObject *o;
  explicit Ref(PyObject *owned) : o(owned)
  {
    if (!o) throw Failed{};
  }
  Ref(const Ref &) = delete;
  ~Ref() { Py_DECREF(o); }
};

// An integer, whatever has an index (numpy's integers), or what g_plain makes one of; the value modulo 2^64.
unsigned long long integer(PyObject *o, bool plain = false)
{
  if (!PyLong_Check(o)) {
    if (PyIndex_Check(o)) return integer(Ref(PyNumber_Index(o)).o);
    if (!plain) return integer(Ref(PyObject_CallOneArg(g_plain, o)).o, true);
    PyErr_Format(PyExc_TypeError, "an integer is required, not %.80s", Py_TYPE(o)->tp_name);
    throw Failed{};
  }
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (PyErr_Occurred()) throw Failed{};
  return v;
}

// The same for addresses and handles, with None for a null pointer.
void *pointer(PyObject *o)
{
  if (o == Py_None) return nullptr;
  if (PyLong_Check(o) || PyIndex_Check(o)) return reinterpret_cast<void *>(integer(o));
  const Ref p(PyObject_CallOneArg(g_plain, o));
  return p.o == Py_None ? nullptr : reinterpret_cast<void *>(integer(p.o, true));
}

// Device addresses: a contiguous tensor on the GPU, or None.
void *address(PyObject *o)
{
  if (o == Py_None) return nullptr;
  if (THPVariable_Check(o)) {
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
      PyErr_SetString(PyExc_AssertionError, "device, contiguous tensors only");
      throw Failed{};
    }
    return t.data_ptr();
  }
  return pointer(Ref(PyObject_CallOneArg(g_address, o)).o);
}

// A stream object's handle; None: the current device's current stream.
void *stream_handle(PyObject *o)
{
  if (o != Py_None) return pointer(Ref(PyObject_GetAttrString(o, "cuda_stream")).o);
  const Ref device(PyObject_CallNoArgs(g_current_device));
  return pointer(Ref(PyObject_CallOneArg(g_current_stream, device.o)).o);
}

template <typename T>
struct From {  // pointers to device memory
  static_assert(std::is_pointer<T>::value, "");
  static T get(PyObject *o) { return static_cast<T>(address(o)); }
};
template <>
struct From<apex_replay_t *> {
  static apex_replay_t *get(PyObject *o) { return static_cast<apex_replay_t *>(pointer(o)); }
};
template <>
struct From<apex_pipeline_t *> {
  static apex_pipeline_t *get(PyObject *o) { return static_cast<apex_pipeline_t *>(pointer(o)); }
};
template <>
struct From<apex_pe_replay_t *> {
  static apex_pe_replay_t *get(PyObject *o) { return static_cast<apex_pe_replay_t *>(pointer(o)); }
};
template <>
struct From<uint32_t> {
  static uint32_t get(PyObject *o) { return static_cast<uint32_t>(integer(o)); }
};
template <>
struct From<uint64_t> {
  static uint64_t get(PyObject *o) { return static_cast<uint64_t>(integer(o)); }
};
template <>
struct From<int> {
  static int get(PyObject *o) { return static_cast<int>(integer(o)); }
};
template <>
struct From<float> {
  static float get(PyObject *o)
  {
    double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred() && PyErr_ExceptionMatches(PyExc_TypeError)) {
      PyErr_Clear();
      v = PyFloat_AsDouble(Ref(PyObject_CallOneArg(g_plain, o)).o);
    }
    if (v == -1.0 && PyErr_Occurred()) throw Failed{};
    return static_cast<float>(v);
  }
};

// What a call is given does not fit it: an AssertionError, raised where the interpreter's lock is held.
struct Refused {
  const char *why;
};

void require(bool holds, const char *why)
{
  if (!holds) throw Refused{why};
}

// A tensor on the GPU as the operators take theirs: sizes, strides in elements, type.
struct View {
  void *p = nullptr;
  int64_t n[3] = {0, 0, 0}, stride[3] = {0, 0, 0}, count = 0;
  int dim = 0, dtype = -1;  // apex_dtype, or -1
  int device = -1;
  bool contiguous = false, is_int = false, is_long = false;
  bool is_none() const { return dim == 0; }  // (a tensor without elements has no address either)
  bool fits(int64_t a, int64_t b) const { return dim == 2 && n[0] == a && n[1] == b; }
  bool fits(int64_t a, int64_t b, int64_t c) const { return dim == 3 && n[0] == a && n[1] == b && n[2] == c; }
  // the last index is contiguous (where there is anything to step over), the others step forward
  bool rows() const
  {
    bool forward = n[dim - 1] < 2 || stride[dim - 1] == 1;
    for (int i = 0; i + 1 < dim; ++i) forward = forward && stride[i] >= 0;
    return forward;
  }
};
template <>
struct From<View> {
  static View get(PyObject *o)
  {
    View v;
    if (o == Py_None) return v;
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "a tensor is required, not %.80s", Py_TYPE(o)->tp_name);
      throw Failed{};
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() < 1 || t.dim() > 3) {
      PyErr_SetString(PyExc_AssertionError, "device tensors of one to three dimensions only");
      throw Failed{};
    }
    v.p = t.data_ptr();
    v.dim = (int)t.dim();
    for (int i = 0; i < v.dim; ++i) {
      v.n[i] = t.size(i), v.stride[i] = t.stride(i);
      if (v.n[i] > INT32_MAX) {
        PyErr_SetString(PyExc_AssertionError, "sizes of 31 bits only");
        throw Failed{};
      }
    }
    v.count = t.numel();
    v.device = t.get_device();
    const at::ScalarType s = t.scalar_type();
    v.dtype = s == at::kFloat ? APEX_F32 : s == at::kBFloat16 ? APEX_BF16 : s == at::kHalf ? APEX_F16 : -1;
    v.is_int = s == at::kInt;
    v.is_long = s == at::kLong;
    v.contiguous = t.is_contiguous();
    return v;
  }
};

// A tensor [S,T,heads,width] on the GPU whose heads lie side by side.
struct Heads {
  void *p;
  int64_t n[4], seq, time;
  int dtype;
  bool contiguous;
  int device;
  bool fits(int64_t a, int64_t b, int64_t c, int64_t d) const { return n[0] == a && n[1] == b && n[2] == c && n[3] == d; }
};
template <>
struct From<Heads> {
  static Heads get(PyObject *o)
  {
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "a tensor is required, not %.80s", Py_TYPE(o)->tp_name);
      throw Failed{};
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    const bool fits = t.is_cuda() && t.dim() == 4;
    if (!fits || (t.size(3) > 1 && t.stride(3) != 1) || (t.size(2) > 1 && t.stride(2) != t.size(3)) || t.stride(0) < 0 || t.stride(1) < 0) {
      PyErr_SetString(PyExc_AssertionError, "device tensors [S,T,heads,width] only, the heads of a step side by side");
      throw Failed{};
    }
    Heads h{t.data_ptr(), {}, t.stride(0), t.stride(1), -1, t.is_contiguous(), (int)t.get_device()};
    for (int i = 0; i < 4; ++i) {
      h.n[i] = t.size(i);
      if (h.n[i] > INT32_MAX) {
        PyErr_SetString(PyExc_AssertionError, "sizes of 31 bits only");
        throw Failed{};
      }
    }
    const at::ScalarType s = t.scalar_type();
    h.dtype = s == at::kFloat ? APEX_F32 : s == at::kBFloat16 ? APEX_BF16 : s == at::kHalf ? APEX_F16 : -1;
    return h;
  }
};

// A fp32 state, of any dimensions; None: no address and no elements.
struct State {
  float *p = nullptr;
  int64_t count = 0;
  bool none = true;
  int device = -1;
  float *of(int64_t elements, const char *why) const
  {
    require(none || count == elements, why);
    return p;
  }
};
template <>
struct From<State> {
  static State get(PyObject *o)
  {
    State s;
    if (o == Py_None) return s;
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "a tensor is required, not %.80s", Py_TYPE(o)->tp_name);
      throw Failed{};
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kFloat || !t.is_contiguous()) {
      PyErr_SetString(PyExc_AssertionError, "states and gates: device, contiguous fp32 tensors only");
      throw Failed{};
    }
    s.p = static_cast<float *>(t.data_ptr());
    s.count = t.numel();
    s.none = false;
    s.device = t.get_device();
    return s;
  }
};

// A list or tuple of contiguous tensors of floating types on the GPU; None: none.
struct Tensors {
  std::vector<void *> p;
  std::vector<uint64_t> elements;
  std::vector<int> dtype;
  bool none = false;
  int device = -1;
};
template <>
struct From<Tensors> {
  static Tensors get(PyObject *o)
  {
    Tensors r;
    r.none = o == Py_None;
    if (r.none) return r;
    const Ref seq(PySequence_Fast(o, "a list or a tuple of tensors is required"));
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq.o);
    r.p.reserve(n), r.elements.reserve(n), r.dtype.reserve(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject *const item = PySequence_Fast_GET_ITEM(seq.o, i);
      if (!THPVariable_Check(item)) {
        PyErr_Format(PyExc_TypeError, "a tensor is required, not %.80s", Py_TYPE(item)->tp_name);
        throw Failed{};
      }
      const at::Tensor &t = THPVariable_Unpack(item);
      const at::ScalarType s = t.scalar_type();
      const int dtype = s == at::kFloat ? APEX_F32 : s == at::kBFloat16 ? APEX_BF16 : s == at::kHalf ? APEX_F16 : -1;
      if (!t.is_cuda() || !t.is_non_overlapping_and_dense() || dtype < 0 || (i && t.get_device() != r.device)) {
        PyErr_SetString(PyExc_AssertionError, "dense tensors of a floating type on one device only");
        throw Failed{};
      }
      r.device = t.get_device();
      r.p.push_back(t.data_ptr());
      r.elements.push_back((uint64_t)t.numel());
      r.dtype.push_back(dtype);
    }
    return r;
  }
};

// A workspace, and how large it is where that can be known: that of a tensor.
struct Space {
  void *p;
  size_t bytes;
  int device;
  // bytes_of(sizes): what it has to hold; sizes that the library does not take are the call's own to refuse
  template <typename F, typename... A>
  void *of(F bytes_of, A... sizes) const
  {
    size_t n = 0;
    require(!p || bytes_of(sizes..., &n) != APEX_OK || bytes >= n, "workspace: smaller than these sizes need");
    return p;
  }
};
template <>
struct From<Space> {
  static Space get(PyObject *o)
  {
    if (o == Py_None || !THPVariable_Check(o)) return Space{address(o), SIZE_MAX, -1};
    return Space{address(o), THPVariable_Unpack(o).nbytes(), (int)THPVariable_Unpack(o).get_device()};
  }
};

// The address of a contiguous fp32 array of `count` elements, or null where there is none.
float *floats(const View &v, int64_t count, const char *why)
{
  require(v.is_none() || (v.dtype == APEX_F32 && v.contiguous && v.count == count), why);
  return static_cast<float *>(v.p);
}
int32_t *ints(const View &v, int64_t count, const char *why)
{
  require(v.is_none() || (v.count == count && (count == 0 || (v.is_int && v.contiguous))), why);
  return static_cast<int32_t *>(v.p);
}

// The last argument of the verbs that take a stream.
struct Stream {
  void *h;
  operator void *() const { return h; }
};
template <>
struct From<Stream> {
  static Stream get(PyObject *o) { return Stream{stream_handle(o)}; }
};

// What the calls give back: the status, or the status and what the call reports.
template <int N>
struct Reported {
  int rc;
  uint64_t v[N];
};
PyObject *to_python(int rc) { return PyLong_FromLong(rc); }
PyObject *to_python(const Reported<1> &r) { return Py_BuildValue("iK", r.rc, (unsigned long long)r.v[0]); }
PyObject *to_python(const Reported<2> &r)
{
  return Py_BuildValue("iKK", r.rc, (unsigned long long)r.v[0], (unsigned long long)r.v[1]);
}

// Gives the interpreter's lock up, until the end of the scope: also where an exception leaves it.
struct Unlocked {
  PyThreadState *const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

template <typename R, typename... A, size_t... I>
PyObject *invoke(R (*f)(A...), PyObject *const *args, std::index_sequence<I...>)
{
  const std::tuple<A...> a{From<A>::get(args[I])...};
  const R r = [&] {
    const Unlocked unlocked;
    return f(std::get<I>(a)...);
  }();
  return to_python(r);
}

template <typename R, typename... A>
PyObject *call(R (*f)(A...), PyObject *const *args, Py_ssize_t n)
{
  if (n != (Py_ssize_t)sizeof...(A)) {
    PyErr_Format(PyExc_TypeError, "%zd arguments are expected, not %zd", (Py_ssize_t)sizeof...(A), n);
    return nullptr;
  }
  try {
    return invoke(f, args, std::index_sequence_for<A...>{});
  } catch (const Failed &) {
  } catch (const Refused &r) {
    PyErr_SetString(PyExc_AssertionError, r.why);
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// Entry points of the library, filled in by load().
#define APEX_ENTRIES(X)                                                                                             \
  X(apex_nstep_priorities) X(apex_replay_add) X(apex_replay_add_payload) X(apex_replay_add_publish)                 \
  X(apex_replay_add_payload_encoded) X(apex_replay_sample) X(apex_replay_sample_noalloc)                            \
  X(apex_replay_update_priorities) X(apex_replay_update_from_q) X(apex_replay_evict) X(apex_pipeline_fork)          \
  X(apex_pipeline_join) X(apex_pipeline_steps) X(apex_pipeline_add_begin) X(apex_pipeline_add_end) X(apex_pe_add)   \
  X(apex_pe_sample) X(apex_pe_update_priorities) X(apex_pe_evict_enqueue) X(apex_pe_add_round) X(apex_pe_sample_update) \
  X(apex_gated_scan) X(apex_gated_scan_backward) X(apex_distill_topk) X(apex_verify_draft)                          \
  X(apex_gated_scan_workspace_bytes) X(apex_verify_draft_workspace_bytes)                                           \
  X(apex_delta_rule) X(apex_delta_rule_backward) X(apex_delta_rule_workspace_bytes)                                 \
  X(apex_embedding) X(apex_embedding_backward) X(apex_embedding_backward_workspace_bytes)                           \
  X(apex_clip_gradients) X(apex_clip_gradients_workspace_bytes)
#define X(name) decltype(&::name) p_##name = nullptr;
APEX_ENTRIES(X)
#undef X

#define VERB(name, ...)                                                       \
  PyObject *name(PyObject *, PyObject *const *args, Py_ssize_t n)             \
  {                                                                           \
    return call(+__VA_ARGS__, args, n);                                       \
  }

typedef apex_replay_t *Rep;
typedef apex_pipeline_t *Pipe;
typedef apex_pe_replay_t *Pe;
typedef const float *F;
typedef const uint64_t *U64;
typedef const void *V;

VERB(nstep_priorities, [](uint32_t S, uint32_t T, uint32_t n_, uint32_t A, F qo, F qt, const int32_t *ac, F rw, F dc, float alpha,
                          float eps, uint32_t frac_bits, uint64_t slots, float *prio, float *ret, float *gacc, uint64_t *fx, Stream s) {
  return p_apex_nstep_priorities(S, T, n_, A, qo, qt, ac, rw, dc, alpha, eps, frac_bits, slots, prio, ret, gacc, fx, s);
})
VERB(add, [](Rep r, uint64_t count, V obs, V act, F ret, F gacc, F prio, Stream s) {
  Reported<1> o{0, {0}};
  o.rc = p_apex_replay_add(r, count, obs, act, ret, gacc, prio, &o.v[0], s);
  return o;
})
VERB(add_payload, [](Rep r, uint64_t count, V obs, V act, F ret, F gacc, Stream s) {
  return p_apex_replay_add_payload(r, count, obs, act, ret, gacc, s);
})
VERB(add_publish, [](Rep r, uint64_t count, F prio, Stream s) {
  Reported<1> o{0, {0}};
  o.rc = p_apex_replay_add_publish(r, count, prio, &o.v[0], s);
  return o;
})
VERB(add_payload_encoded, [](Rep r, uint64_t count, V raw, uint32_t raw_bytes, V act, F ret, F gacc, Stream s) {
  return p_apex_replay_add_payload_encoded(r, count, raw, raw_bytes, act, ret, gacc, s);
})
VERB(sample, [](Rep r, uint32_t nb, uint32_t k, float beta, U64 rnd, uint64_t *key, uint32_t *slot, float *weight, void *obs,
                void *act, float *ret, float *gacc, Stream s) {
  return p_apex_replay_sample(r, nb, k, beta, rnd, key, slot, weight, obs, act, ret, gacc, s);
})
VERB(sample_noalloc, [](Rep r, uint32_t nb, uint32_t k, float beta, U64 rnd, uint64_t *key, uint32_t *slot, float *weight,
                        void *obs, void *act, float *ret, float *gacc, Stream s) {
  return p_apex_replay_sample_noalloc(r, nb, k, beta, rnd, key, slot, weight, obs, act, ret, gacc, s);
})
VERB(update_priorities, [](Rep r, uint64_t m, U64 key, F prio, Stream s) {
  return p_apex_replay_update_priorities(r, m, key, prio, s);
})
VERB(update_from_q, [](Rep r, uint64_t m, U64 key, uint32_t A, F taken, F online, F target, float *prio_out, Stream s) {
  return p_apex_replay_update_from_q(r, m, key, A, taken, online, target, prio_out, s);
})
VERB(evict, [](Rep r, Stream s) {
  Reported<1> o{0, {0}};
  o.rc = p_apex_replay_evict(r, &o.v[0], s);
  return o;
})
VERB(pipeline_fork, [](Pipe p, Stream s) { return p_apex_pipeline_fork(p, s); })
VERB(pipeline_join, [](Pipe p, Stream s) { return p_apex_pipeline_join(p, s); })
VERB(pipeline_steps, [](Pipe p, uint32_t n_, float beta, U64 rnd, F new_prio) {
  uint32_t first = 0;
  Reported<1> o{0, {0}};
  o.rc = p_apex_pipeline_steps(p, n_, beta, rnd, new_prio, &first);
  o.v[0] = first;
  return o;
})
VERB(pipeline_add_begin, [](Pipe p, uint32_t S, uint32_t T, uint32_t n_, uint32_t A, F qo, F qt, const int32_t *ac, F rw, F dc,
                            V obs, V act, float *prio, float *ret, float *gacc) {
  return p_apex_pipeline_add_begin(p, S, T, n_, A, qo, qt, ac, rw, dc, obs, act, prio, ret, gacc);
})
VERB(pipeline_add_end, [](Pipe p, int evict_) {
  Reported<2> o{0, {0, 0}};
  o.rc = p_apex_pipeline_add_end(p, evict_, &o.v[0], &o.v[1]);
  return o;
})
VERB(pe_add, [](Pe r, uint64_t count, V obs, V act, F ret, F gacc, F prio, Stream s) {
  return p_apex_pe_add(r, count, obs, act, ret, gacc, prio, s);
})
VERB(pe_sample, [](Pe r, uint32_t nb, uint32_t k, float beta, U64 rnd, uint64_t *key, uint32_t *slot, float *weight, void *obs,
                   void *act, float *ret, float *gacc, Stream s) {
  return p_apex_pe_sample(r, nb, k, beta, rnd, key, slot, weight, obs, act, ret, gacc, s);
})
VERB(pe_update_priorities, [](Pe r, uint64_t m, U64 key, F prio, Stream s) {
  return p_apex_pe_update_priorities(r, m, key, prio, s);
})
VERB(pe_evict_enqueue, [](Pe r, uint32_t rounds, U64 rnd, Stream s) {
  Reported<1> o{0, {0}};
  o.rc = p_apex_pe_evict_enqueue(r, rounds, rnd, &o.v[0], s);
  return o;
})
VERB(pe_add_round, [](Pe r, uint32_t S, uint32_t T, uint32_t n_, uint32_t A, F qo, F qt, const int32_t *ac, F rw, F dc, V obs,
                      V act, Stream s) { return p_apex_pe_add_round(r, S, T, n_, A, qo, qt, ac, rw, dc, obs, act, s); })
VERB(pe_sample_update, [](Pe r, uint32_t k, float beta, U64 rnd, F new_prio, uint64_t *key, uint32_t *slot, float *weight,
                          void *obs, void *act, float *ret, float *gacc, Stream s) {
  return p_apex_pe_sample_update(r, k, beta, rnd, new_prio, key, slot, weight, obs, act, ret, gacc, s);
})

// The two strided arrays of a scan, and the shape that everything else of it follows.
void scan_inputs(const View &g, const View &x)
{
  require(g.p && x.p && g.dim == 3 && x.fits(g.n[0], g.n[1], g.n[2]) && g.dtype >= 0 && x.dtype == g.dtype,
          "g and x: [S,T,D] of one floating type");
  require(g.rows() && x.rows(), "g and x: contiguous channels");
}

VERB(gated_scan, [](View g, View x, int gate, View discount, View length, View h0, View h, View h_last, View carry, Space workspace, Stream s) {
  scan_inputs(g, x);
  const int64_t S = g.n[0], T = g.n[1], D = g.n[2], chunks = (T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  require(h.p && h.fits(S, T, D) && h.contiguous && h.dtype == g.dtype, "h: [S,T,D], contiguous, of g's type");
  return p_apex_gated_scan(S, T, D, g.dtype, gate, g.p, g.stride[0], g.stride[1], x.p, x.stride[0], x.stride[1],
                           floats(discount, S * T, "discount: fp32 [S,T]"), ints(length, S, "length: int32 [S]"),
                           floats(h0, S * D, "h0: fp32 [S,D]"), h.p, floats(h_last, S * D, "h_last: fp32 [S,D]"),
                           floats(carry, S * chunks * D, "carry: fp32 [S,chunks,D]"),
                           workspace.of(p_apex_gated_scan_workspace_bytes, S, T, D), s);
})
VERB(gated_scan_backward, [](View g, View x, int gate, View discount, View length, View carry, View dh, View dh_last, View dg, View dx,
                             View dh0, Space workspace, Stream s) {
  scan_inputs(g, x);
  const int64_t S = g.n[0], T = g.n[1], D = g.n[2], chunks = (T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  require(dh.p && dh.fits(S, T, D) && dh.contiguous && dh.dtype == g.dtype, "dh: [S,T,D], contiguous, of g's type");
  const auto gradient = [&](const View &v) { return v.p && v.fits(S, T, D) && v.dtype == g.dtype && v.rows(); };
  require(gradient(dg) && gradient(dx), "dg and dx: [S,T,D] of g's type, contiguous channels");
  return p_apex_gated_scan_backward(S, T, D, g.dtype, gate, g.p, g.stride[0], g.stride[1], x.p, x.stride[0], x.stride[1],
                                    floats(discount, S * T, "discount: fp32 [S,T]"), ints(length, S, "length: int32 [S]"),
                                    floats(carry, S * chunks * D, "carry: fp32 [S,chunks,D]"), dh.p,
                                    floats(dh_last, S * D, "dh_last: fp32 [S,D]"), dg.p, dg.stride[0], dg.stride[1], dx.p,
                                    dx.stride[0], dx.stride[1], floats(dh0, S * D, "dh0: fp32 [S,D]"),
                                    workspace.of(p_apex_gated_scan_workspace_bytes, S, T, D), s);
})
VERB(distill_topk, [](View logits, View index, View value, View top_lse, View weight, float temperature, View loss, View lse, View grad,
                      V workspace, Stream s) {
  require(logits.p && logits.dim == 2 && logits.dtype >= 0 && logits.rows(), "logits: [N,V] of a floating type, contiguous rows");
  const int64_t N = logits.n[0], vocabulary = logits.n[1];
  require(index.p && index.dim == 2 && index.n[0] == N, "top_index: int32 [N,K]");
  const int64_t K = index.n[1];
  require(value.p && value.fits(N, K) && value.contiguous && value.dtype >= 0, "top_value: [N,K] of a floating type");
  require(grad.is_none() || (grad.fits(N, vocabulary) && grad.dtype == logits.dtype && grad.rows()), "grad: [N,V] of the logits' type");
  return p_apex_distill_topk(N, vocabulary, K, logits.dtype, logits.p, logits.stride[0], ints(index, N * K, "top_index: int32 [N,K]"),
                             value.dtype, value.p, floats(top_lse, N, "top_lse: fp32 [N]"), floats(weight, N, "weight: fp32 [N]"),
                             temperature, floats(loss, N, "loss: fp32 [N]"), floats(lse, N, "lse: fp32 [N]"), grad.p, grad.stride[0],
                             const_cast<void *>(workspace), s);
})
VERB(verify_draft, [](View target, View draft, View token, View rnd, View length, View accepted, View token_out, Space workspace, Stream s) {
  require(target.p && target.dim == 3 && target.dtype >= 0 && target.rows() && target.n[1] > 0,
          "target: [B,G+1,V] of a floating type, contiguous rows");
  const int64_t B = target.n[0], G = target.n[1] - 1, vocabulary = target.n[2];
  require(!G || (draft.p && draft.fits(B, G, vocabulary) && draft.dtype == target.dtype && draft.rows()),
          "draft: [B,G,V] of the target's type, contiguous rows");
  require(rnd.is_long && rnd.contiguous && rnd.count == B * (G + 1), "rnd: int64 [B,G+1]");
  return p_apex_verify_draft(B, G, vocabulary, target.dtype, target.p, target.stride[0], target.stride[1], draft.p, draft.stride[0],
                             draft.stride[1], ints(token, B * G, "token: int32 [B,G]"), static_cast<const uint64_t *>(rnd.p),
                             ints(length, B, "length: int32 [B]"), ints(accepted, B, "accepted: int32 [B]"),
                             ints(token_out, B * (G + 1), "token_out: int32 [B,G+1]"),
                             workspace.of(p_apex_verify_draft_workspace_bytes, B, vocabulary), s);
})

// Tensors of one call are on one device (-1: there is none).
template <typename... A>
void on_one_device(const A &...a)
{
  int first = -1;
  const auto same = [&](int device) {
    if (first < 0) first = device;
    return device < 0 || device == first;
  };
  bool all = true;
  ((all = same(a.device) && all), ...);
  require(all, "tensors of one device only");
}

struct DeltaSizes {
  int64_t S, T, Hk, H, Dk, Dv, state, slices, gates;
  DeltaSizes(const Heads &q, const Heads &k, const Heads &v)
      : S(q.n[0]), T(q.n[1]), Hk(q.n[2]), H(v.n[2]), Dk(q.n[3]), Dv(v.n[3]), state(S * H * Dk * Dv), slices(S * H * ((Dk + 31) / 32 * 32) * ((Dv + 15) / 16 * 16)), gates(S * T * H)
  {
    require(q.dtype >= 0 && k.dtype == q.dtype && v.dtype == q.dtype, "q, k and v: of one floating type");
    require(k.fits(S, T, Hk, Dk) && v.n[0] == S && v.n[1] == T, "q and k: [S,T,Hk,Dk], v: [S,T,H,Dv]");
  }
};

VERB(delta_rule, [](Heads q, Heads k, Heads v, State g, State beta, float scale, View discount, View length, State h0, Heads o, State h_last,
                    State carry, Space workspace, Stream s) {
  const DeltaSizes n(q, k, v);
  on_one_device(q, k, v, g, beta, discount, length, h0, o, h_last, carry, workspace);
  require(o.dtype == q.dtype && o.fits(n.S, n.T, n.H, n.Dv) && o.contiguous, "o: [S,T,H,Dv], contiguous, of q's type");
  require(!g.none && !beta.none, "g and beta: fp32 [S,T,H]");
  const int64_t chunks = (n.T + APEX_DELTA_CHUNK - 1) / APEX_DELTA_CHUNK;
  return p_apex_delta_rule(n.S, n.T, n.Hk, n.H, n.Dk, n.Dv, q.dtype, q.p, q.seq, q.time, k.p, k.seq, k.time, v.p, v.seq, v.time,
                           g.of(n.gates, "g: fp32 [S,T,H]"), beta.of(n.gates, "beta: fp32 [S,T,H]"), scale,
                           floats(discount, n.S * n.T, "discount: fp32 [S,T]"), ints(length, n.S, "length: int32 [S]"),
                           h0.of(n.state, "h0: fp32 [S,H,Dk,Dv]"), o.p, h_last.of(n.state, "h_last: fp32 [S,H,Dk,Dv]"),
                           carry.of(chunks * n.slices, "carry: fp32, of delta_rule_carry_shape"),
                           workspace.of(p_apex_delta_rule_workspace_bytes, n.S, n.T, n.H, n.Dk, n.Dv, 0), s);
})
VERB(delta_rule_backward, [](Heads q, Heads k, Heads v, State g, State beta, float scale, View discount, View length, State carry, Heads d_o,
                             State dh_last, Heads dq, Heads dk, Heads dv, State dg, State dbeta, State dh0, Space workspace, Stream s) {
  const DeltaSizes n(q, k, v);
  on_one_device(q, k, v, g, beta, discount, length, carry, d_o, dh_last, dq, dk, dv, dg, dbeta, dh0, workspace);
  require(d_o.dtype == q.dtype && d_o.fits(n.S, n.T, n.H, n.Dv) && d_o.contiguous, "do: [S,T,H,Dv], contiguous, of q's type");
  require(dq.dtype == q.dtype && dk.dtype == q.dtype && dv.dtype == q.dtype && dq.fits(n.S, n.T, n.Hk, n.Dk) &&
              dk.fits(n.S, n.T, n.Hk, n.Dk) && dv.fits(n.S, n.T, n.H, n.Dv), "dq, dk and dv: as q, k and v");
  require(!g.none && !beta.none && !carry.none && !dg.none && !dbeta.none, "g, beta, dg, dbeta: fp32 [S,T,H], and a carry");
  const int64_t chunks = (n.T + APEX_DELTA_CHUNK - 1) / APEX_DELTA_CHUNK;
  return p_apex_delta_rule_backward(n.S, n.T, n.Hk, n.H, n.Dk, n.Dv, q.dtype, q.p, q.seq, q.time, k.p, k.seq, k.time, v.p, v.seq, v.time,
                                    g.of(n.gates, "g: fp32 [S,T,H]"), beta.of(n.gates, "beta: fp32 [S,T,H]"), scale,
                                    floats(discount, n.S * n.T, "discount: fp32 [S,T]"), ints(length, n.S, "length: int32 [S]"),
                                    carry.of(chunks * n.slices, "carry: fp32, of delta_rule_carry_shape"), d_o.p,
                                    dh_last.of(n.state, "dh_last: fp32 [S,H,Dk,Dv]"), dq.p, dq.seq, dq.time, dk.p, dk.seq, dk.time, dv.p,
                                    dv.seq, dv.time, dg.of(n.gates, "dg: fp32 [S,T,H]"), dbeta.of(n.gates, "dbeta: fp32 [S,T,H]"),
                                    dh0.of(n.state, "dh0: fp32 [S,H,Dk,Dv]"),
                                    workspace.of(p_apex_delta_rule_workspace_bytes, n.S, n.T, n.H, n.Dk, n.Dv, 1), s);
})
VERB(embedding, [](View table, View token, float scale, View out, Stream s) {
  on_one_device(table, token, out);
  require(table.dim == 2 && table.dtype >= 0 && table.rows(), "table: [V,D] of a floating type, contiguous rows");
  require(!token.is_none() && out.fits(token.count, table.n[1]) && out.dtype == table.dtype && out.rows(),
          "out: [N,D] of the table's type, contiguous rows");
  return p_apex_embedding(token.count, table.n[0], table.n[1], table.dtype, table.p, table.stride[0], ints(token, token.count, "token: int32"),
                          scale, out.p, out.stride[0], s);
})
VERB(embedding_backward, [](View dout, View token, float scale, int add, View dtable, Space workspace, Stream s) {
  on_one_device(dout, token, dtable, workspace);
  require(dtable.dim == 2 && dtable.dtype >= 0 && dtable.rows(), "dtable: [V,D] of a floating type, contiguous rows");
  require(!token.is_none() && dout.fits(token.count, dtable.n[1]) && dout.dtype == dtable.dtype && dout.rows(),
          "dout: [N,D] of the table's type, contiguous rows");
  return p_apex_embedding_backward(token.count, dtable.n[0], dtable.n[1], dout.dtype, dout.p, dout.stride[0],
                                   ints(token, token.count, "token: int32"), scale, add, dtable.p, dtable.stride[0],
                                   workspace.of(p_apex_embedding_backward_workspace_bytes, token.count, dtable.n[0], dtable.n[1]), s);
})
VERB(clip_gradients, [](Tensors grad, Tensors out, float max_norm, View norm, Space workspace, Stream s) {
  on_one_device(grad, out, norm, workspace);
  require(!grad.none && (out.none || (out.elements == grad.elements && out.dtype == grad.dtype)), "out: as the gradients");
  return p_apex_clip_gradients(grad.p.size(), grad.p.data(), out.none ? nullptr : out.p.data(), grad.elements.data(), grad.dtype.data(),
                               max_norm, floats(norm, 1, "norm: fp32 [1]"), workspace.of(p_apex_clip_gradients_workspace_bytes, grad.p.size()), s);
})

// load(path of the library, _ptr, _plain, current device, current raw stream)
PyObject *load(PyObject *, PyObject *args)
{
  const char *path;
  PyObject *address_of, *plain, *device, *stream;
  if (!PyArg_ParseTuple(args, "sOOOO", &path, &address_of, &plain, &device, &stream)) return nullptr;
  void *const lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (!lib) return PyErr_Format(PyExc_ImportError, "%s", dlerror());
#define X(name)                                                            \
  p_##name = reinterpret_cast<decltype(&::name)>(dlsym(lib, #name));       \
  if (!p_##name) return PyErr_Format(PyExc_ImportError, "%s lacks %s", path, #name);
  APEX_ENTRIES(X)
#undef X
  Py_INCREF(address_of), Py_INCREF(plain), Py_INCREF(device), Py_INCREF(stream);
  Py_XSETREF(g_address, address_of);
  Py_XSETREF(g_plain, plain);
  Py_XSETREF(g_current_device, device);
  Py_XSETREF(g_current_stream, stream);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"load", load, METH_VARARGS, nullptr},
    FAST(nstep_priorities), FAST(add), FAST(add_payload), FAST(add_publish), FAST(add_payload_encoded), FAST(sample),
    FAST(sample_noalloc), FAST(update_priorities), FAST(update_from_q), FAST(evict), FAST(pipeline_fork), FAST(pipeline_join),
    FAST(pipeline_steps), FAST(pipeline_add_begin), FAST(pipeline_add_end), FAST(pe_add), FAST(pe_sample),
    FAST(pe_update_priorities), FAST(pe_evict_enqueue), FAST(pe_add_round), FAST(pe_sample_update),
    FAST(gated_scan), FAST(gated_scan_backward), FAST(distill_topk), FAST(verify_draft),
    FAST(delta_rule), FAST(delta_rule_backward), FAST(embedding), FAST(embedding_backward), FAST(clip_gradients),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "apex_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_apex_binding(void) { return PyModule_Create(&module); }
