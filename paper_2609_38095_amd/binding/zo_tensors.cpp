// Marshalling of torch tensors into the argument structs of zo_decode.h, as a Python module (_tensors).
//
// A decode step's calls take less time on the GPU than ten tensors' shapes, strides and addresses take to
// read from Python (11 us of a 14 us call); here they take about one. Nothing is computed: each function checks
// its tensors, allocates results that were not given, fills one struct and calls the library, whose entry
// points decode.py hands over by address. Returned are the results, or the library's status if it is not ZO_OK.

#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "zo_decode.h"

namespace {

struct Entry {
  decltype(&zo_norm_rotate) norm_rotate;
  decltype(&zo_norm_rotate_put) norm_rotate_put;
  decltype(&zo_norm_rotate_back) norm_rotate_back;
  decltype(&zo_norm_rotate_back_work) norm_rotate_back_work;
  decltype(&zo_cache_attend) cache_attend;
  decltype(&zo_cache_attend_work) cache_attend_work;
  decltype(&zo_cache_copy) cache_copy;
  decltype(&zo_draw_split) draw_split;
  decltype(&zo_draw_work) draw_work;
} entry = {};

struct Refusal {  // a Python exception to raise
  PyObject* type;
  std::string what;
};

[[noreturn]] void refuse(PyObject* type, const char* format, ...) {
  char text[256];
  va_list args;
  va_start(args, format);
  std::vsnprintf(text, sizeof text, format, args);
  va_end(args);
  throw Refusal{type, text};
}

// The positional arguments of a call; every function begins with the current device and the stream.
struct Args {
  PyObject* const* at;
  Py_ssize_t left;
  int device;
  void* stream;

  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t wanted) : at(args), left(n) {
    if (n != wanted) refuse(PyExc_TypeError, "%zd arguments, not %zd", wanted, n);
    device = static_cast<int>(integer());
    stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer()));
  }
  PyObject* next() { return *at++; }
  long long integer() {
    const long long v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
  }
  double number() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
  }
  bool flag() {
    const int v = PyObject_IsTrue(next());
    if (v < 0) throw python_error();
    return v != 0;
  }
  // A tensor on the current device; nullptr for None.
  const at::Tensor* tensor(const char* name) {
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a CUDA (HIP) torch tensor", name);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) refuse(PyExc_TypeError, "%s must be a CUDA (HIP) torch tensor", name);
    if (t.get_device() != device)
      refuse(PyExc_ValueError, "%s lives on cuda:%d, the current device is cuda:%d", name, static_cast<int>(t.get_device()), device);
    return &t;
  }
};

int32_t type_of(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kFloat) return ZO_F32;
  if (t.scalar_type() == at::kBFloat16) return ZO_BF16;
  refuse(PyExc_TypeError, "%s must be a float32 or bfloat16 tensor", name);
}

void check_type(const at::Tensor& t, const char* name, at::ScalarType type) {
  if (t.scalar_type() != type) refuse(PyExc_TypeError, "%s must be %s, not %s", name, at::toString(type), at::toString(t.scalar_type()));
}

zo_heads rows(const at::Tensor* t, const char* name, at::ScalarType type, int64_t tokens, int64_t heads, int64_t dim) {
  if (t == nullptr) refuse(PyExc_TypeError, "%s is needed", name);
  check_type(*t, name, type);
  if (t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != dim)
    refuse(PyExc_ValueError, "%s must be [%lld, %lld, %lld]", name, static_cast<long long>(tokens), static_cast<long long>(heads),
           static_cast<long long>(dim));
  if (t->stride(2) != 1 && dim > 1) refuse(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
  return zo_heads{t->data_ptr(), t->stride(0), t->stride(1)};
}

// A contiguous tensor of n elements; nullptr for None.
template <class T>
T* vector_of(const at::Tensor* t, const char* name, at::ScalarType type, int64_t n) {
  if (t == nullptr) return nullptr;
  check_type(*t, name, type);
  if (t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
    refuse(PyExc_ValueError, "%s must be contiguous and hold %lld elements", name, static_cast<long long>(n));
  return static_cast<T*>(t->data_ptr());
}

uint32_t count_of(int64_t n, const char* name) {
  if (n > 0xFFFFFFFFll) refuse(PyExc_ValueError, "%s has too many entries", name);
  return static_cast<uint32_t>(n);
}

// The same sizes, and the same strides wherever there is more than one entry.
bool same_layout(const at::Tensor& a, const at::Tensor& b) {
  if (a.sizes() != b.sizes()) return false;
  for (int64_t i = 0; i < a.dim(); ++i)
    if (a.size(i) > 1 && a.stride(i) != b.stride(i)) return false;
  return true;
}

zo_cache cache_of(const at::Tensor* k, const at::Tensor* v, at::ScalarType type) {
  if (k == nullptr || v == nullptr) refuse(PyExc_TypeError, "k_cache and v_cache are needed");
  check_type(*k, "k_cache", type);
  check_type(*v, "v_cache", type);
  if (k->dim() != 4) refuse(PyExc_ValueError, "k_cache must be [pages, heads, page_tokens, dim]");
  if (!same_layout(*k, *v))
    refuse(PyExc_ValueError, "k_cache and v_cache must have the same shape and strides");
  if (k->stride(3) != 1 && k->size(3) > 1) refuse(PyExc_ValueError, "the last dimension of the cache must be contiguous");
  return zo_cache{k->data_ptr(), v->data_ptr(), k->stride(0), k->stride(1), k->stride(2), count_of(k->size(0), "k_cache"),
                  count_of(k->size(1), "k_cache"), count_of(k->size(2), "k_cache"), count_of(k->size(3), "k_cache")};
}

zo_page_table table_of(const at::Tensor* t) {
  if (t == nullptr) refuse(PyExc_TypeError, "table is needed");
  check_type(*t, "table", at::kInt);
  if (t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1))
    refuse(PyExc_ValueError, "table must be [sequences, pages], its rows contiguous");
  return zo_page_table{static_cast<const int32_t*>(t->data_ptr()), t->stride(0), count_of(t->size(0), "table"), count_of(t->size(1), "table")};
}

// A host buffer of one dimension, held during the call; None: no elements.
struct Host {
  Py_buffer view = {};
  bool held = false;
  Host(PyObject* o, const char* name, const char* format) {
    if (o == Py_None) return;
    if (PyObject_GetBuffer(o, &view, PyBUF_CONTIG_RO | PyBUF_FORMAT) != 0) throw python_error();
    held = true;
    if (view.ndim != 1 || view.format == nullptr || std::strcmp(view.format, format) != 0) {
      PyBuffer_Release(&view);
      refuse(PyExc_TypeError, "%s must be a contiguous array of one dimension and of type '%s'", name, format);
    }
  }
  ~Host() {
    if (held) PyBuffer_Release(&view);
  }
  Py_ssize_t count() const { return held ? view.shape[0] : 0; }
  const void* data() const { return view.buf; }
};

at::Tensor fresh(const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type) { return at::empty(shape, like.options().dtype(type)); }

PyObject* status(int rc) { return PyLong_FromLong(rc); }

PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

PyObject* tuple_of(std::initializer_list<at::Tensor> tensors) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
  if (r == nullptr) throw python_error();
  Py_ssize_t i = 0;
  for (const at::Tensor& t : tensors) {
    PyObject* o = wrap_or_none(t);
    if (o == nullptr) {
      Py_DECREF(r);
      throw python_error();
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// What the rotations' calls share: q and k (of which one may be None) and their sizes.
struct Sides {
  const at::Tensor *q, *k, *like;
  at::ScalarType type;
  int64_t tokens, dim, q_heads, k_heads;
  Sides(const at::Tensor* q_in, const at::Tensor* k_in) : q(q_in), k(k_in), like(q_in ? q_in : k_in) {
    if (like == nullptr) refuse(PyExc_ValueError, "queries or keys are needed");
    if (like->dim() != 3 || (k && k->dim() != 3)) refuse(PyExc_ValueError, "q and k must be [tokens, heads, dim]");
    type = like->scalar_type();
    tokens = like->size(0);
    dim = like->size(2);
    q_heads = q ? q->size(1) : 0;
    k_heads = k ? k->size(1) : 0;
  }
};

// positions, turns, interleaved, magnitude, q_gamma, k_gamma, norm_eps
struct Rule {
  const at::Tensor* positions;
  Host turns;
  bool interleaved;
  double magnitude;
  const at::Tensor *q_gamma, *k_gamma;
  double eps;
  explicit Rule(Args& a)
      : positions(a.tensor("positions")), turns(a.next(), "turns", "d"), interleaved(a.flag()), magnitude(a.number()),
        q_gamma(a.tensor("q_gamma")), k_gamma(a.tensor("k_gamma")), eps(a.number()) {}
  void fill(zo_rotate& r, const Sides& s) const {
    r.q_gamma = vector_of<void>(q_gamma, "q_gamma", s.type, s.dim);
    r.k_gamma = vector_of<void>(k_gamma, "k_gamma", s.type, s.dim);
    r.positions = vector_of<const int32_t>(positions, "positions", at::kInt, s.tokens);
    r.turns = static_cast<const double*>(turns.data());
    r.tokens = count_of(s.tokens, "q");
    r.q_heads = count_of(s.q_heads, "q");
    r.k_heads = count_of(s.k_heads, "k");
    r.dim = count_of(s.dim, "q");
    r.rotary = 2 * count_of(turns.count(), "turns");
    r.interleaved = interleaved;
    r.norm_eps = static_cast<float>(eps);
    r.magnitude = static_cast<float>(magnitude);
    r.dtype = type_of(*s.like, "q and k");
  }
};

PyObject* norm_rotate(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 13);
  const at::Tensor *q = a.tensor("q"), *k = a.tensor("k");
  const Sides s(q, k);
  const Rule rule(a);
  const at::Tensor *q_given = a.tensor("q_out"), *k_given = a.tensor("k_out");
  zo_rotate r = {};
  rule.fill(r, s);
  at::Tensor q_out, k_out;
  if (q) {
    r.q = rows(q, "q", s.type, s.tokens, s.q_heads, s.dim);
    q_out = q_given ? *q_given : fresh(*q, {s.tokens, s.q_heads, s.dim}, s.type);
    r.q_out = rows(&q_out, "q_out", s.type, s.tokens, s.q_heads, s.dim);
  }
  if (k) {
    r.k = rows(k, "k", s.type, s.tokens, s.k_heads, s.dim);
    k_out = k_given ? *k_given : fresh(*k, {s.tokens, s.k_heads, s.dim}, s.type);
    r.k_out = rows(&k_out, "k_out", s.type, s.tokens, s.k_heads, s.dim);
  }
  const int rc = entry.norm_rotate(&r, a.stream);
  return rc == ZO_OK ? tuple_of({q_out, k_out}) : status(rc);
}

PyObject* norm_rotate_put(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 17);
  const at::Tensor *q = a.tensor("q"), *k = a.tensor("k"), *v = a.tensor("v");
  const at::Tensor *k_cache = a.tensor("k_cache"), *v_cache = a.tensor("v_cache"), *table = a.tensor("table");
  const Sides s(q, k);
  const Rule rule(a);
  const at::Tensor *seqs = a.tensor("seqs"), *q_given = a.tensor("q_out");
  zo_rotate_put p = {};
  rule.fill(p.a, s);
  at::Tensor q_out;
  if (q) {
    p.a.q = rows(q, "q", s.type, s.tokens, s.q_heads, s.dim);
    q_out = q_given ? *q_given : fresh(*q, {s.tokens, s.q_heads, s.dim}, s.type);
    p.a.q_out = rows(&q_out, "q_out", s.type, s.tokens, s.q_heads, s.dim);
  }
  p.a.k = rows(k, "k", s.type, s.tokens, s.k_heads, s.dim);
  p.v = rows(v, "v", s.type, s.tokens, s.k_heads, s.dim);
  p.cache = cache_of(k_cache, v_cache, s.type);
  p.table = table_of(table);
  p.seqs = vector_of<const int32_t>(seqs, "seqs", at::kInt, s.tokens);
  const int rc = entry.norm_rotate_put(&p, a.stream);
  return rc == ZO_OK ? wrap_or_none(q_out) : status(rc);
}

// (address, bytes) of a workspace, allocated if none is given.
void work_of(const at::Tensor* given, const at::Tensor& like, uint64_t bytes, at::Tensor& hold, void*& at, uint64_t& size) {
  if (given == nullptr) {
    hold = fresh(like, {static_cast<int64_t>(bytes < 16 ? 16 : bytes)}, at::kByte);
    given = &hold;
  }
  if (!given->is_contiguous()) refuse(PyExc_ValueError, "work must be contiguous");
  at = given->data_ptr();
  size = given->nbytes();
}

PyObject* norm_rotate_back(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 16);
  const at::Tensor *dq_out = a.tensor("dq_out"), *dk_out = a.tensor("dk_out"), *q = a.tensor("q"), *k = a.tensor("k");
  const Sides s(dq_out, dk_out);
  const Rule rule(a);
  const at::Tensor *dq_given = a.tensor("dq"), *dk_given = a.tensor("dk"), *work = a.tensor("work");
  zo_rotate_back b = {};
  rule.fill(b.a, s);
  at::Tensor dq, dk, dq_gamma, dk_gamma, hold;
  const auto side = [&](const at::Tensor* dy, const at::Tensor* x, const at::Tensor* gamma, const at::Tensor* given, int64_t heads,
                        const char* dy_name, const char* x_name, const char* dx_name, zo_heads& dy_rows, zo_heads& x_rows, zo_heads& dx_rows,
                        at::Tensor& dx, at::Tensor& dgamma, float*& dgamma_at) {
    if (dy == nullptr) return;
    dy_rows = rows(dy, dy_name, s.type, s.tokens, heads, s.dim);
    dx = given ? *given : fresh(*dy, {s.tokens, heads, s.dim}, s.type);
    dx_rows = rows(&dx, dx_name, s.type, s.tokens, heads, s.dim);
    if (gamma == nullptr) return;
    x_rows = rows(x, x_name, s.type, s.tokens, heads, s.dim);
    dgamma = fresh(*dy, {s.dim}, at::kFloat);
    dgamma_at = static_cast<float*>(dgamma.data_ptr());
  };
  side(dq_out, q, rule.q_gamma, dq_given, s.q_heads, "dq_out", "q", "dq", b.a.q_out, b.a.q, b.dq, dq, dq_gamma, b.dq_gamma);
  side(dk_out, k, rule.k_gamma, dk_given, s.k_heads, "dk_out", "k", "dk", b.a.k_out, b.a.k, b.dk, dk, dk_gamma, b.dk_gamma);
  if (dq_gamma.defined() || dk_gamma.defined())
    work_of(work, *s.like, entry.norm_rotate_back_work(b.a.tokens, b.a.q_heads, b.a.k_heads, b.a.dim), hold, b.work, b.work_bytes);
  const int rc = entry.norm_rotate_back(&b, a.stream);
  return rc == ZO_OK ? tuple_of({dq, dk, dq_gamma, dk_gamma}) : status(rc);
}

PyObject* cache_attend(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 11);
  const at::Tensor *q = a.tensor("q"), *k_cache = a.tensor("k_cache"), *v_cache = a.tensor("v_cache"), *table = a.tensor("table");
  const at::Tensor* lengths = a.tensor("lengths");
  PyObject* scale = a.next();
  const at::Tensor* out_given = a.tensor("out");
  const bool lse = a.flag();
  const at::Tensor* work = a.tensor("work");
  if (q == nullptr) refuse(PyExc_TypeError, "q must be a CUDA (HIP) torch tensor");
  zo_attend p = {};
  p.dtype = type_of(*q, "q");
  if (q->dim() != 3) refuse(PyExc_ValueError, "q must be [sequences, heads, dim]");
  const int64_t seqs = q->size(0), heads = q->size(1), dim = q->size(2);
  p.q = rows(q, "q", q->scalar_type(), seqs, heads, dim);
  p.cache = cache_of(k_cache, v_cache, q->scalar_type());
  if (p.cache.dim != dim)
    refuse(PyExc_ValueError, "the cache's heads hold %u dims, the queries' %lld", p.cache.dim, static_cast<long long>(dim));
  p.table = table_of(table);
  if (p.table.seqs != seqs) refuse(PyExc_ValueError, "the table has one row for each sequence");
  if (lengths == nullptr) refuse(PyExc_TypeError, "lengths is needed");
  p.lengths = vector_of<const int32_t>(lengths, "lengths", at::kInt, seqs);
  p.q_heads = count_of(heads, "q");
  if (scale == Py_None) {
    p.scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(dim)));
  } else {
    const double v = PyFloat_AsDouble(scale);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    p.scale = static_cast<float>(v);
  }
  at::Tensor sums, hold;
  const at::Tensor out = out_given ? *out_given : fresh(*q, {seqs, heads, dim}, q->scalar_type());
  p.out = rows(&out, "out", q->scalar_type(), seqs, heads, dim);
  if (lse) {
    sums = fresh(*q, {seqs, heads}, at::kFloat);
    p.lse = static_cast<float*>(sums.data_ptr());
  }
  work_of(work, *q, entry.cache_attend_work(p.table.seqs, p.q_heads, p.cache.heads, p.cache.dim), hold, p.work, p.work_bytes);
  const int rc = entry.cache_attend(&p, a.stream);
  if (rc != ZO_OK) return status(rc);
  return lse ? tuple_of({out, sums}) : THPVariable_Wrap(out);
}

PyObject* cache_copy(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 7);
  PyObject* lists[2] = {a.next(), a.next()};
  const Host src(a.next(), "src", "i"), dst(a.next(), "dst", "i"), rows_in(a.next(), "rows", "i");
  if (!PyList_Check(lists[0]) || !PyList_Check(lists[1]) || PyList_GET_SIZE(lists[0]) != PyList_GET_SIZE(lists[1]))
    refuse(PyExc_ValueError, "one v_cache for each k_cache");
  const Py_ssize_t layers = PyList_GET_SIZE(lists[0]);
  if (layers == 0) Py_RETURN_NONE;
  if (src.count() != dst.count() || (rows_in.held && rows_in.count() != src.count()))
    refuse(PyExc_ValueError, "one dst, and one count of rows, for each src");
  std::vector<void*> tensors;
  tensors.reserve(2 * layers);
  const at::Tensor* first = nullptr;
  zo_cache shape = {};
  int32_t dtype = 0;
  for (PyObject* list : lists) {
    for (Py_ssize_t i = 0; i < layers; ++i) {
      PyObject* o = PyList_GET_ITEM(list, i);
      Args one = a;
      one.at = &o;
      const at::Tensor* t = one.tensor("each cache");
      if (first == nullptr) {
        if (t == nullptr) refuse(PyExc_TypeError, "each cache must be a CUDA (HIP) torch tensor");
        first = t;
        dtype = type_of(*t, "each cache");
        shape = cache_of(t, t, t->scalar_type());
      }
      if (t == nullptr || t->scalar_type() != first->scalar_type() || !same_layout(*t, *first))
        refuse(PyExc_ValueError, "each cache must have the type, shape and strides of the first");
      tensors.push_back(t->data_ptr());
    }
  }
  std::vector<zo_page_move> moves(src.count());
  for (size_t i = 0; i < moves.size(); ++i)
    moves[i] = zo_page_move{static_cast<const int32_t*>(src.data())[i], static_cast<const int32_t*>(dst.data())[i],
                            rows_in.held ? static_cast<const int32_t*>(rows_in.data())[i] : static_cast<int32_t>(shape.page_tokens)};
  const int rc = entry.cache_copy(&shape, tensors.data(), static_cast<uint32_t>(tensors.size()), moves.data(),
                                  static_cast<uint32_t>(moves.size()), static_cast<zo_dtype>(dtype), a.stream);
  if (rc != ZO_OK) return status(rc);
  Py_RETURN_NONE;
}

PyObject* draw(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 11);
  const at::Tensor* logits = a.tensor("logits");
  const at::Tensor *u = a.tensor("u"), *temperature = a.tensor("temperature"), *top_k = a.tensor("top_k"), *top_p = a.tensor("top_p");
  const at::Tensor* min_p = a.tensor("min_p");
  const bool logprobs = a.flag();
  const at::Tensor *given = a.tensor("tokens"), *work = a.tensor("work");
  if (logits == nullptr || u == nullptr) refuse(PyExc_TypeError, "logits and u must be CUDA (HIP) torch tensors");
  zo_draw_args p = {};
  p.dtype = type_of(*logits, "logits");
  if (logits->dim() != 2 || (logits->size(1) > 1 && logits->stride(1) != 1))
    refuse(PyExc_ValueError, "logits must be [rows, vocab], its rows contiguous");
  const int64_t count = logits->size(0);
  p.logits = logits->data_ptr();
  p.row_stride = logits->stride(0);
  p.rows = count_of(count, "logits");
  p.vocab = count_of(logits->size(1), "logits");
  p.u = vector_of<const float>(u, "u", at::kFloat, count);
  p.temperature = vector_of<const float>(temperature, "temperature", at::kFloat, count);
  p.top_k = vector_of<const int32_t>(top_k, "top_k", at::kInt, count);
  p.top_p = vector_of<const float>(top_p, "top_p", at::kFloat, count);
  p.min_p = vector_of<const float>(min_p, "min_p", at::kFloat, count);
  const at::Tensor tokens = given ? *given : fresh(*logits, {count}, at::kInt);
  p.tokens = vector_of<int32_t>(&tokens, "tokens", at::kInt, count);
  at::Tensor probs;
  if (logprobs) {
    probs = fresh(*logits, {count}, at::kFloat);
    p.logprobs = static_cast<float*>(probs.data_ptr());
  }
  at::Tensor hold;
  void* at = nullptr;
  uint64_t bytes = 0;
  if (const uint64_t needed = entry.draw_work(p.rows, p.vocab, p.top_k != nullptr)) work_of(work, *logits, needed, hold, at, bytes);
  const int rc = entry.draw_split(&p, at, bytes, a.stream);
  if (rc != ZO_OK) return status(rc);
  return logprobs ? tuple_of({tokens, probs}) : THPVariable_Wrap(tokens);
}

// bind(addresses of the library's entry points, in Entry's order)
PyObject* bind(PyObject* const* args, Py_ssize_t n) {
  if (n != static_cast<Py_ssize_t>(sizeof(Entry) / sizeof(void*))) refuse(PyExc_TypeError, "an address for each entry point");
  void* at[sizeof(Entry) / sizeof(void*)];
  for (Py_ssize_t i = 0; i < n; ++i) {
    at[i] = PyLong_AsVoidPtr(args[i]);
    if (at[i] == nullptr) refuse(PyExc_ValueError, "an address for each entry point");
  }
  std::memcpy(&entry, at, sizeof entry);
  Py_RETURN_NONE;
}

// Refusals, Python's and torch's errors become Python exceptions; nothing else leaves.
template <PyObject* (*kCall)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    return kCall(args, n);
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.what.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*kCall)(PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<kCall>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"), method<norm_rotate>("norm_rotate"), method<norm_rotate_put>("norm_rotate_put"),
                         method<norm_rotate_back>("norm_rotate_back"), method<cache_attend>("cache_attend"),
                         method<cache_copy>("cache_copy"), method<draw>("draw"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
