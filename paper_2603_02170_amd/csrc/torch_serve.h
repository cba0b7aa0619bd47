// The part of torch_host.cpp for the operators of sagebwd_serve.h (included there, inside its namespace): the same manner, argument checks,
// allocation of outputs and workspaces, the stream, and the autograd node of the rotary positions.

// ---- tensor arguments ----------------------------------------------------------------------------
bool value_error(const char* name, const char* need) {
  PyErr_Format(PyExc_ValueError, "%s: %s", name, need);
  return false;
}
// A dense GPU tensor of a type and shape (a size of -1: any), on the device of the call's other tensors.
struct DeviceOf {
  c10::optional<at::Device> device;
  bool take(const Tensor& t, const char* name) {
    if (!device.has_value()) device = t.device();
    return t.device() == *device || value_error(name, "on another device than the call's other tensors");
  }
};
const Tensor* dense(PyObject* o, at::ScalarType dtype, at::IntArrayRef shape, const char* name, DeviceOf& dev) {
  const Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (t == nullptr) {
    PyErr_Format(PyExc_TypeError, "%s: need a tensor", name);
    return nullptr;
  }
  bool ok = t->scalar_type() == dtype && t->dim() == (int64_t)shape.size() && t->is_contiguous() && t->is_cuda();
  for (size_t k = 0; ok && k < shape.size(); k++) ok = shape[k] < 0 || t->size((int64_t)k) == shape[k];
  if (!ok) {
    std::string want, got;
    for (const int64_t s : shape) want += (want.empty() ? "" : ", ") + (s < 0 ? std::string("any") : std::to_string(s));
    for (const int64_t s : t->sizes()) got += (got.empty() ? "" : ", ") + std::to_string(s);
    PyErr_Format(PyExc_ValueError, "%s: need contiguous cuda %s (%s), got %s%s %s (%s)", name, c10::toString(dtype), want.c_str(),
                 t->is_contiguous() ? "" : "strided ", t->is_cuda() ? "cuda" : "cpu", c10::toString(t->scalar_type()), got.c_str());
    return nullptr;
  }
  return dev.take(*t, name) ? t : nullptr;
}
bool dense_or_none(PyObject* o, at::ScalarType dtype, at::IntArrayRef shape, const char* name, DeviceOf& dev, Tensor* out) {
  if (o == Py_None) return true;
  const Tensor* t = dense(o, dtype, shape, name, dev);
  if (t != nullptr) *out = *t;
  return t != nullptr;
}
// Stride of a dimension as the library takes it: of a dimension of one element, none.
int64_t stride_of(const Tensor& t, int64_t k) { return t.size(k) <= 1 ? 0 : t.stride(k); }
bool rows_fit(const Tensor& t) {
  bool ok = t.stride(-1) == 1 && ((uintptr_t)t.data_ptr() & 15) == 0;
  for (int64_t k = 0; k + 1 < t.dim(); k++) ok = ok && stride_of(t, k) % 8 == 0;
  return ok;
}
// A bf16 GPU tensor [T, H, d] whose channels are adjacent and whose rows begin on 16 bytes: a slice of a projection's output is one.
const Tensor* token_rows(PyObject* o, int64_t T, int64_t H, int64_t d, const char* name, DeviceOf& dev) {
  const Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (t == nullptr) {
    PyErr_Format(PyExc_TypeError, "%s: need a tensor", name);
    return nullptr;
  }
  if (t->scalar_type() != at::kBFloat16 || !t->is_cuda() || t->dim() != 3 || (T >= 0 && t->size(0) != T) || (H >= 0 && t->size(1) != H) ||
      t->size(2) != d) {
    PyErr_Format(PyExc_ValueError, "%s: need cuda bfloat16 [tokens, heads, %lld]", name, (long long)d);
    return nullptr;
  }
  if (!rows_fit(*t)) {
    value_error(name, "need adjacent channels, strides that are multiples of 8 and rows that begin on 16 bytes");
    return nullptr;
  }
  return dev.take(*t, name) ? t : nullptr;
}
const Tensor* pool_arg(PyObject* o, sagebwd_cache_params& p, DeviceOf& dev) {
  p.pages = 1;
  size_t bytes = 0;
  const int rc = sagebwd_cache_page_bytes(&p, &bytes);
  if (rc != SAGEBWD_OK) {
    raise_status(rc, "sagebwd_cache_page_bytes");
    return nullptr;
  }
  const Tensor* t = dense(o, at::kByte, {-1, p.H, (int64_t)bytes / p.H}, "cache", dev);
  if (t == nullptr) return nullptr;
  if (t->size(0) < 1 || t->size(0) > INT32_MAX) {
    value_error("cache", "need 1 to 2^31 - 1 pages");
    return nullptr;
  }
  p.pages = (int32_t)t->size(0);
  return t;
}
bool size_arg(PyObject* o, const char* name, int64_t least, int64_t* out) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) return false;
  if (x < least || x > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s: %lld is out of range", name, x);
    return false;
  }
  *out = x;
  return true;
}
// (H, d, page, group, block) as five arguments
bool cache_params(PyObject* const* a, sagebwd_cache_params& p) {
  int64_t x[5];
  const char* names[5] = {"H", "d", "page", "group", "block"};
  for (int k = 0; k < 5; k++)
    if (!size_arg(a[k], names[k], 0, &x[k])) return false;
  p = sagebwd_cache_params{(int32_t)x[0], (int32_t)x[1], (int32_t)x[2], x[4] == 0 ? (int32_t)x[3] : 0, 0, (int32_t)x[4]};
  return true;
}

// A tensor of one dimension in another one's memory.
Tensor part_of(const Tensor& all, at::ScalarType dtype, int64_t offset, int64_t n) {
  Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(dtype));
  t.unsafeGetTensorImpl()->set_storage_offset(offset);
  t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
  return t;
}

// ---- the cache -------------------------------------------------------------------------------------
// plan(held, added, table, free_pages, free_count, page, rows, out | None) -> (slots, positions, cu_new, lengths, granted, free_left)
PyObject* py_cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  const Tensor *held, *added, *table, *free_pages, *free_count;
  int64_t page, rows;
  if (!arg_count(n, 8, "cache_plan") || !(held = dense(a[0], at::kInt, {-1}, "held", dev)) ||
      !(added = dense(a[1], at::kInt, {held->size(0)}, "added", dev)) ||
      !(table = dense(a[2], at::kInt, {held->size(0), -1}, "block_table", dev)) || !(free_pages = dense(a[3], at::kInt, {-1}, "free_pages", dev)) ||
      !(free_count = dense(a[4], at::kInt, {1}, "free_count", dev)) || !size_arg(a[5], "page", 0, &page) || !size_arg(a[6], "rows", 0, &rows))
    return nullptr;
  if (rows > 1 << 30) return raise_status(SAGEBWD_UNSUPPORTED_SHAPE, "sagebwd_cache_plan");      // (before its outputs are allocated)
  const int64_t R = held->size(0);
  const std::array<int64_t, 6> sizes = {rows, rows, R + 1, R, R, 1};
  const char* names[6] = {"slots", "positions", "cu_new", "lengths", "granted", "free_left"};
  Tensor out[6];
  if (a[7] != Py_None) {
    THPObjectPtr seq(PySequence_Fast(a[7], "out: need the six tensors of a plan"));
    if (!seq) return nullptr;
    if (PySequence_Fast_GET_SIZE(seq.get()) != 6) {
      PyErr_SetString(PyExc_ValueError, "out: need the six tensors of a plan");
      return nullptr;
    }
    for (int k = 0; k < 6; k++) {
      const Tensor* t = dense(PySequence_Fast_GET_ITEM(seq.get(), k), k == 0 ? at::kLong : at::kInt, {sizes[k]}, names[k], dev);
      if (t == nullptr) return nullptr;
      out[k] = *t;
    }
  }
  if (table->size(1) < 1 || table->size(1) > INT32_MAX || R > INT32_MAX || free_pages->size(0) > INT32_MAX) {
    value_error("block_table", "sizes are out of range");
    return nullptr;
  }
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(held->device());
    if (!out[0].defined()) {
      // One allocation, of which the six are parts: the smallest calls are bound by the host (six narrow() took 6 of 8.4 us).
      const Tensor all = at::empty({2 * rows + rows + (R + 1) + 2 * R + 1}, held->options());
      int64_t word = 0;
      for (int k = 0; k < 6; k++) {
        out[k] = part_of(all, k == 0 ? at::kLong : at::kInt, k == 0 ? word / 2 : word, sizes[k]);
        word += k == 0 ? 2 * rows : sizes[k];
      }
    }
    rc = sagebwd_cache_plan((const int32_t*)held->data_ptr(), (const int32_t*)added->data_ptr(), (int32_t*)table->data_ptr(),
                            (const int32_t*)free_pages->data_ptr(), (const int32_t*)free_count->data_ptr(), (int32_t)R, (int32_t)table->size(1),
                            (int32_t)page, (int32_t)free_pages->size(0), (int32_t)rows, (int64_t*)out[0].data_ptr(), (int32_t*)out[1].data_ptr(),
                            (int32_t*)out[2].data_ptr(), (int32_t*)out[3].data_ptr(), (int32_t*)out[4].data_ptr(), (int32_t*)out[5].data_ptr(),
                            (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_plan");
  return Py_BuildValue("(NNNNNN)", THPVariable_Wrap(out[0]), THPVariable_Wrap(out[1]), THPVariable_Wrap(out[2]), THPVariable_Wrap(out[3]),
                       THPVariable_Wrap(out[4]), THPVariable_Wrap(out[5]));
  END_HANDLE_TH_ERRORS
}

// trim(keep, lengths, table, free_pages, free_count, page)
PyObject* py_cache_trim(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  const Tensor *keep, *lengths, *table, *free_pages, *free_count;
  int64_t page;
  if (!arg_count(n, 6, "cache_trim") || !(keep = dense(a[0], at::kInt, {-1}, "keep", dev)) ||
      !(lengths = dense(a[1], at::kInt, {keep->size(0)}, "lengths", dev)) ||
      !(table = dense(a[2], at::kInt, {keep->size(0), -1}, "block_table", dev)) || !(free_pages = dense(a[3], at::kInt, {-1}, "free_pages", dev)) ||
      !(free_count = dense(a[4], at::kInt, {1}, "free_count", dev)) || !size_arg(a[5], "page", 0, &page))
    return nullptr;
  if (table->size(1) < 1 || table->size(1) > INT32_MAX || keep->size(0) > INT32_MAX || free_pages->size(0) > INT32_MAX) {
    value_error("block_table", "sizes are out of range");
    return nullptr;
  }
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(keep->device());
    rc = sagebwd_cache_trim((const int32_t*)keep->data_ptr(), (int32_t*)lengths->data_ptr(), (int32_t*)table->data_ptr(),
                            (int32_t*)free_pages->data_ptr(), (int32_t*)free_count->data_ptr(), (int32_t)keep->size(0), (int32_t)table->size(1),
                            (int32_t)page, (int32_t)free_pages->size(0), (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_trim");
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// lengths, table, free_pages, free_count, shares: what the calls on shared pages change, five arguments from `a` on, of R requests.
struct SharedPages {
  const Tensor *lengths, *table, *free_pages, *free_count, *shares;
  int32_t R, columns, capacity, pages;
  bool take(PyObject* const* a, int64_t requests, DeviceOf& dev) {
    if (!(lengths = dense(a[0], at::kInt, {requests}, "lengths", dev)) || !(table = dense(a[1], at::kInt, {requests, -1}, "block_table", dev)) ||
        !(free_pages = dense(a[2], at::kInt, {-1}, "free_pages", dev)) || !(free_count = dense(a[3], at::kInt, {1}, "free_count", dev)) ||
        !(shares = dense(a[4], at::kInt, {3, -1}, "shares", dev)))
      return false;
    if (table->size(1) < 1 || table->size(1) > INT32_MAX || requests > INT32_MAX || free_pages->size(0) > INT32_MAX || shares->size(1) > INT32_MAX)
      return value_error("block_table", "sizes are out of range");
    R = (int32_t)requests;
    columns = (int32_t)table->size(1);
    capacity = (int32_t)free_pages->size(0);
    pages = (int32_t)shares->size(1);
    return true;
  }
};

// free(keep, lengths, table, free_pages, free_count, shares, page)
PyObject* py_cache_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  const Tensor* keep;
  SharedPages s;
  int64_t page;
  if (!arg_count(n, 7, "cache_free") || !(keep = dense(a[0], at::kInt, {-1}, "keep", dev)) || !s.take(a + 1, keep->size(0), dev) ||
      !size_arg(a[6], "page", 0, &page))
    return nullptr;
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(keep->device());
    rc = sagebwd_cache_free((const int32_t*)keep->data_ptr(), (int32_t*)s.lengths->data_ptr(), (int32_t*)s.table->data_ptr(),
                            (int32_t*)s.free_pages->data_ptr(), (int32_t*)s.free_count->data_ptr(), (int32_t*)s.shares->data_ptr(), s.R, s.columns,
                            (int32_t)page, s.capacity, s.pages, (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_free");
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// fork(parents, lengths, table, free_pages, free_count, shares, page)
PyObject* py_cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  const Tensor* parents;
  SharedPages s;
  int64_t page;
  if (!arg_count(n, 7, "cache_fork") || !(parents = dense(a[0], at::kInt, {-1}, "parents", dev)) || !s.take(a + 1, parents->size(0), dev) ||
      !size_arg(a[6], "page", 0, &page))
    return nullptr;
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(parents->device());
    size_t bytes = 0;
    rc = sagebwd_cache_fork_workspace_bytes(s.R, s.columns, &bytes);
    if (rc == SAGEBWD_OK) {
      const Tensor ws = at::empty({(int64_t)bytes}, parents->options().dtype(at::kByte));
      rc = sagebwd_cache_fork((const int32_t*)parents->data_ptr(), (int32_t*)s.lengths->data_ptr(), (int32_t*)s.table->data_ptr(),
                              (int32_t*)s.free_pages->data_ptr(), (int32_t*)s.free_count->data_ptr(), (int32_t*)s.shares->data_ptr(), s.R, s.columns,
                              (int32_t)page, s.capacity, s.pages, ws.data_ptr(), bytes, (void*)current_stream());
    }
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_fork");
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

bool shares_fit(const SharedPages& s, const sagebwd_cache_params& p) {
  return s.pages == p.pages || value_error("shares", "has another number of pages than the cache");
}

// own(added, lengths, table, free_pages, free_count, shares, cache, H, d, page, group, block, out | None) -> added
PyObject* py_cache_own(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  sagebwd_cache_params p;
  const Tensor *added, *pool;
  Tensor out;
  SharedPages s;
  if (!arg_count(n, 13, "cache_own") || !cache_params(a + 7, p) || !(pool = pool_arg(a[6], p, dev)) || !(added = dense(a[0], at::kInt, {-1}, "added", dev)) ||
      !s.take(a + 1, added->size(0), dev) || !shares_fit(s, p) || !dense_or_none(a[12], at::kInt, {added->size(0)}, "out", dev, &out))
    return nullptr;
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(added->device());
    if (!out.defined()) out = at::empty({s.R}, added->options());
    const Tensor ws = at::empty({8 * (int64_t)s.R + 16}, added->options().dtype(at::kByte));
    rc = sagebwd_cache_own((const int32_t*)added->data_ptr(), (const int32_t*)s.lengths->data_ptr(), (int32_t*)s.table->data_ptr(),
                           (const int32_t*)s.free_pages->data_ptr(), (int32_t*)s.free_count->data_ptr(), (int32_t*)s.shares->data_ptr(), s.R, s.columns,
                           s.capacity, &p, pool->data_ptr(), (int32_t*)out.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_own");
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// compact(lengths, table, cache, H, d, page, group, block, out | None) -> (table, free_pages, free_count, shares, used)
PyObject* py_cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  sagebwd_cache_params p;
  const Tensor *lengths, *table, *pool;
  if (!arg_count(n, 9, "cache_compact") || !cache_params(a + 3, p) || !(pool = pool_arg(a[2], p, dev)) ||
      !(lengths = dense(a[0], at::kInt, {-1}, "lengths", dev)) || !(table = dense(a[1], at::kInt, {lengths->size(0), -1}, "block_table", dev)))
    return nullptr;
  const int64_t R = lengths->size(0);
  if (table->size(1) < 1 || table->size(1) > INT32_MAX || R > INT32_MAX) {
    value_error("block_table", "sizes are out of range");
    return nullptr;
  }
  Tensor out[5];
  if (a[8] != Py_None) {
    THPObjectPtr seq(PySequence_Fast(a[8], "out: need the five tensors of a compaction"));
    if (!seq) return nullptr;
    if (PySequence_Fast_GET_SIZE(seq.get()) != 5) {
      PyErr_SetString(PyExc_ValueError, "out: need the five tensors of a compaction");
      return nullptr;
    }
    const char* names[5] = {"block_table", "free_pages", "free_count", "shares", "used"};
    const std::vector<int64_t> shapes[5] = {{R, table->size(1)}, {-1}, {1}, {3, p.pages}, {1}};
    for (int k = 0; k < 5; k++) {
      const Tensor* t = dense(PySequence_Fast_GET_ITEM(seq.get(), k), at::kInt, shapes[k], names[k], dev);
      if (t == nullptr) return nullptr;
      out[k] = *t;
    }
    if (out[1].size(0) < p.pages || out[1].size(0) > INT32_MAX) {
      value_error("free_pages", "has no room for every page");
      return nullptr;
    }
  }
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(lengths->device());
    size_t bytes = 0;
    rc = sagebwd_cache_compact_workspace_bytes(p.pages, &bytes);
    if (rc == SAGEBWD_OK) {
      if (!out[0].defined()) {
        out[0] = at::empty(table->sizes(), lengths->options());
        out[1] = at::empty({p.pages}, lengths->options());
        out[2] = at::empty({1}, lengths->options());
        out[3] = at::zeros({3, p.pages}, lengths->options());
        out[4] = at::empty({1}, lengths->options());
      }
      const Tensor ws = at::empty({(int64_t)bytes}, lengths->options().dtype(at::kByte));
      rc = sagebwd_cache_compact((const int32_t*)lengths->data_ptr(), (const int32_t*)table->data_ptr(), (int32_t)R, (int32_t)table->size(1), &p,
                                 pool->data_ptr(), (int32_t*)out[0].data_ptr(), (int32_t*)out[1].data_ptr(), (int32_t)out[1].size(0),
                                 (int32_t*)out[2].data_ptr(), (int32_t*)out[3].data_ptr(), (int32_t*)out[4].data_ptr(), ws.data_ptr(), bytes,
                                 (void*)current_stream());
    }
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_compact");
  return Py_BuildValue("(NNNNN)", THPVariable_Wrap(out[0]), THPVariable_Wrap(out[1]), THPVariable_Wrap(out[2]), THPVariable_Wrap(out[3]),
                       THPVariable_Wrap(out[4]));
  END_HANDLE_TH_ERRORS
}

const float* data_or_null(const Tensor& t) { return t.defined() ? (const float*)t.data_ptr() : nullptr; }

// append(K, V, slots, cache, H, d, page, group, block, k_mean | None, v_mean | None)
PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  sagebwd_cache_params p;
  const Tensor *K, *V, *slots, *pool;
  Tensor km, vm;
  if (!arg_count(n, 11, "cache_append") || !cache_params(a + 4, p) || !(pool = pool_arg(a[3], p, dev)) ||
      !(K = token_rows(a[0], -1, p.H, p.d, "K", dev)) || !(V = token_rows(a[1], K->size(0), p.H, p.d, "V", dev)) ||
      !(slots = dense(a[2], at::kLong, {K->size(0)}, "slots", dev)) || !dense_or_none(a[9], at::kFloat, {p.H, p.d}, "k_mean", dev, &km) ||
      !dense_or_none(a[10], at::kFloat, {p.H, p.d}, "v_mean", dev, &vm))
    return nullptr;
  if (K->size(0) > INT32_MAX) {
    value_error("K", "too many tokens");
    return nullptr;
  }
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(K->device());
    rc = sagebwd_cache_append(K->data_ptr(), V->data_ptr(), stride_of(*K, 0), stride_of(*K, 1), stride_of(*V, 0), stride_of(*V, 1),
                              (const int64_t*)slots->data_ptr(), (int32_t)K->size(0), data_or_null(km), data_or_null(vm), &p, pool->data_ptr(),
                              (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_append");
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// read(slots, cache, H, d, page, group, block, k_mean | None, v_mean | None, K | None, V | None) -> (K, V)
PyObject* py_cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  sagebwd_cache_params p;
  const Tensor *slots, *pool;
  Tensor km, vm, K, V;
  if (!arg_count(n, 11, "cache_read") || !cache_params(a + 2, p) || !(pool = pool_arg(a[1], p, dev)) ||
      !(slots = dense(a[0], at::kLong, {-1}, "slots", dev)) || !dense_or_none(a[7], at::kFloat, {p.H, p.d}, "k_mean", dev, &km) ||
      !dense_or_none(a[8], at::kFloat, {p.H, p.d}, "v_mean", dev, &vm))
    return nullptr;
  const std::array<int64_t, 3> shape = {slots->size(0), p.H, p.d};
  if (!dense_or_none(a[9], at::kBFloat16, shape, "K", dev, &K) || !dense_or_none(a[10], at::kBFloat16, shape, "V", dev, &V)) return nullptr;
  if (shape[0] > INT32_MAX) {
    value_error("slots", "too many tokens");
    return nullptr;
  }
  int rc;
  WITHOUT_GIL({
    const c10::DeviceGuard guard(pool->device());
    if (!K.defined()) K = at::empty(shape, pool->options().dtype(at::kBFloat16));
    if (!V.defined()) V = at::empty(shape, pool->options().dtype(at::kBFloat16));
    rc = sagebwd_cache_read((const int64_t*)slots->data_ptr(), (int32_t)shape[0], data_or_null(km), data_or_null(vm), &p, pool->data_ptr(),
                            K.data_ptr(), V.data_ptr(), (void*)current_stream());
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_read");
  return wrap2(K, V);
  END_HANDLE_TH_ERRORS
}

// attention(Q, cache, table, lengths, cu, H, d, page, group, block, max_new, causal, sm_scale, v_mean | None, max_length, workspace | None, O | None,
//           LSE | None) -> (O, LSE)
PyObject* py_cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  DeviceOf dev;
  sagebwd_cache_params p;
  const Tensor *Q, *pool, *table, *lengths, *cu;
  Tensor vm, ws, O, L;
  int64_t max_new, max_length;
  if (!arg_count(n, 18, "cache_attention") || !cache_params(a + 5, p) || !(pool = pool_arg(a[1], p, dev)) ||
      !(Q = token_rows(a[0], -1, -1, p.d, "Q", dev)) || !(lengths = dense(a[3], at::kInt, {-1}, "lengths", dev)) ||
      !(table = dense(a[2], at::kInt, {lengths->size(0), -1}, "block_table", dev)) ||
      !(cu = dense(a[4], at::kInt, {lengths->size(0) + 1}, "cu", dev)) || !size_arg(a[10], "max_new", 1, &max_new) ||
      !dense_or_none(a[13], at::kFloat, {p.H, p.d}, "v_mean", dev, &vm) || !size_arg(a[14], "max_length", 0, &max_length) ||
      !dense_or_none(a[15], at::kByte, {-1}, "workspace", dev, &ws))
    return nullptr;
  const int causal = PyObject_IsTrue(a[11]);
  const double sm_scale = PyFloat_AsDouble(a[12]);
  if (causal < 0 || (sm_scale == -1.0 && PyErr_Occurred())) return nullptr;
  const int64_t T = Q->size(0), Hq = Q->size(1);
  const std::array<int64_t, 3> oshape = {T, Hq, p.d};
  const std::array<int64_t, 2> lshape = {Hq, T};
  if (!dense_or_none(a[16], at::kBFloat16, oshape, "O", dev, &O) || !dense_or_none(a[17], at::kFloat, lshape, "LSE", dev, &L)) return nullptr;
  if (T > INT32_MAX || Hq > INT32_MAX || table->size(1) < 1 || table->size(1) > INT32_MAX || lengths->size(0) > INT32_MAX) {
    value_error("block_table", "sizes are out of range");
    return nullptr;
  }
  sagebwd_cache_call c;
  c.R = (int32_t)lengths->size(0);
  c.T = (int32_t)T;
  c.Hq = (int32_t)Hq;
  c.columns = (int32_t)table->size(1);
  c.max_new = (int32_t)max_new;
  c.max_length = (int32_t)max_length;
  c.causal = causal;
  c.sm_scale = (float)sm_scale;
  c.q_token_stride = stride_of(*Q, 0);
  c.q_head_stride = stride_of(*Q, 1);
  int rc = SAGEBWD_OK;
  const char* where = "sagebwd_cache_workspace_bytes";
  WITHOUT_GIL({
    const c10::DeviceGuard guard(Q->device());
    if (!ws.defined()) {
      size_t bytes = 0;
      rc = sagebwd_cache_workspace_bytes(&p, &c, &bytes);
      if (rc == SAGEBWD_OK) ws = at::empty({(int64_t)bytes}, Q->options().dtype(at::kByte));
    }
    if (rc == SAGEBWD_OK) {
      where = "sagebwd_cache_attention";
      if (!O.defined()) O = at::empty(oshape, Q->options());
      if (!L.defined()) L = at::empty(lshape, Q->options().dtype(at::kFloat));
      rc = sagebwd_cache_attention(Q->data_ptr(), pool->data_ptr(), (const int32_t*)table->data_ptr(), (const int32_t*)lengths->data_ptr(),
                                   (const int32_t*)cu->data_ptr(), data_or_null(vm), &p, &c, O.data_ptr(), (float*)L.data_ptr(), ws.data_ptr(),
                                   (size_t)ws.numel(), (void*)current_stream());
    }
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, where);
  return wrap2(O, L);
  END_HANDLE_TH_ERRORS
}

// workspace_bytes(H, d, page, group, block, R, T, Hq, columns, max_new, max_length) -> bytes
PyObject* py_cache_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  sagebwd_cache_params p;
  if (!arg_count(n, 11, "cache_workspace_bytes") || !cache_params(a, p)) return nullptr;
  p.pages = 1;
  int64_t x[6];
  const char* names[6] = {"R", "T", "Hq", "columns", "max_new", "max_length"};
  for (int k = 0; k < 6; k++)
    if (!size_arg(a[5 + k], names[k], 0, &x[k])) return nullptr;
  const sagebwd_cache_call c = {(int32_t)x[0], (int32_t)x[1], (int32_t)x[2], (int32_t)x[3], (int32_t)x[4], (int32_t)x[5], 1, 0.f, 0, 0};
  size_t bytes = 0;
  const int rc = sagebwd_cache_workspace_bytes(&p, &c, &bytes);
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_cache_workspace_bytes");
  return PyLong_FromSize_t(bytes);
  END_HANDLE_TH_ERRORS
}

// ---- rotary positions ------------------------------------------------------------------------------
struct RotaryCall {
  Tensor positions, inv_freq;     // [axes, B N], [rotary_dim / 2]
  int axes;
  std::array<int32_t, 4> sections;
  bool adjacent, token_major;
};
// batch, row, head strides
void rotary_strides(const Tensor& t, bool token_major, int64_t* s) {
  if (t.dim() == 3) {
    s[0] = 0;
    s[1] = stride_of(t, 0);
    s[2] = stride_of(t, 1);
  } else {
    s[0] = stride_of(t, 0);
    s[1] = stride_of(t, token_major ? 1 : 2);
    s[2] = stride_of(t, token_major ? 2 : 1);
  }
}
int64_t rotary_heads(const Tensor& t, bool token_major) { return t.size(t.dim() == 3 ? 1 : token_major ? 2 : 1); }

// Turned Q and K (either may be undefined) as new dense tensors; no autograd.
int rotary_launch(const RotaryCall& c, const Tensor& Q, const Tensor& K, bool inverse, Tensor* Qo, Tensor* Ko) {
  const bool both = Q.defined() && K.defined();
  // (a copy, not contiguous(): a view of a larger buffer may be dense and begin off 16 bytes)
  const auto fitting = [](const Tensor& t) { return rows_fit(t) ? t : t.clone(at::MemoryFormat::Contiguous); };
  const Tensor x = fitting(Q.defined() ? Q : K), z = both ? fitting(K) : Tensor();
  Tensor y = at::empty(x.sizes(), x.options()), w;
  if (both) w = at::empty(z.sizes(), z.options());
  sagebwd_rotary_params p;
  memset(&p, 0, sizeof(p));
  const bool three = x.dim() == 3;
  p.B = three ? 1 : (int32_t)x.size(0);
  p.N = (int32_t)x.size(three ? 0 : c.token_major ? 1 : 2);
  p.Hq = (int32_t)rotary_heads(x, c.token_major);
  p.Hk = both ? (int32_t)rotary_heads(z, c.token_major) : 0;
  p.d = (int32_t)x.size(-1);
  p.rotary_dim = 2 * (int32_t)c.inv_freq.numel();
  p.axes = c.axes;
  for (int k = 0; k < 4; k++) p.sections[k] = c.sections[k];
  p.adjacent = c.adjacent;
  p.inverse = inverse;
  p.positions64 = c.positions.scalar_type() == at::kLong;
  rotary_strides(x, c.token_major, p.q_strides);
  rotary_strides(y, c.token_major, p.qo_strides);
  if (both) {
    rotary_strides(z, c.token_major, p.k_strides);
    rotary_strides(w, c.token_major, p.ko_strides);
  }
  const int rc = sagebwd_rotary(x.data_ptr(), both ? z.data_ptr() : nullptr, y.data_ptr(), both ? w.data_ptr() : nullptr, c.positions.data_ptr(),
                                (const float*)c.inv_freq.data_ptr(), &p, (void*)current_stream());
  if (Q.defined()) {
    *Qo = y;
    if (both) *Ko = w;
  } else {
    *Ko = y;
  }
  return rc;
}

int rotary_apply(const RotaryCall& c, const Tensor& Q, const Tensor& K, bool inverse, Tensor* Qo, Tensor* Ko);

// The turn is linear: its gradient is the turn by the negative angles, and that of a gradient again the turn.
struct SageRotaryBackward : torch::autograd::Node {
  torch::autograd::SavedVariable positions, inv_freq;
  RotaryCall call;
  bool inverse;
  std::string name() const override { return "SageRotaryBackward"; }
  void release_variables() override {
    std::lock_guard<std::mutex> lock(mutex_);
    positions.reset_data();
    inv_freq.reset_data();
  }
  torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
    std::lock_guard<std::mutex> lock(mutex_);
    RotaryCall c = call;
    c.positions = positions.unpack();
    c.inv_freq = inv_freq.unpack();
    torch::autograd::variable_list out(grads.size());
    const Tensor dQ = grads[0], dK = grads.size() > 1 ? grads[1] : Tensor();
    if (!dQ.defined() && !dK.defined()) return out;
    if ((dQ.defined() && is_transformed(dQ)) || (dK.defined() && is_transformed(dK)))       // (double backward has a rule, a tangent of the gradient none)
      throw_python([] { refuse_transformed("sage_rotary"); });
    Tensor q, k;
    const c10::DeviceGuard guard(c.positions.device());
    const int rc = rotary_apply(c, dQ, dK, !inverse, &q, &k);
    if (rc != SAGEBWD_OK) throw_python([&] { raise_status(rc, "sagebwd_rotary"); });
    out[0] = q;
    if (out.size() > 1) out[1] = k;
    return out;
  }
};

int rotary_apply(const RotaryCall& c, const Tensor& Q, const Tensor& K, bool inverse, Tensor* Qo, Tensor* Ko) {
  const bool track = at::GradMode::is_enabled() && ((Q.defined() && Q.requires_grad()) || (K.defined() && K.requires_grad()));
  int rc;
  {
    at::NoGradGuard no_grad;
    rc = rotary_launch(c, Q, K, inverse, Qo, Ko);
  }
  if (rc != SAGEBWD_OK || !track) return rc;
  std::shared_ptr<SageRotaryBackward> node(new SageRotaryBackward(), torch::autograd::deleteNode);
  torch::autograd::edge_list edges = K.defined() && Q.defined() ? torch::autograd::collect_next_edges(Q, K)
                                     : torch::autograd::collect_next_edges(Q.defined() ? Q : K);
  node->positions = torch::autograd::SavedVariable(c.positions, false);
  node->inv_freq = torch::autograd::SavedVariable(c.inv_freq, false);
  node->call = c;
  node->call.positions = Tensor();
  node->call.inv_freq = Tensor();
  node->inverse = inverse;
  node->set_next_edges(std::move(edges));
  if (Q.defined()) torch::autograd::set_history(*Qo, node);
  if (K.defined()) torch::autograd::set_history(*Ko, node);
  return rc;
}

// rotary(Q, K | None, positions, inv_freq, sections | None, adjacent, token_major, inverse) -> (Q, K | None)
PyObject* py_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arg_count(n, 8, "rotary")) return nullptr;
  for (int k = 0; k < 2; k++) {
    if (k == 1 && a[k] == Py_None) continue;
    if (!THPVariable_Check(a[k])) {
      PyErr_SetString(PyExc_TypeError, "sage_rotary: Q and K are tensors");
      return nullptr;
    }
  }
  for (int k = 0; k < 4; k++) {       // (the positions and frequencies too: their other checks come later)
    if (THPVariable_Check(a[k]) && is_transformed(THPVariable_Unpack(a[k]))) {
      refuse_transformed("sage_rotary");
      return nullptr;
    }
  }
  const int adjacent = PyObject_IsTrue(a[5]), token_major = PyObject_IsTrue(a[6]), inverse = PyObject_IsTrue(a[7]);
  if (adjacent < 0 || token_major < 0 || inverse < 0) return nullptr;
  DeviceOf dev;
  const Tensor Q = THPVariable_Unpack(a[0]), K = a[1] != Py_None ? THPVariable_Unpack(a[1]) : Tensor();
  const bool three = Q.dim() == 3;
  RotaryCall c;
  c.adjacent = adjacent;
  c.token_major = three || token_major;
  for (int k = 0; k < (K.defined() ? 2 : 1); k++) {
    const Tensor& t = k == 0 ? Q : K;
    const char* name = k == 0 ? "Q" : "K";
    if (t.scalar_type() != at::kBFloat16 || !t.is_cuda() || t.dim() != Q.dim() || (t.dim() != 3 && t.dim() != 4) || t.size(-1) != Q.size(-1)) {
      value_error(name, "need cuda bfloat16 [tokens, heads, d] or four dimensions");
      return nullptr;
    }
    if (!dev.take(t, name)) return nullptr;
  }
  const int64_t B = three ? 1 : Q.size(0), N = Q.size(three ? 0 : token_major ? 1 : 2);
  if (K.defined() && ((three ? 1 : K.size(0)) != B || K.size(three ? 0 : token_major ? 1 : 2) != N)) {
    value_error("K", "has other tokens than Q");
    return nullptr;
  }
  const Tensor* freq = dense(a[3], at::kFloat, {-1}, "inv_freq", dev);
  if (freq == nullptr) return nullptr;
  c.inv_freq = *freq;
  if (at::GradMode::is_enabled() && freq->requires_grad()) {
    PyErr_SetString(PyExc_NotImplementedError, "sage_rotary: inv_freq gets no gradient (detach it)");
    return nullptr;
  }
  c.sections = {0, 0, 0, 0};
  if (a[4] == Py_None) {
    c.axes = 1;
    c.sections[0] = (int32_t)freq->numel();
  } else {
    THPObjectPtr seq(PySequence_Fast(a[4], "sections: need a list of one to four numbers"));
    if (!seq) return nullptr;
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq.get());
    if (count < 1 || count > 4) {
      value_error("sections", "need a list of one to four numbers");
      return nullptr;
    }
    c.axes = (int)count;
    int64_t sum = 0;
    for (int k = 0; k < c.axes; k++) {
      int64_t x;
      if (!size_arg(PySequence_Fast_GET_ITEM(seq.get(), k), "sections", 0, &x)) return nullptr;
      c.sections[k] = (int32_t)x;
      sum += x;
    }
    if (sum != freq->numel()) {
      value_error("sections", "their sum is not the number of frequencies");
      return nullptr;
    }
  }
  // positions [axes, B, N], or less a leading dimension that is 1 or the same for all: [axes, N], and for one axis [B, N], [N]
  if (!THPVariable_Check(a[2])) {
    PyErr_SetString(PyExc_TypeError, "positions: need a tensor");
    return nullptr;
  }
  Tensor pos = THPVariable_Unpack(a[2]);
  if ((pos.scalar_type() != at::kInt && pos.scalar_type() != at::kLong) || !pos.is_cuda()) {
    value_error("positions", "need cuda int32 or int64");
    return nullptr;
  }
  if (!dev.take(pos, "positions")) return nullptr;
  const auto is = [&](std::initializer_list<int64_t> shape) { return pos.sizes() == at::IntArrayRef(shape); };
  if (B > INT32_MAX || N > INT32_MAX || Q.size(-1) > INT32_MAX || freq->numel() > INT32_MAX / 2 || rotary_heads(Q, c.token_major) > INT32_MAX) {
    value_error("Q", "sizes are out of range");
    return nullptr;
  }
  Tensor Qo, Ko;
  int rc;
  {
    const at::NoGradGuard no_grad;
    if (three ? is({c.axes, N}) : is({c.axes, B, N})) {
    } else if (c.axes == 1 && (three ? is({N}) : is({B, N}))) {
    } else if (!three && is({c.axes, N})) {
      pos = pos.unsqueeze(1).expand({c.axes, B, N});
    } else if (!three && c.axes == 1 && is({N})) {
      pos = pos.unsqueeze(0).expand({B, N});
    } else {
      value_error("positions", "need [axes, tokens], or without the first where there is one axis");
      return nullptr;
    }
    c.positions = pos.contiguous();
  }
  WITHOUT_GIL({
    const c10::DeviceGuard guard(Q.device());
    rc = rotary_apply(c, Q, K, inverse, &Qo, &Ko);
  })
  if (rc != SAGEBWD_OK) return raise_status(rc, "sagebwd_rotary");
  if (!K.defined()) return Py_BuildValue("(NO)", THPVariable_Wrap(Qo), Py_None);
  return wrap2(Qo, Ko);
  END_HANDLE_TH_ERRORS
}
