// Python extension _lists: what the C ABI's calls take of torch tensors, read and checked.
// From Python a tensor costs some 0.4 us for its pointer, type, size, device and
// layout; of a list, read here, 10 ns, and one by itself 0.1.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <string>
#include <utility>
#include <vector>

namespace {

// Codes of the C ABI's element types, two more for bytes and one for schedules.
int code_of(const at::Tensor &t) {
    switch (t.scalar_type()) {
        case at::kFloat: return 0;
        case at::kBFloat16: return 1;
        case at::kHalf: return 2;
        case at::kChar: return 3;
        case at::kByte: return 4;
        case at::kDouble: return 5;
        default: return -1;
    }
}
std::string names_of(int types) {
    static const char *const name[] = {"float32", "bfloat16", "float16", "int8", "uint8", "float64"};
    std::string s;
    for (int k = 0; k < 6; ++k)
        if (types >> k & 1) s += (s.empty() ? "" : " or ") + std::string(name[k]);
    return s;
}

template <typename T>
PyObject *bytes_of(const std::vector<T> &v) {
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(v.data()), (Py_ssize_t)(v.size() * sizeof(T)));
}

bool overlap(std::vector<std::pair<uintptr_t, uintptr_t>> &spans) {
    auto meet = [&]() {
        for (size_t k = 1; k < spans.size(); ++k)
            if (spans[k].first < spans[k - 1].second) return true;
        return false;
    };
    if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
    return meet();
}

struct Held {      // a reference that ends with its scope
    PyObject *p;
    ~Held() { Py_XDECREF(p); }
};

PyObject *fail(const std::string &text) {
    PyErr_SetString(PyExc_ValueError, text.c_str());
    return nullptr;
}

// read(tensors, name, types, device, written, sizes, block) -> (count, device, pointers, codes, sizes, elements)
//   types: bit k allows code k; device: index, or -1: the first tensor's; written: whether the
//   tensors must not overlap; sizes: bytes of int64 that the elements have to be, or None;
//   with block > 0 two for each block of so many.
PyObject *read(PyObject *, PyObject *args) {
    PyObject *tensors, *expected;
    const char *name;
    int types, device, written;
    long long block;
    if (!PyArg_ParseTuple(args, "OsiipOL", &tensors, &name, &types, &device, &written, &expected, &block)) return nullptr;
    try {
        const Held list{PySequence_Fast(tensors, "a list of tensors is wanted")};
        if (!list.p) return nullptr;
        const size_t n = (size_t)PySequence_Fast_GET_SIZE(list.p);
        if (n == 0 && device < 0) return fail(std::string(name) + " must hold a tensor");
        const int64_t *want = nullptr;
        if (expected != Py_None) {
            if (!PyBytes_Check(expected)) return fail("sizes must be bytes");
            if ((size_t)PyBytes_GET_SIZE(expected) != n * sizeof(int64_t))
                return fail(std::string(name) + " must hold " + std::to_string(PyBytes_GET_SIZE(expected) / sizeof(int64_t)) + " tensors");
            want = reinterpret_cast<const int64_t *>(PyBytes_AS_STRING(expected));
        }
        std::vector<uintptr_t> pointers(n);
        std::vector<int32_t> codes(n);
        std::vector<int64_t> sizes(n);
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        if (written) spans.reserve(n);
        int64_t total = 0;
        for (size_t k = 0; k < n; ++k) {
            PyObject *item = PySequence_Fast_GET_ITEM(list.p, (Py_ssize_t)k);
            auto at = [&]() { return std::string(name) + "[" + std::to_string(k) + "]"; };
            if (!THPVariable_Check(item)) return fail(at() + " must be a tensor");
            const at::Tensor &t = THPVariable_Unpack(item);
            codes[k] = code_of(t);
            if (!t.is_cuda() || t.layout() != at::kStrided || codes[k] < 0 || !(types >> codes[k] & 1) || !t.is_contiguous())
                return fail(at() + " must be a contiguous device tensor of " + names_of(types));
            if (device < 0) device = (int)t.get_device();
            if (t.get_device() != device) return fail(at() + " must be on cuda:" + std::to_string(device));
            sizes[k] = t.numel();
            if (want) {
                int64_t w;
                std::memcpy(&w, want + k, sizeof w);
                if (block > 0) w = 2 * ((w + block - 1) / block);
                if (sizes[k] != w) return fail(at() + " must have " + std::to_string(w) + " elements, got " + std::to_string(sizes[k]));
            }
            total += sizes[k];
            pointers[k] = sizes[k] > 0 ? reinterpret_cast<uintptr_t>(t.data_ptr()) : 0;
            if (written && sizes[k] > 0) spans.emplace_back(pointers[k], pointers[k] + (uintptr_t)sizes[k] * t.element_size());
        }
        if (written && overlap(spans)) return fail(std::string(name) + " must not overlap each other");
        return Py_BuildValue("niNNNL", (Py_ssize_t)n, device, bytes_of(pointers), bytes_of(codes), bytes_of(sizes), (long long)total);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_ValueError, (std::string(name) + ": " + e.what()).c_str());
        return nullptr;
    }
}

struct Span {      // of bytes that a list's tensors have
    uintptr_t first, end;
    Py_ssize_t list;
    bool operator<(const Span &other) const { return first < other.first; }
};

// A list as read() gives it; `n` below 0 where it is none.
struct ReadList {
    Py_ssize_t n = -1, number;
    const char *pointers, *codes, *sizes;
    ReadList(PyObject *read, Py_ssize_t number) : number(number) {
        if (PyTuple_GET_SIZE(read) != 6) return;
        for (int k = 2; k < 5; ++k)
            if (!PyBytes_Check(PyTuple_GET_ITEM(read, k))) return;
        const auto size = [&](int k) { return (size_t)PyBytes_GET_SIZE(PyTuple_GET_ITEM(read, k)); };
        const size_t count = size(2) / sizeof(uintptr_t);
        if (size(3) != count * sizeof(int32_t) || size(4) != count * sizeof(int64_t)) return;
        pointers = PyBytes_AS_STRING(PyTuple_GET_ITEM(read, 2));
        codes = PyBytes_AS_STRING(PyTuple_GET_ITEM(read, 3));
        sizes = PyBytes_AS_STRING(PyTuple_GET_ITEM(read, 4));
        n = (Py_ssize_t)count;
    }
    // f(first byte, end) of each tensor that is not empty; false where there is no such type or size.
    template <typename F>
    bool each(F f) const {
        static const uintptr_t width[] = {4, 2, 2, 1, 1, 8};
        for (Py_ssize_t k = 0; k < n; ++k) {
            uintptr_t p;
            int32_t code;
            int64_t elements;
            std::memcpy(&p, pointers + k * sizeof p, sizeof p);
            std::memcpy(&code, codes + k * sizeof code, sizeof code);
            std::memcpy(&elements, sizes + k * sizeof elements, sizeof elements);
            if (code < 0 || code > 5 || elements < 0) return false;
            if (elements > 0) f(p, p + (uintptr_t)elements * width[code]);
        }
        return n >= 0;
    }
};

// Whether spans in order are apart; `at` is the first of two that are not.
bool in_order_apart(const std::vector<Span> &spans, size_t &at) {
    for (at = 0; at + 1 < spans.size(); ++at)
        if (spans[at + 1].first < spans[at].end) return false;
    return true;
}

// Adds what a list's tensors have: in order, and as one where they touch or overlap each other.
void add_spans(const ReadList &list, std::vector<Span> &spans) {
    const size_t from = spans.size();
    list.each([&](uintptr_t p, uintptr_t end) { spans.push_back({p, end, list.number}); });
    const auto begin = spans.begin() + (std::ptrdiff_t)from;
    if (!std::is_sorted(begin, spans.end())) std::sort(begin, spans.end());
    size_t to = from;
    for (size_t k = from; k < spans.size(); ++k) {
        if (to > from && spans[k].first <= spans[to - 1].end) spans[to - 1].end = std::max(spans[to - 1].end, spans[k].end);
        else spans[to++] = spans[k];
    }
    spans.resize(to);
}

// Sorts spans whose runs, from each of `starts` to the next, are in order.
void merge_runs(std::vector<Span> &spans, std::vector<size_t> starts) {
    std::vector<Span> other(spans.size());
    for (; starts.size() > 1; spans.swap(other)) {
        std::vector<size_t> next;
        const auto at = [&](size_t k) { return spans.begin() + (std::ptrdiff_t)(k < starts.size() ? starts[k] : spans.size()); };
        for (size_t k = 0; k < starts.size(); k += 2) {
            next.push_back(starts[k]);
            std::merge(at(k), at(k + 1), at(k + 1), at(k + 2), other.begin() + (std::ptrdiff_t)starts[k]);
        }
        starts.swap(next);
    }
}

// apart(names, lists): that no tensor of a list overlaps one of another; lists as read() gives them, or None. Of lists that
// are their pointers alone (bytes) only that no two have the same at a place.
PyObject *apart(PyObject *, PyObject *args) try {
    PyObject *names, *lists;
    if (!PyArg_ParseTuple(args, "O!O!", &PyTuple_Type, &names, &PyTuple_Type, &lists)) return nullptr;
    const Py_ssize_t n = PyTuple_GET_SIZE(lists);
    if (PyTuple_GET_SIZE(names) != n) return fail("as many names as lists are wanted");
    Py_ssize_t size = -1;
    std::vector<ReadList> read;
    std::vector<Span> spans;
    for (Py_ssize_t a = 0; a < n; ++a) {
        PyObject *list = PyTuple_GET_ITEM(lists, a);
        if (!PyUnicode_Check(PyTuple_GET_ITEM(names, a))) return fail("names are wanted");
        if (list == Py_None) continue;
        if (PyTuple_Check(list)) {
            // From the first byte of any to the last: lists of one buffer each are told apart by these.
            Span all{UINTPTR_MAX, 0, a};
            read.emplace_back(list, a);
            if (!read.back().each([&](uintptr_t p, uintptr_t end) { all.first = std::min(all.first, p), all.end = std::max(all.end, end); }))
                return fail("lists must be as they were read");
            if (all.end > 0) spans.push_back(all);
            continue;
        }
        if (!PyBytes_Check(list)) return fail("bytes are wanted");
        if (size >= 0 && PyBytes_GET_SIZE(list) != size) return fail("lists must be as long as each other");
        size = PyBytes_GET_SIZE(list);
    }
    std::sort(spans.begin(), spans.end());
    size_t at = 0;
    if (!in_order_apart(spans, at)) {
        std::vector<size_t> starts;
        size_t total = 0;
        for (const ReadList &list : read) total += (size_t)list.n;
        spans.clear();
        spans.reserve(total);
        for (const ReadList &list : read) {
            starts.push_back(spans.size());
            add_spans(list, spans);
        }
        merge_runs(spans, std::move(starts));
        if (!in_order_apart(spans, at)) {
            const Py_ssize_t x = spans[at].list, y = spans[at + 1].list;
            return PyErr_Format(PyExc_ValueError, "%U and %U must not overlap each other", PyTuple_GET_ITEM(names, std::min(x, y)),
                                PyTuple_GET_ITEM(names, std::max(x, y)));
        }
    }
    for (Py_ssize_t a = 0; a < n; ++a)
        for (Py_ssize_t b = a + 1; b < n; ++b) {
            PyObject *x = PyTuple_GET_ITEM(lists, a), *y = PyTuple_GET_ITEM(lists, b);
            if (!PyBytes_Check(x) || !PyBytes_Check(y)) continue;
            for (Py_ssize_t k = 0; k + (Py_ssize_t)sizeof(uintptr_t) <= size; k += sizeof(uintptr_t)) {
                uintptr_t p, q;
                std::memcpy(&p, PyBytes_AS_STRING(x) + k, sizeof p);
                std::memcpy(&q, PyBytes_AS_STRING(y) + k, sizeof q);
                if (p != 0 && p == q) {
                    PyErr_Format(PyExc_ValueError, "%U and %U must not overlap each other", PyTuple_GET_ITEM(names, a), PyTuple_GET_ITEM(names, b));
                    return nullptr;
                }
            }
        }
    Py_RETURN_NONE;
} catch (const std::exception &e) {
    return fail(e.what());
}

// wrote(list, ..): raises the versions of lists of tensors (or None) that a call has written through their pointers, as torch
// does for its own operations in place: a graph that has saved one then refuses to use it.
PyObject *wrote(PyObject *, PyObject *lists) try {
    for (Py_ssize_t a = 0; a < PyTuple_GET_SIZE(lists); ++a) {
        if (PyTuple_GET_ITEM(lists, a) == Py_None) continue;
        const Held list{PySequence_Fast(PyTuple_GET_ITEM(lists, a), "a list of tensors is wanted")};
        if (!list.p) return nullptr;
        for (Py_ssize_t k = 0; k < PySequence_Fast_GET_SIZE(list.p); ++k) {
            PyObject *item = PySequence_Fast_GET_ITEM(list.p, k);
            if (!THPVariable_Check(item)) return fail("a list of tensors is wanted");
            const at::Tensor &t = THPVariable_Unpack(item);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
    }
    Py_RETURN_NONE;
} catch (const std::exception &e) {
    return fail(e.what());
}

std::string shape_of(long long rows, long long cols) {
    auto side = [](long long n) { return n < 0 ? std::string("any") : std::to_string(n); };
    return "(" + side(rows) + ", " + side(cols) + ")";
}

// The tensor that an argument is, of a type among `types` on `device` (-1: any); null with an error set.
const at::Tensor *tensor_of(PyObject *item, const char *name, int types, int device) {
    if (!THPVariable_Check(item)) {
        fail(std::string(name) + " must be a tensor");
        return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(item);
    const int code = code_of(t);
    if (!t.is_cuda() || t.layout() != at::kStrided || code < 0 || !(types >> code & 1)) {
        fail(std::string(name) + " must be a device tensor of " + names_of(types));
        return nullptr;
    }
    if (device >= 0 && t.get_device() != device) {
        fail(std::string(name) + " must be on cuda:" + std::to_string(device));
        return nullptr;
    }
    return &t;
}

// matrix(tensor, name, types, device, rows, cols) -> (pointer, code, rows, cols, row stride, device)
//   rows of contiguous elements; a size of -1 is any.
PyObject *matrix(PyObject *, PyObject *args) {
    PyObject *item;
    const char *name;
    int types, device;
    long long rows, cols;
    if (!PyArg_ParseTuple(args, "OsiiLL", &item, &name, &types, &device, &rows, &cols)) return nullptr;
    try {
        const at::Tensor *t = tensor_of(item, name, types, device);
        if (!t) return nullptr;
        if (t->dim() != 2 || (rows >= 0 && t->size(0) != rows) || (cols >= 0 && t->size(1) != cols))
            return fail(std::string(name) + " must be a matrix of shape " + shape_of(rows, cols));
        rows = t->size(0);
        cols = t->size(1);
        if (cols > 1 && t->stride(1) != 1) return fail(std::string(name) + " must have contiguous rows");
        // a stride is only used between rows; torch leaves it free where there is one
        const long long stride = rows > 1 ? t->stride(0) : (cols > 1 ? cols : 1);
        return Py_BuildValue("KiLLLi", (unsigned long long)reinterpret_cast<uintptr_t>(t->data_ptr()), code_of(*t), rows, cols, stride,
                             (int)t->get_device());
    } catch (const std::exception &e) {
        return fail(std::string(name) + ": " + e.what());
    }
}

// vector(tensor, name, types, device, elements) -> (pointer, code, elements): contiguous; -1 elements are any.
PyObject *vector(PyObject *, PyObject *args) {
    PyObject *item;
    const char *name;
    int types, device;
    long long n;
    if (!PyArg_ParseTuple(args, "OsiiL", &item, &name, &types, &device, &n)) return nullptr;
    try {
        const at::Tensor *t = tensor_of(item, name, types, device);
        if (!t) return nullptr;
        if (!t->is_contiguous() || (n >= 0 && t->numel() != n))
            return fail(std::string(name) + " must be contiguous" + (n >= 0 ? " with " + std::to_string(n) + " elements" : std::string()));
        return Py_BuildValue("KiL", (unsigned long long)reinterpret_cast<uintptr_t>(t->data_ptr()), code_of(*t), (long long)t->numel());
    } catch (const std::exception &e) {
        return fail(std::string(name) + ": " + e.what());
    }
}

PyMethodDef methods[] = {{"matrix", matrix, METH_VARARGS, "Pointer, type, sizes and row stride of a matrix."},
                         {"vector", vector, METH_VARARGS, "Pointer, type and size of a contiguous tensor."},
                         {"apart", apart, METH_VARARGS, "Refuses lists whose tensors overlap."},
                         {"read", read, METH_VARARGS, "Pointers, types and sizes of a list of tensors."},
                         {"wrote", wrote, METH_VARARGS, "Raises the versions of lists of tensors."}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lists() { return PyModule_Create(&module); }
