// Lists of torch tensors as the arrays of addresses and sizes that libgsr takes.  Host code of the Python binding, called through ctypes with
// the interpreter lock held: a list of 115 tensors takes 1 us more than the call itself, against 28 us with the five attributes of each
// tensor read from Python.
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {
enum Refusal { FINE = 0, NOT_A_LIST, NOT_A_TENSOR, OTHER_DEVICE, OTHER_TYPE, NOT_CONTIGUOUS, OTHER_SIZE };
}

extern "C" {

// The tensors of a list or tuple of n: addresses[n], and their sizes to counts[n] or, with `compare`, held against it.  All of them contiguous, on
// GPU `device`, float32 (dtype 0) or bfloat16 (1).  Returns 0 or why not, *which: the first such tensor.
__attribute__((visibility("default"))) int gsr_marshal_list(PyObject* list, int64_t n, int device, int dtype, int compare,
                                                            uint64_t* addresses, int64_t* counts, int64_t* which) {
    *which = 0;
    try {
        const bool is_list = PyList_Check(list);
        if ((!is_list && !PyTuple_Check(list)) || (is_list ? PyList_GET_SIZE(list) : PyTuple_GET_SIZE(list)) != n) return NOT_A_LIST;
        const at::ScalarType type = dtype == 0 ? at::kFloat : at::kBFloat16;
        for (int64_t i = 0; i < n; ++i) {
            *which = i;
            PyObject* o = is_list ? PyList_GET_ITEM(list, i) : PyTuple_GET_ITEM(list, i);
            if (!THPVariable_Check(o)) return NOT_A_TENSOR;
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.defined() || t.layout() != at::kStrided) return NOT_A_TENSOR;
            if (!t.is_cuda() || t.get_device() != device) return OTHER_DEVICE;
            if (t.scalar_type() != type) return OTHER_TYPE;
            if (!t.is_contiguous()) return NOT_CONTIGUOUS;
            if (compare ? counts[i] != t.numel() : (counts[i] = t.numel(), false)) return OTHER_SIZE;
            addresses[i] = reinterpret_cast<uint64_t>(t.data_ptr());
        }
        return FINE;
    } catch (...) {
        return NOT_A_TENSOR;
    }
}

}  // extern "C"
