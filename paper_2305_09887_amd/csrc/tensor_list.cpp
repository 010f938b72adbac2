// Host code of the binding: what a call that takes many tensors has to know of each of them.  Asked one by one from Python, type, device, layout, length and address take
// half a microsecond a tensor: clipping 281 gradients of a small model into new ones 147 us, of which the GPU worked 15.  Called with the interpreter's lock held.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

// the torch whose classes this was compiled for
extern "C" const char *tma_lists_torch() { return TMA_TORCH; }

enum { kRead = 0, kNoTensor = 1, kOtherType = 2, kOtherDevice = 3, kNotDense = 4, kOtherLength = 5 };

// Addresses and lengths of `n` tensors, a list or a tuple: dense, of fp32 or bf16 (dtype 0, 1), on device `device` (-1: the host's memory).  same: lengths are given, and
// the tensors' have to be those.  *at: the tensor that is refused.
extern "C" int tma_read_tensors(PyObject *tensors, int32_t n, int32_t dtype, int32_t device, int32_t same, uint64_t *addresses, int64_t *lengths, int32_t *at)
{
    *at = 0;
    if (!PyList_Check(tensors) && !PyTuple_Check(tensors)) return kNoTensor;
    if (PySequence_Fast_GET_SIZE(tensors) != n) return kOtherLength;
    PyObject **items = PySequence_Fast_ITEMS(tensors);
    const at::ScalarType type = dtype == 1 ? at::kBFloat16 : at::kFloat;
    try {
        for (int32_t i = 0; i < n; ++i) {
            *at = i;
            if (!THPVariable_Check(items[i])) return kNoTensor;
            const at::Tensor &t = THPVariable_Unpack(items[i]);
            if (t.scalar_type() != type) return kOtherType;
            if ((t.is_cpu() ? -1 : t.is_cuda() ? int32_t(t.get_device()) : -2) != device) return kOtherDevice;
            if (t.layout() != c10::kStrided || !t.is_contiguous()) return kNotDense;
            if (same && t.numel() != lengths[i]) return kOtherLength;
            lengths[i] = t.numel();
            addresses[i] = reinterpret_cast<uint64_t>(t.data_ptr());
        }
    } catch (...) {      // (a tensor without memory of its own)
        return kNotDense;
    }
    return kRead;
}
