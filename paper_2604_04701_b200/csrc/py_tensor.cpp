// Reads a torch tensor's address, shape and strides from the object itself.  Asked for as Python attributes they cost a third of a
// microsecond a tensor, which for a norm at a decode step with its six tensors is as much as the launch (5.6 -> 3.6 us a call in all).
#include "py_tensor.h"

#include <torch/csrc/autograd/python_variable.h>

int tensor_info_of(PyObject *obj, tensor_info *out) {
    if (!THPVariable_CheckExact(obj)) return 0;
    try {
        const at::Tensor &t = THPVariable_Unpack(obj);
        const auto type = t.scalar_type();
        out->dtype = type == at::kHalf ? TENSOR_F16 : type == at::kFloat ? TENSOR_F32 : type == at::kInt ? TENSOR_I32 : TENSOR_OTHER;
        out->device = t.is_cuda() ? (int)t.get_device() : -1;
        const auto sizes = t.sizes(), strides = t.strides();
        out->dim = sizes.size() > 3 ? 4 : (int)sizes.size();
        for (int i = 0; i < out->dim && i < 3; ++i) {
            out->size[i] = sizes[i];
            out->stride[i] = strides[i];
        }
        out->ptr = t.data_ptr();
        return 1;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return -1;
    } catch (...) {
        PyErr_SetString(PyExc_ValueError, "a tensor that cannot be read");
        return -1;
    }
}
