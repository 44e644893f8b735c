/* What the binding reads of a torch tensor. */
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef enum { TENSOR_F16 = 0, TENSOR_F32 = 1, TENSOR_I32 = 2, TENSOR_OTHER = 3 } tensor_dtype; /* the first two as MUXQ_OUT_* */
typedef struct {
    void *ptr;
    int64_t size[3], stride[3];
    int dtype, device, dim; /* device: -1 on the CPU; dim: 4 stands for more than 3 */
} tensor_info;

#ifdef __cplusplus
extern "C" {
#endif
/* 1: read; 0: not a plain torch tensor (nothing read); -1: a Python exception is set */
int tensor_info_of(PyObject *t, tensor_info *out);
#ifdef __cplusplus
}
#endif
