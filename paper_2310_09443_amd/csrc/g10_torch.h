// What the marshalling of torch tensors shares: checks that raise ValueError, streams, workspaces.
#pragma once

#include <torch/extension.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>

#include <math.h>
#include <optional>
#include <unordered_map>
#include <vector>

#include "g10_ops.h"

namespace py = pybind11;
typedef std::optional<at::Tensor> Maybe;

static inline void check(int rc, const char* what) {
  if (!rc) return;
  TORCH_CHECK_VALUE(rc != G10_EINVAL, what, " refuses these sizes or numbers");       // (what the checks here leave to the library's)
  py::object error = py::module_::import("paper_2310_09443_amd.binding").attr("G10Error");
  PyErr_SetObject(error.ptr(), error(rc, what).ptr());
  throw py::error_already_set();
}

static inline int type_of(at::ScalarType t) {
  return t == at::kFloat ? G10_F32 : t == at::kHalf ? G10_F16 : t == at::kBFloat16 ? G10_BF16 : -1;
}

static inline void on_device(const at::Tensor& t, const char* name, const at::Device* dev) {
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must lie in GPU memory");
  TORCH_CHECK_VALUE(!dev || t.device() == *dev, name, " must lie on the device of the other tensors");
}

static inline void* stream_of(const at::Device& dev) { return (void*)c10::hip::getCurrentHIPStream(dev.index()).stream(); }

static inline at::Tensor room(uint64_t bytes, const at::Device& dev) {
  return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(dev));
}

// (csrc/g10_torch_layer.cpp)
void layer_calls(py::module_& m);
