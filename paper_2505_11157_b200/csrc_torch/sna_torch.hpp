// Shared by the native autograd functions.
#pragma once
#include <torch/extension.h>

namespace sna_torch {

// Raises sna.SnaError for a failing status of the C ABI.
void check(int status);
// The operators around the attention of a layer (sna_layer.cpp).
void bind_layer(pybind11::module_& m);

}  // namespace sna_torch
