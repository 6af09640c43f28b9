// What the extension module's translation units share.
#pragma once
#include <torch/extension.h>

#include <utility>

namespace tconv_torch {

// Raises TconvError; callable without the GIL (the autograd engine's threads).
[[noreturn]] void fail(int rc, const char* where);

// Rows and values of a row of a tensor's 8-bit form (tconv.h).
std::pair<int64_t, int64_t> q8_rows(at::IntArrayRef shape);
// Raises ValueError unless these are the codes and scales of such rows, dense and on `like`'s device.
struct Q8 {
    at::Tensor codes, scales;
};
Q8 q8_empty(const at::Tensor& like, int64_t rows, int64_t inner);
void q8_check(const Q8& q, const at::Tensor& like, int64_t rows, int64_t inner);

// Adds the functions of torch_seq.cpp.
void bind_seq(pybind11::module& m);

}  // namespace tconv_torch
