// What the extension module's translation units share.
#pragma once
#include <pybind11/pybind11.h>

namespace tconv_torch {

// Raises TconvError; callable without the GIL (the autograd engine's threads).
[[noreturn]] void fail(int rc, const char* where);

// Adds the functions of torch_seq.cpp.
void bind_seq(pybind11::module& m);

}  // namespace tconv_torch
