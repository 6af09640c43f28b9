// What the library's translation units share of the calling thread's records.
#pragma once

namespace tconv {

// Clears the text of the last CUDA error at the start of a call.
void call_begins();
// After `n` kernel launches of variant `name`: counts them and returns TCONV_OK, or the launch's error with its text kept.
int launched(int n, const char* name);

}  // namespace tconv
