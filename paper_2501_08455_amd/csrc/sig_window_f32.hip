#include "sig_window.h"

hipError_t sig::launch_window_f32(const WindowArgs &A, WindowPass pass, hipStream_t st) { return launch_window<float>(A, pass, st); }
