#include "sig_window.h"

hipError_t sig::launch_window_f16(const WindowArgs &A, WindowPass pass, hipStream_t st) { return launch_window<f16>(A, pass, st); }
