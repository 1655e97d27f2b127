#include "sig_window.h"

// The gradient's terms u are products of an upstream gradient of any size with probabilities, and out of float16's range long before what they add
// up to is: its products are float32's.
hipError_t sig::launch_window_f16(const WindowArgs &A, WindowPass pass, hipStream_t st)
{
    return pass == WINDOW_FORWARD ? launch_window<f16, f16>(A, pass, st) : launch_window<f16, float>(A, pass, st);
}
