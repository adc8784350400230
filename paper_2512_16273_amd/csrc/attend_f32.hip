#include "attend_launch.h"

template hipError_t tslt::launch_attend<float>(const tslt::AttendParams&, int, hipStream_t);
