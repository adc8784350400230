#include "attend_launch.h"

template hipError_t tslt::launch_attend<tslt::Bf16>(const tslt::AttendParams&, int, hipStream_t);
