#include "sttm_queries_kernel.h"

template void sttm::launch_queries<0>(const sttm::QueryArgs&, const sttm::KeyArgs&, bool, hipStream_t);  // f32
