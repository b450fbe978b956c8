#include "sttm_queries_kernel.h"

template void sttm::launch_queries<2>(const sttm::QueryArgs&, const sttm::KeyArgs&, bool, hipStream_t);  // f16
