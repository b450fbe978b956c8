#include "sttm_queries_kernel.h"

template void sttm::launch_queries<0>(sttm::QueryJobs&, bool, hipStream_t);  // f32
