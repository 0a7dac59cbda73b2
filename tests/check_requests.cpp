// The host-only checks of requests, as functions that a test can call without a device.
#include "qsv_requests.h"

extern "C" const char* request_sample(const qsv_sample_req* q, int n, int64_t batch) { return qsv::check_sample(q, n, batch); }
extern "C" const char* request_distill(const qsv_distill_req* q, const qsv_teacher* t) { return qsv::check_distill(q, t); }
