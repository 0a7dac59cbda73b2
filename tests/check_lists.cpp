// The host-only checks of qsv_adjust and of the calls on lists of tensors, as functions that a test can call without a device.
#include "qsv_requests.h"

extern "C" const char* request_adjust(const qsv_adjust_req* q) { return qsv::check_adjust(q); }
extern "C" const char* request_adjust_grad(const qsv_adjust_req* q, const qsv_adjust_grad_req* g) { return qsv::check_adjust_grad(q, g); }
extern "C" const char* request_clip(const qsv_tensor* g, const qsv_tensor* o, int64_t n, double m) { return qsv::check_clip(g, o, n, m); }
extern "C" const char* request_adam(const qsv_adam_tensor* t, int64_t n, double m) { return qsv::check_adam_list(t, n, m); }
extern "C" const char* request_clip_norm(const qsv_tensor* g, const qsv_tensor* o, int64_t n, double m, const float* norm) { return qsv::check_clip(g, o, n, m, norm); }
extern "C" const char* request_adam_norm(const qsv_adam_tensor* t, int64_t n, double m, const float* norm) { return qsv::check_adam_list(t, n, m, norm); }
