// The functions of the HIP runtime that host code with kernels refers to, doing
// nothing: for libraries whose kernels are never launched.
extern "C" {
int __hipPopCallConfiguration(...) { return 1; }
int __hipPushCallConfiguration(...) { return 1; }
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipRegisterFunction(...) {}
void __hipUnregisterFatBinary(void**) {}
int hipGetLastError() { return 1; }
int hipLaunchKernel(...) { return 1; }
}
