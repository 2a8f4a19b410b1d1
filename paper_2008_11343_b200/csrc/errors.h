// The calling thread's message buffer (apms_last_error(NULL)), shared by the library's translation units.
#pragma once

constexpr int kThreadErrorBytes = 256;
__attribute__((visibility("hidden"))) char* apms_thread_error();
