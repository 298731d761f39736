// A stand-in for the CUDA runtime's host calls that writes down what it is asked for: which stream waits for which event,
// what is freed when.
#pragma once

#include <cstdint>
#include <map>
#include <string>
#include <vector>

#include <cuda_runtime_api.h>

extern std::vector<std::string> calls;                       // what was asked for
extern std::map<cudaStream_t, unsigned long long> captures;  // streams under capture, and the capture's id
extern long next_handle;                                     // of an event or a buffer
extern bool no_memory;                                       // operator new throws
bool noted(const char *what, const void *a, const void *b);
