// What the native parts of the binding share: the current stream of a device, and
// the look-up of a cached workspace (tilefuse.py makes them and says how they are
// kept).
#pragma once

#include <Python.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>

#include <cstdint>

namespace tf_binding {

// A reference held until the end of the scope.
struct Held {
    PyObject* o = nullptr;
    ~Held() { Py_XDECREF(o); }
};

// The current stream of the tensors' device, from `current` (device index -> handle).
// False: a Python error, or not the current device, to which a launch would go
// whatever its stream is (the general path makes it current).
inline bool stream_of(PyObject* current, int dev, void*& stream) {
    if (c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index() != dev) return false;
    const Held index{PyLong_FromLong(dev)};
    const Held handle{index.o ? PyObject_CallOneArg(current, index.o) : nullptr};
    if (!handle.o) return false;
    stream = PyLong_AsVoidPtr(handle.o);
    return !PyErr_Occurred();
}

// The runtime's query of a stream's capture: its state (0: none) and its number.
using CaptureFn = int (*)(void* stream, int* state, unsigned long long* number);

// The workspace kept in `cached` under (device, stream, capture), or none (null).
// False: not to be told here, or a Python error.
inline bool find_workspace(PyObject* cached, CaptureFn capture, int dev, void* stream, Held& found) {
    int state = 0;
    unsigned long long number = 0;
    // (the default stream cannot be captured)
    if (stream && (!capture || capture(stream, &state, &number) != 0)) return false;
    const Held key{Py_BuildValue("(iKK)", dev, (unsigned long long)(uintptr_t)stream, state ? number + 1 : 0ULL)};
    if (!key.o) return false;
    found.o = Py_XNewRef(PyDict_GetItemWithError(cached, key.o));
    return found.o || !PyErr_Occurred();
}

}  // namespace tf_binding
