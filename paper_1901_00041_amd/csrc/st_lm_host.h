// What the host sources of the operators of language models share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace st {

// Makes a plan's device the current one for a call, and puts back the caller's.
struct OnDevice {
  hipError_t error = hipSuccess;
  int before = -1;
  explicit OnDevice(int device) {
    int now = -1;
    error = hipGetDevice(&now);
    if (error == hipSuccess && now != device) {
      error = hipSetDevice(device);
      if (error == hipSuccess) before = now;
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
};

// Whether what is queued on a stream becomes part of a graph.
inline hipError_t is_captured(void* hip_stream, bool* captured) {
  hipStreamCaptureStatus now = hipStreamCaptureStatusNone;
  const hipError_t e = hip_stream ? hipStreamIsCapturing((hipStream_t)hip_stream, &now) : hipSuccess;      // the default stream cannot be
  *captured = now != hipStreamCaptureStatusNone;
  return e;
}

// A launch holds fewer than 2^32 threads, which its largest workgroups of 512 reach with this many.
constexpr int64_t kMostWorkgroups = (int64_t)1 << 23;

// What a matrix of rows spans; whether two of them share a byte.
struct Span {
  uintptr_t at;
  int64_t rows, row_bytes, turn;     // turn: bytes from a row to the next
  uintptr_t end() const { return at + (uintptr_t)((rows - 1) * turn + row_bytes); }
};
inline bool overlap(const Span& a, const Span& b) {
  if (a.rows <= 0 || b.rows <= 0 || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.turn == b.turn) {             // columns of one matrix that lie beside each other
    const int64_t off = (((int64_t)b.at - (int64_t)a.at) % a.turn + a.turn) % a.turn;      // where b's rows start in a's
    if (off >= a.row_bytes && off + b.row_bytes <= a.turn) return false;
  }
  return true;
}

}  // namespace st
