// The buffers of batches and calls that were given back (calvo_window.hip): which one is used again, when one is made, when one goes.  No device types here.
//
// A buffer that is given back is used again behind the launches that read it, on the same stream, so nobody waits for them; only its pinned source must have
// been read before it is written again.  A few of a size are used in turn, so that a program that is some steps ahead of the device finds one that
// has been.
//
// Giving back never frees, because that waits for the device.  Buffers go where one has to be made anyway: those that are too small for it, the smallest
// first, until few are left.  Sizes are powers of two (above 16 MiB multiples of that), so a batch whose contexts grow makes a few per doubling
// (128 requests of 300 to 33000 tokens, 16000 steps, three of them ahead of the device: 9 in all).
#pragma once
#include <algorithm>
#include <cstddef>
#include <mutex>
#include <new>
#include <vector>

namespace calvo {

constexpr size_t kStepDevMin = 65536, kStepHostMin = 16384;

inline size_t step_buf_size(size_t bytes, size_t least) {
  constexpr size_t kBig = (size_t)16 << 20;
  if (bytes > kBig) return (bytes + kBig - 1) / kBig * kBig;
  size_t n = least;
  while (n < bytes) n *= 2;
  return n;
}

// Buf: d_bytes, h_bytes, pending (its source may be unread).  Dev: int make(Buf&) for the sizes in it, void free(Buf&) (both may wait for the device),
// bool was_read(Buf&), int wait(Buf&); ints are 0 or an error.
template <class Buf>
class StepBufs {
 public:
  static constexpr int kInTurn = 4;
  static constexpr size_t kKeep = 16, kKeepBytes = (size_t)256 << 20;      // given back, while another is made

  // On an error `out` holds what was made of it.
  template <class Dev>
  int take(Dev& dev, size_t d_bytes, size_t h_bytes, Buf& out) {
    out = Buf();
    if (!find(dev, d_bytes, h_bytes, out)) {
      trim(dev, d_bytes, h_bytes, kKeep, kKeepBytes);
      out.d_bytes = step_buf_size(d_bytes, kStepDevMin);
      out.h_bytes = step_buf_size(h_bytes, kStepHostMin);
      const int rc = make(dev, out);
      if (rc != 0) return rc;
    }
    if (out.pending) {
      const int rc = dev.wait(out);
      if (rc != 0) return rc;
      out.pending = false;
    }
    return 0;
  }

  // Waits for nothing.  false: there is no host memory to list it
  bool give(Buf& b) {
    std::lock_guard<std::mutex> lk(mu_);
    try {
      list_.push_back(b);
    } catch (const std::bad_alloc&) {
      return false;
    }
    b = Buf();
    return true;
  }

  template <class Dev>
  void clear(Dev& dev) {
    std::vector<Buf> all;
    {
      std::lock_guard<std::mutex> lk(mu_);
      all.swap(list_);
    }
    for (Buf& b : all) dev.free(b);
  }

 private:
  // The smallest that is large enough and has been read; one that has not if there are several in turn already
  template <class Dev>
  bool find(Dev& dev, size_t d_bytes, size_t h_bytes, Buf& out) {
    std::lock_guard<std::mutex> lk(mu_);
    int best = -1, fit = 0;
    bool best_read = false;
    for (int i = 0; i < (int)list_.size(); i++) {
      Buf& b = list_[i];
      if (b.d_bytes < d_bytes || b.h_bytes < h_bytes) continue;
      fit++;
      if (b.pending && !best_read && dev.was_read(b)) b.pending = false;
      const bool better = best < 0 || (!b.pending && !best_read) || (!b.pending && b.d_bytes < list_[best].d_bytes);
      if (better) { best = i; best_read = !b.pending; }
    }
    if (best < 0 || !(best_read || fit >= kInTurn)) return false;
    out = list_[best];
    list_.erase(list_.begin() + best);
    return true;
  }

  // Frees buffers that are too small, the smallest first, until `keep` of them and `bytes` are left or all that are left would do.
  template <class Dev>
  void trim(Dev& dev, size_t d_bytes, size_t h_bytes, size_t keep, size_t bytes) {
    for (;;) {
      Buf b;
      {
        std::lock_guard<std::mutex> lk(mu_);
        size_t held = 0;
        int least = -1;
        for (int i = 0; i < (int)list_.size(); i++) {
          const Buf& x = list_[i];
          held += x.d_bytes + x.h_bytes;
          if (x.d_bytes >= d_bytes && x.h_bytes >= h_bytes) continue;
          if (least < 0 || x.d_bytes + x.h_bytes < list_[least].d_bytes + list_[least].h_bytes) least = i;
        }
        if (least < 0 || (list_.size() <= keep && held <= bytes)) return;
        b = list_[least];
        list_.erase(list_.begin() + least);
      }
      dev.free(b);
    }
  }

  // Where memory is short, what was given back goes first.
  template <class Dev>
  int make(Dev& dev, Buf& out) {
    const size_t d = out.d_bytes, h = out.h_bytes;
    int rc = dev.make(out);
    if (rc == 0) return rc;
    dev.free(out);
    clear(dev);
    out = Buf();
    out.d_bytes = d;
    out.h_bytes = h;
    return dev.make(out);
  }

  std::mutex mu_;
  std::vector<Buf> list_;
};

}  // namespace calvo
