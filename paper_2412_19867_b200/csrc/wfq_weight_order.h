// Whether a product may fetch weights before the kernel in front of it has ended (host bookkeeping of one layer).
//
// A product's launch may begin as soon as the kernel in front of it on its stream lets it, and the kernel that writes the
// weights does so at its start.  Behind that kernel, on its own stream, the next product therefore waits for it; once a
// launch on that stream has waited, whatever follows there begins behind the weights' last write.  On any other stream the
// caller has put an event or a synchronisation in between, which nothing passes; the first product there waits all the
// same.  A call under capture is only recorded: it waits when it is replayed, and tells nothing about now; and where a
// graph writes the weights its replays do so unseen, so that every product waits.
//
// Streams are told apart by their handles (cudaStreamGetId ends a capture).  NULL and cudaStreamLegacy are one stream; a
// handle that is used again for a new stream, and the per-thread one in another thread, only make a product wait.
#pragma once

namespace wfq {

class WeightOrder {
public:
    // Weights are written on this stream.
    void written(const void *stream, bool captured)
    {
        pending_ = true;
        stream_ = one(stream);
        waited_elsewhere_ = false;
        if (captured) by_graph_ = true;
    }
    // Is there a stream on which a product has to wait?
    bool pending() const { return pending_; }
    // May a product on this stream fetch weights early?
    bool settled(const void *stream) const
    {
        return !by_graph_ && (!pending_ || (waited_elsewhere_ && one(stream) != stream_));
    }
    // A product has been launched on this stream that waited for the kernel in front of it, or came behind one that did.
    void waited(const void *stream, bool captured)
    {
        if (captured) return;
        if (one(stream) == stream_) pending_ = false;
        else waited_elsewhere_ = true;
    }

private:
    bool pending_ = false, waited_elsewhere_ = false, by_graph_ = false;
    const void *stream_ = nullptr;
    static const void *one(const void *stream) { return stream == reinterpret_cast<const void *>(1) ? nullptr : stream; }
};

}  // namespace wfq
