"""Host offload of saved records and their prefetch during the backward walk (host orchestration only:
copies, streams and events; no arithmetic).

Section 4.3 of the paper: the activations a serving step leaves behind may not fit next to the serving
state, so they are copied to pinned host memory on a stream of their own and brought back when the trainer
needs them; Section 4.3.2: the backward pass consumes them one layer at a time, from the output layer to the
input layer, so the copy of layer l-1 can run while layer l computes.

`RecordStore` keeps one pinned host copy per layer and two device staging slots.  `offload(l, record)`
enqueues the device-to-host copies of layer l behind the work already on the caller's stream.
With bits=8 a record crosses the link, and waits in host memory, as int8 codes with a scale for every 64 elements
(alch_capture_gather_q8 in front of the copies out, alch_record_expand behind those back): 53 % of the bytes of
bf16.  O and LSE are not kept then but recomputed by the backward, so that they belong to the queries, keys
and values that were read back.
`prefetching_backward(...)` runs `alch_stack_backward` (or its adapter variant) with every layer's record
pointers aimed at the staging slot l % 2 and a `layer_ready` hook that (1) makes the compute stream wait
for layer l's host-to-device copy and (2) lets the copy of layer l-1 start as soon as the kernels of layer
l+1 -- the previous user of that slot -- have finished.
"""
import torch

from . import binding as B

KEYS = B.RECORD_KEYS + ("LSE",)


def _coded(like, **kw):
    """Room for a tensor [rows, width] in 8 bits: (codes, scales)."""
    rows, width = like.shape
    return (torch.empty((rows, width), dtype=torch.int8, **kw), torch.empty((rows, -(-width // B.Q8_GROUP)), dtype=torch.float32, **kw))


class RecordStore:
    def __init__(self, n_layers, example_record, keys=KEYS, bits=16):
        """example_record: dict of device tensors with the shapes and dtypes of one layer's record.  bits: 16 keeps the
        tensors as they are, 8 all but O and LSE in 8 bits."""
        if bits not in (8, 16):
            raise ValueError("bits = %s: 16 or 8" % (bits,))
        self.keys = tuple(k for k in keys if example_record.get(k) is not None and not (bits == 8 and k in ("O", "LSE")))
        self.n_layers, self.bits = n_layers, bits
        if bits == 8:
            rows = {k: example_record[k].shape[0] for k in self.keys}
            if len(set(rows.values())) > 1:
                raise ValueError("tensors of different numbers of rows: %s" % rows)
            some = example_record[self.keys[0]] if self.keys else None
            self.batch = B.Batch([0, some.shape[0]], device=some.device) if self.keys else None
            # codes and scales on their way to a slot: both directions use a stream in order, one place is enough
            self.coded = {k: _coded(example_record[k], device=example_record[k].device) for k in self.keys}
            self.host = [{k: _coded(example_record[k], pin_memory=True) for k in self.keys} for _ in range(n_layers)]
        else:
            self.host = [{k: torch.empty(example_record[k].shape, dtype=example_record[k].dtype, pin_memory=True)
                          for k in self.keys} for _ in range(n_layers)]
        self.slots = [{k: torch.empty_like(example_record[k]) for k in self.keys} for _ in range(2)]
        self.copy_stream = torch.cuda.Stream()
        self.bytes_per_layer = sum(t.numel() * t.element_size() for h in self.host[:1] for e in h.values() for t in (e if bits == 8 else (e,)))

    def offload(self, layer, record, stream=None):
        """Device -> pinned host, asynchronous, ordered after what `stream` holds now."""
        stream = stream or torch.cuda.current_stream()
        coded = None
        if self.bits == 8 and self.keys:
            coded = dict(zip(self.keys, B.alch_capture_gather_q8(self.batch, [record[k] for k in self.keys], stream=stream)))
            for k in self.keys:
                record[k].record_stream(stream)
        done = torch.cuda.Event()
        done.record(stream)
        self.copy_stream.wait_event(done)
        with torch.cuda.stream(self.copy_stream):
            for k in self.keys:
                pairs = [(self.host[layer][k], record[k])] if coded is None else zip(self.host[layer][k], coded[k])
                for to, of in pairs:
                    to.copy_(of, non_blocking=True)
                    of.record_stream(self.copy_stream)

    def _fetch(self, layer):
        """Pinned host -> staging slot layer % 2 on the copy stream; returns the event of its completion."""
        with torch.cuda.stream(self.copy_stream):
            slot, host = self.slots[layer % 2], self.host[layer]
            if self.bits == 8:
                for k in self.keys:
                    for to, of in zip(self.coded[k], host[k]):
                        to.copy_(of, non_blocking=True)
                B.alch_record_expand([self.coded[k] for k in self.keys], outs=[slot[k] for k in self.keys], stream=self.copy_stream)
            else:
                for k in self.keys:
                    slot[k].copy_(host[k], non_blocking=True)
            ev = torch.cuda.Event()
            ev.record(self.copy_stream)
        return ev

    def prefetching_backward(self, backward, stream=None):
        """backward(saved_layers, hooks) must call alch_stack_backward[_lora] with those two arguments on `stream`.
        Returns what it returns."""
        stream = stream or torch.cuda.current_stream()
        L = self.n_layers
        ready = {}
        # the walk starts at layer L-1: its record and the next one go out first
        self.copy_stream.wait_stream(stream)
        for l in (L - 1, L - 2):
            if l >= 0:
                ready[l] = self._fetch(l)

        def layer_ready(_user, l):
            # kernels of layer l+1 are enqueued: once they are done its slot may be overwritten by layer l-1
            if l + 1 < L and l - 1 >= 0:
                freed = torch.cuda.Event()
                freed.record(stream)
                self.copy_stream.wait_event(freed)
                ready[l - 1] = self._fetch(l - 1)
            stream.wait_event(ready[l])
            return 0

        saved = [self.slots[l % 2] for l in range(L)]
        out = backward(saved, (layer_ready, None))
        # the staging slots must outlive the kernels that read them
        self.copy_stream.wait_stream(stream)
        return out
