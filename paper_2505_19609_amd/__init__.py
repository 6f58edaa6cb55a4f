"""MI355X-native packed varlen causal attention (forward + backward) for one
scheduled micro-batch of whole short sequences and context-parallel query
shards of long ones, and the operators that a training step runs around it:
rotary positions of its rows, norm, the loss over the vocabulary, attention to
a window of keys, the residual stream, and products with what follows them.  The
compute lives in ``csrc/`` (HIP, gfx950) behind the C ABI declared in
``include/skrull_*.h``; :mod:`.binding` only marshals arguments.  Nothing here
falls back to the CPU."""

__all__ = ["binding", "workloads"]
