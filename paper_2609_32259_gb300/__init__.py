"""GB300 (sm_103a) implementation of HeteroFold's prefill-free K/V transfer.

Modules:
  binding   ctypes binding of include/heterofold.h (libheterofold.so)
  pipeline  TransferJob: torch-allocated buffers + the ABI calls of a transfer;
            KVCache: a receiver's cache, appended to, read and attended over
  receiver  ReceiverSteps: a receiver's next tokens behind a transferred context
            (python -m paper_2609_32259_gb300.receiver runs one)
  workloads seeded synthetic inputs shaped like the paper's model pairs
  build     nvcc build of libheterofold.so (in-tree)

Importing the package loads nothing; the CUDA library is loaded on first use
and its absence is an error, never a fallback.
"""

__all__ = ["binding", "pipeline", "receiver", "workloads", "build"]
