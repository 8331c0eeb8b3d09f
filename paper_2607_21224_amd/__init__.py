"""MI355X-native (gfx950) implementation of the reconcile hot path of
Controlled Periodic Data Parallelism (CPDP) with SlowMo, and of the 8-bit
activation path of the models it trains.

Submodules
  cpdp   ctypes binding of the C ABI in include/cpdp.h (libcpdp.so)
  state  HBM-resident replica state (flat layout), the host cadence driving
         it, step tables and HIP-graph capture, checkpoint/resume
  multi  the same for a model held as separate tensors (multi-tensor plans)
  q8     binding of include/cpdp_q8.h (libcpdp_q8.so, through the extension module
         _q8): norm, products, activations and the loss on rows of 8-bit numbers,
         and their backward passes
  layer  the MLP half of a transformer block, and a model's head with its loss, on
         that path, with their weights and gradients in replica rows
  build  hipcc build of the shared libraries

Importing ``cpdp`` or ``q8`` (directly or through ``state``) raises ImportError
when its HIP library is not built: there is no CPU fallback.
"""
__all__ = ["cpdp", "state", "multi", "q8", "layer", "build"]
