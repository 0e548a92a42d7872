"""MI355X-native QUASAR per-step loss-aware reconstruction.

The compute path is the HIP library ``libquasar.so`` (C ABI, ``include/quasar.h``);
``paper_2608_13966_amd.quasar`` is its thin ctypes binding and
``paper_2608_13966_amd.synth`` draws the seeded synthetic workloads.  ``ops``
has the operators around the reconstruction (``include/quasar_ops.h``), ``ste``
the trainable layer and their autograd forms, and ``example`` runs them together.
Importing this package loads nothing; the library is opened on first use.
"""
__all__ = ["example", "ops", "quasar", "ste", "synth"]
