"""MI355X-native batched serving simulator for AlpaServe-style placement search.

Subpackages and modules:
  workload/   seeded synthetic inputs: Gamma arrival traces (C library
              libas_gen.so) and the problem builders for the five workloads
  csrc/       HIP kernels for gfx950 and the C-ABI library libalpaserve_sim.so
  sim.py      thin ctypes binding of the C-ABI (argument marshalling only)
  ops.py      binding of the operators of a served model: norms and linear
              layers in 8 bits, a 4-bit paged cache, attention over it and over
              packed prompts, pages of a pool, eviction
  served.py   a served decoder block of these operators, requests that come and
              go, measured latency and bytes, and the placement that follows
  build.py    compiles the two native libraries in-tree

Importing this package loads nothing native; sim.py loads the HIP library on
first use and raises if it is not built.
"""
