"""Batched graph-driven tile-graph simulation (GPU-Tile-Sim backend) for GB300.

* ``workloads`` -- seeded synthetic tile graphs and design-point tables;
* ``gts``       -- binding of libgts (include/gts.h), the CUDA implementation;
* ``serving``   -- operators of a decode step: rotary positions, append to a
                   paged cache, attention over a shared prefix;
* ``decode``    -- a decode step run with them, and its tile graph;
* ``build``     -- nvcc build of libgts for sm_103a.
"""
