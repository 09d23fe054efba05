"""Fused multi-tenant convolution ("super-kernel") for MI355X / gfx950.

`synth` (seeded workloads, numpy only) can be imported anywhere.  The bindings (`st_conv`, and `st_lm` for the
operators of language models) load the HIP shared library on first use and fail loudly if it has not been built.
"""
__all__ = ["synth", "st_conv", "st_lm"]
