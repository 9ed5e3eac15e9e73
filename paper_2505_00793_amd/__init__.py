"""MixFlow-MG meta-gradients on MI355X: HIP kernels behind a C ABI (include/mfmg.h).

``paper_2505_00793_amd._lib`` is the ctypes binding; ``build`` compiles the
library in-tree.  Importing the package does not load the library.
"""
from . import _lib  # noqa: F401
from ._lib import Attention, Problem, lib, make_attn_desc, make_desc, mfmg_seq_plan, MfmgError  # noqa: F401
