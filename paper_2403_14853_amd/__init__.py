"""MI355X-native sparse GNN hot path (SpMM, cached-transpose backward, SDDMM, FusedMM, attention over a graph) and the row-wise
operators around it (layer norm, log probabilities of labels).

Thin ctypes binding over the C-ABI library ``libisp.so`` (see ``include/isp.h``).  The binding
only marshals arguments: every step of the path runs in the library's HIP kernels.  PyTorch is
used for device memory and streams.  There is no CPU fallback: without the compiled library
the import of :mod:`paper_2403_14853_amd.binding` fails loudly.
"""
from .binding import (  # noqa: F401
    CSR, IspError, lib_path, load_library, csr_build, csr_build_workspace, csr_transpose_cached,
    csr_transpose_workspace, csr_values_changed, csr_alias, csr_alias_workspace, spmm, spmm_static_scratch, sddmm, fusedmm,
    fusedmm_backward, spmm_reduce, spmm_reduce_backward, attention, attention_backward, attention_workspace,
    attention_backward_workspace, layer_norm, layer_norm_backward, layer_norm_backward_workspace,
    label_logprob, label_logprob_backward, label_logprob_workspace, EXPORTED_SYMBOLS,
)
