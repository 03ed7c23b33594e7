"""GB300-native fused DendSN layer (dendritic spiking neuron, arXiv 2412.06355).

The forward and the BPTT backward of a DendSN layer run as hand-written CUDA
kernels for sm_103a behind the C ABI in include/dendsn.h; `binding` is the thin
Python layer over it and `workloads` draws seeded synthetic layer inputs. Around the
layer stand the operators a token sequence needs: embedding, gated compartment scan and
the cross entropy of a linear readout.
"""
from . import binding, workloads
from .binding import (DendSNError, DendSNFunction, EmbedFunction, ScanFunction, XentFunction,
                      config_of, dendsn_backward, dendsn_forward, dendsn_workspace_size,
                      embed_backward, embed_forward, make_config, make_embed_config,
                      make_scan_config, make_xent_config, scan_backward, scan_forward,
                      xent_backward, xent_forward)

__all__ = ["binding", "workloads", "DendSNError", "DendSNFunction", "EmbedFunction",
           "ScanFunction", "XentFunction", "config_of", "dendsn_backward", "dendsn_forward",
           "dendsn_workspace_size", "embed_backward", "embed_forward", "make_config",
           "make_embed_config", "make_scan_config", "make_xent_config", "scan_backward",
           "scan_forward", "xent_backward", "xent_forward"]
