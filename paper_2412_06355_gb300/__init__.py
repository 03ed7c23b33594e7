"""GB300-native fused DendSN layer (dendritic spiking neuron, arXiv 2412.06355).

The forward and the BPTT backward of a DendSN layer run as hand-written CUDA
kernels for sm_103a behind the C ABI in include/dendsn.h; `binding` is the thin
Python layer over it and `workloads` draws seeded synthetic layer inputs. Around the
layer stand the operators a token sequence needs: embedding, gated compartment scan and
the cross entropy of a linear readout; what a stack of token blocks needs: the norm with the
residual's addition and the gated delta rule; and the AdamW step that trains all of it.
"""
from . import binding, workloads
from .binding import (DeltaFunction, DendSNError, DendSNFunction, EmbedFunction, NormFunction,
                      ScanFunction, XentFunction, adamw_plan, adamw_step, config_of,
                      delta_backward, delta_forward, dendsn_backward, dendsn_forward,
                      dendsn_workspace_size, embed_backward, embed_forward, make_adamw_config,
                      make_config, make_delta_config, make_embed_config, make_norm_config,
                      make_scan_config, make_xent_config, norm_backward, norm_forward,
                      scan_backward, scan_forward, xent_backward, xent_forward)
from .optim import AdamW

__all__ = ["AdamW", "binding", "workloads", "DeltaFunction", "DendSNError", "DendSNFunction",
           "EmbedFunction", "NormFunction", "ScanFunction", "XentFunction", "adamw_plan",
           "adamw_step", "config_of", "delta_backward", "delta_forward", "dendsn_backward",
           "dendsn_forward", "dendsn_workspace_size", "embed_backward", "embed_forward",
           "make_adamw_config", "make_config", "make_delta_config", "make_embed_config",
           "make_norm_config", "make_scan_config", "make_xent_config", "norm_backward",
           "norm_forward", "scan_backward", "scan_forward", "xent_backward", "xent_forward"]
