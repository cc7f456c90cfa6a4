"""MI355X-native additively-quantized (AQ) layer: forward and codebook gradient;
4-bit layers with group scales; distillation and cross-entropy losses.

The product is ``libaq.so`` (HIP kernels for gfx950 behind the C ABI in
``include/aq.h``); this package holds its sources (``csrc/``), the build
script and a ctypes binding with the same entry-point names.
"""
from .aq import (  # noqa: F401
    AQError,
    AQLayer,
    LIB_PATH,
    EXPORTED,
    load_library,
    make_desc,
    aq_layer_create,
    aq_layer_forward,
    aq_layer_forward_static,
    aq_layer_prepare,
    aq_layers_prepare,
    aq_layer_decode,
    aq_layer_codebook_grad,
    aq_layer_set_path,
    aq_layer_set_option,
    aq_layer_get_option,
    aq_layer_set_launch_events,
    aq_layer_last_launches,
    aq_layer_describe,
    OPTION_CODES,
    aq_layer_choose_path,
    aq_layer_destroy,
    USQLayer,
    VocabLoss,
    aq_usq_desc,
    aq_usq_create,
    aq_usq_forward,
    aq_usq_input_grad,
    aq_usq_destroy,
    aq_loss_desc,
    aq_loss_create,
    aq_loss_cross_entropy,
    aq_loss_distill,
    aq_loss_destroy,
    aq_version,
)
