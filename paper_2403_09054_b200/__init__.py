"""B200-native Keyformer score-and-evict path: CUDA kernels behind a C ABI, plus this thin binding."""
from .binding import (Keyformer, KeyformerError, kf_config, make_config, kf_workspace_bytes, kf_strerror,
                      kf_decode_step_static, kf_static_step, KF_STATIC_SCRATCH_BYTES,
                      kf_pack_cache, kf_unpack_cache, kf_packed_slot_bytes, kf_packed_scratch_bytes, kf_decode_step_packed, kf_packed_step,
                      kf_qk_norm_rotate, kf_qk_norm_args, kf_beam_select, kf_beam_args, kf_reorder_rows, kf_row_buffer,
                      KF_TYPE_FP16, KF_TYPE_BF16, KF_TYPE_FP32, KF_NORM_NONE, KF_NORM_RMS, KF_ROTARY_PAIRS, KF_ROTARY_HALVES,
                      LIB, LIB_PATH, EXPORTS,
                      KF_OK, KF_EINVAL, KF_ENOSPC, KF_ESTATE, KF_ECUDA, KF_ETIMEOUT, KF_EBOUNDS,
                      KF_NOISE_GUMBEL, KF_NOISE_NONE, KF_NOISE_CONST, KF_NOISE_GAUSS, KF_BIAS_NONE, KF_BIAS_ALIBI, KF_PREFILL_TENSOR, KF_PREFILL_SIMT,
                      KF_POS_ORIGINAL, KF_POS_NEW, KF_DECODE_AUTO, KF_DECODE_CUDA_CORES, KF_DECODE_TENSOR)
