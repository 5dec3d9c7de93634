"""What calls of the paged operators share between them in the binding."""
import pytest

import paper_2403_01136_amd as lpq

FAKE = 0x10000          # never dereferenced: the calls below must fail validation first
ALIGN, SHAPE = 5, 4


def test_the_cfg_that_calls_share_cannot_be_written_to():
    import torch
    cfg = lpq._attn_cfg_of(8 * 64, 4, 2, torch.float16)
    assert lpq._attn_cfg_of(8 * 64, 4, 2, torch.float16) is cfg
    assert (cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.dtype) == (4, 2, 64, lpq.LPQ_DT_FP16)
    for name, _ in lpq.lpq_attn_cfg._fields_:
        with pytest.raises(AttributeError):
            setattr(cfg, name, 1)
    assert (cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.dtype) == (4, 2, 64, lpq.LPQ_DT_FP16)
    # the library reads it as any other
    L, r = lpq.load_library(), lpq.lpq_rotary(64, 0, 10, 1e-6, FAKE, None, None)
    assert L.lpq_qk_norm_rotary(FAKE + 2, cfg, r, FAKE, None, 3, FAKE + 2, None) == ALIGN
    assert L.lpq_qk_norm_rotary(FAKE, lpq._attn_cfg_of(7 * 64, 3, 2, torch.float16), r, FAKE, None, 3, FAKE, None) == SHAPE
