"""Where a session that was made for "cuda", without an index, allocates later (no GPU needed): on the device that it was made on, not
on the one that is current by then."""
import types

import torch

import paper_2412_06198_amd as sa


def test_later_buffers_stay_on_the_session_s_device():
    cfg = sa.SaConfig()
    cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = 8, 2, 128
    cfg.seq_len, cfg.block, cfg.last_q = 512, 64, 32
    devices = []

    def empty(size, dtype, device):
        devices.append(device)
        return torch.empty(size, dtype=dtype)

    ses = object.__new__(sa.Session)
    ses.torch = types.SimpleNamespace(empty=empty, uint8=torch.uint8, float32=torch.float32, bfloat16=torch.bfloat16)
    ses.device, ses._attend_scratch = torch.device("cuda"), None
    ses.ws = types.SimpleNamespace(device=torch.device("cuda", 1))
    ses.cfg = sa.sa_default_budgets(cfg, 0.5)
    ses.ctx = sa.sa_create(cfg)
    ses.cache(640)
    raw, at, size = ses.attend_scratch()
    assert len(devices) == 7 and set(devices) == {torch.device("cuda", 1)}
    assert at % 256 == 0 and at + size <= raw.data_ptr() + raw.numel()
    ses.close()
