"""emb_paged8_store refuses turns and axes left in host memory, where emb_rotary_turns gives the first and emb_qk_norm_rope takes the
second (CPU only: stand-ins for tensors on the device, and no call reaches a launch)."""
import pytest
import torch

import paper_2607_02501_gb300 as emb

T, H, HK, D = 10, 4, 2, 64
bf, i32, i64, u8 = torch.bfloat16, torch.int32, torch.int64, torch.uint8


class OnDevice:
    """A tensor's sizes, with an address that is never used."""

    def __init__(self, t, at):
        self.t, self.at = t, at

    def data_ptr(self):
        return 0x7f0000000000 + self.at * (4 << 30)

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)


def args(**change):
    t = dict(q=(bf, T, H * D), k=(bf, T, HK * D), v=(bf, T, HK * D), q_out=(bf, T, H * D), k_codes=(u8, 5, 32, HK, D), v_codes=(u8, 5, 32, HK, D),
             k_exp=(u8, 5, 2, HK), v_exp=(u8, 5, 2, HK), slots=(i64, T), positions=(i32, T), turns=(i64, D // 2), axis_of_pair=(u8, D // 2))
    return {n: change[n] if n in change else OnDevice(torch.zeros(*s[1:], dtype=s[0]), i) for i, (n, s) in enumerate(t.items())}


@pytest.fixture(scope="module", autouse=True)
def built():
    emb.build()


@pytest.mark.parametrize("name,bad", [("turns", emb.emb_rotary_turns(D)), ("axis_of_pair", torch.zeros(D // 2, dtype=u8))])
def test_host_memory_is_refused(name, bad):
    with pytest.raises(emb.EmbError, match=f"{name} is in host memory") as e:
        # (eps is refused too, should the call get that far)
        emb.emb_paged8_store(**args(**{name: bad}), eps=-1.0, stream=1)
    assert e.value.status == emb.EMB_EINVAL


def test_stand_ins_are_read_as_tensors():
    """The same call with everything on the device gets as far as the library, which refuses its eps."""
    with pytest.raises(emb.EmbError) as e:
        emb.emb_paged8_store(**args(), eps=-1.0, stream=1)
    assert e.value.status == emb.EMB_EINVAL and "host memory" not in str(e.value)
