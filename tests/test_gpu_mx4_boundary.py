"""The set-up-time check of MXFP4 weights: the three kinds of weight buffers of one layer are told apart, and so are those of other layers."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _refused(ss, call, status):
    with pytest.raises(ss.SSError) as e:
        call()
    assert e.value.status == status


@pytest.mark.parametrize("code,dtype", [("SS_F16", torch.float16), ("SS_BF16", torch.bfloat16)])
@pytest.mark.parametrize("cout,cin", [(40, 96), (1, 4), (300, 1000)])
def test_kinds_of_weights(ss, code, dtype, cout, cin):
    desc = ss.make_desc(cout, cin, 1, 1, getattr(ss, code))
    W = torch.randn((cout, cin), device="cuda").to(dtype)
    M = torch.tensor([1, 0, 0, 1], dtype=torch.uint8, device="cuda").repeat(cout, cin // 4)
    buffers = {ss.SS_WEIGHTS_DENSE: ss.ss_dense_pack(desc, W, M), ss.SS_WEIGHTS_SPARSE: ss.ss_mask_compress(desc, W, M), ss.SS_WEIGHTS_MX4: ss.ss_mx4_pack(desc, W, M)}
    longest = max(b.numel() for b in buffers.values())
    for kind, buffer in buffers.items():
        ss.ss_weights_check(desc, buffer, kind)
        ss.ss_weights_check(desc, buffer, kind, stream=torch.cuda.current_stream())
        wide = torch.zeros(longest, dtype=torch.uint8, device="cuda")      # (long enough for any of them)
        wide[:buffer.numel()] = buffer
        for other in buffers:
            if other != kind:
                _refused(ss, lambda: ss.ss_weights_check(desc, wide, other), ss.SS_ERR_INVALID_ARG)
    packed = buffers[ss.SS_WEIGHTS_MX4]
    ss.ss_weights_check(desc, ss.ss_mx4_pack(desc, W), ss.SS_WEIGHTS_MX4)                            # without a mask, too
    _refused(ss, lambda: ss.ss_weights_check(desc, packed[:-16], ss.SS_WEIGHTS_MX4), ss.SS_ERR_INVALID_ARG)
    _refused(ss, lambda: ss.ss_weights_check(desc, torch.zeros_like(packed), ss.SS_WEIGHTS_MX4), ss.SS_ERR_INVALID_ARG)
    swapped = ss.make_desc(cout, cin, 1, 1, ss.SS_BF16 if code == "SS_F16" else ss.SS_F16)
    _refused(ss, lambda: ss.ss_weights_check(swapped, packed, ss.SS_WEIGHTS_MX4), ss.SS_ERR_INVALID_ARG)
    if cout > 1:
        _refused(ss, lambda: ss.ss_weights_check(ss.make_desc(cout - 1, cin, 1, 1, desc.dtype), packed, ss.SS_WEIGHTS_MX4), ss.SS_ERR_INVALID_ARG)


def test_descriptors_that_have_no_4bit_form(ss):
    buffer = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    for desc in (ss.make_desc(32, 32, 3, 3), ss.make_desc(32, 32, 1, 1, 2)):
        _refused(ss, lambda: ss.ss_weights_check(desc, buffer, ss.SS_WEIGHTS_MX4), ss.SS_ERR_UNSUPPORTED)
