"""The binding of the optimizer step: streams by handle, the device of a list."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


@pytest.mark.parametrize("handle", [0, 1])
def test_a_record_for_the_default_stream_by_handle_is_made_in_its_order(handle):
    """0 and 1 both name the legacy default stream, which is torch's default stream; a call with the handle gives the record
    that one without it gives, also from inside another stream's context."""
    device = torch.device("cuda", torch.cuda.current_device())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with fr._allocating_on(handle, device):
            assert torch.cuda.current_stream() == torch.cuda.default_stream()
        assert torch.cuda.current_stream() == side
    plan = fr.OptPlan(grads=[torch.linspace(-1, 1, 70001, device="cuda")])
    want = plan.clip(0.5, 0.25)
    torch.cuda.synchronize()
    got = plan.clip(0.5, 0.25, stream=handle)
    with torch.cuda.stream(side):
        aside = plan.clip(0.5, 0.25, stream=handle)
    torch.cuda.synchronize()
    assert float(fr.clip_view(want)[0]) > 0
    assert torch.equal(got, want) and torch.equal(aside, want)


@pytest.mark.parametrize("sizes", [(5,), (5, 0), ()])
def test_a_list_that_starts_with_an_empty_host_tensor_has_its_records_on_the_gpu(sizes):
    grads = [torch.empty(0)] + [torch.full((n,), 2.0, device="cuda") for n in sizes]
    plan = fr.OptPlan(grads=grads)
    record = plan.clip()
    assert plan.device.type == record.device.type == "cuda"
    norm, scale, bad = (x.item() for x in fr.clip_view(record))
    assert abs(norm - 2.0 * sum(sizes) ** 0.5) <= 1e-6 and scale == 1.0 and bad == 0
