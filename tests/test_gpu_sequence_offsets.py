"""Offsets that leave rows out at either end, which the operators report like every other bad offset (their results are
then unspecified), in the forward calls and in the gradients; good offsets beside them are not reported."""
import pytest

from test_gpu_sequence import make_conv, make_scan, torch, wm  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(wm, lens, T):  # noqa: F811
    """The four calls that take offsets and a status, on the rows of `lens`."""
    a, _, good, dy, _ = make_scan("f32", lens, 16, 8, 60)
    args = (a["u"], a["delta"], a["A"], a["Bm"], a["Cm"])
    x, _, w, b, _, cdy, _ = make_conv("f32", lens, 16, 3, 61)
    kept = wm.selective_scan(*args, good, T_max=T, need_checkpoints=True)["checkpoints"]
    return (lambda o, st: wm.selective_scan(*args, o, T_max=T, status=st),
            lambda o, st: wm.selective_scan_grad(dy, *args, o, kept, T_max=T, status=st),
            lambda o, st: wm.causal_conv(x, o, w, b, T_max=T, status=st),
            lambda o, st: wm.causal_conv_grad(cdy, x, o, w, b, T_max=T, status=st))


@pytest.mark.parametrize("lens,T,bad", [
    ([6, 6], 12, [0, 4, 8]), ([6, 6], 12, [3, 6, 12]), ([6, 6], 12, [1, 6, 11]), ([6, 6], 12, [0, 0, 0]), ([12], 12, [0, 11]),
    ([1] * 9, 1, list(range(1, 10)) + [9]), ([1] * 9, 1, list(range(9)) + [8]),       # single steps
    ([300], 300, [0, 299]), ([300], 300, [1, 300]),                                   # cut into chunks
])
def test_rows_left_out_are_reported(wm, lens, T, bad):  # noqa: F811
    for i, call in enumerate(calls(wm, lens, T)):
        print(f"[offsets] {bad[:4]} of {sum(lens)} rows, call {i}", flush=True)
        status = torch.zeros(64, dtype=torch.int32, device="cuda")
        call(torch.tensor(bad, dtype=torch.int32, device="cuda"), status)
        with pytest.raises(wm.WMError, match="do not run from 0") as e:
            wm.device_status(status)
        assert e.value.status == 5
        wm.device_status(status)                        # cleared
        good = [0]
        for n in lens:
            good.append(good[-1] + n)
        call(torch.tensor(good, dtype=torch.int32, device="cuda"), status)
        wm.device_status(status)
