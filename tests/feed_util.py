"""Helpers of the feed-forward operators' tests: operands inside larger arrays of NaN, results inside larger arrays of a mark."""
import numpy as np

MARK = -7.0
TYPE = {"f32": "float32", "bf16": "bfloat16"}
GATES = ("silu", "gelu", "gelu_tanh")


def rounded(torch, x, dtype):
    """x in the given type, as 64-bit numpy and as a torch tensor on the CPU."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(getattr(torch, TYPE[dtype]))
    return t.double().numpy(), t


def put(torch, t, pad=0, shift=0, device="cuda:0"):
    """`t` on the device, its rows `pad` elements further apart and its first element `shift` elements into its array; NaN everywhere else."""
    rows, cols = t.shape
    nan = 0x7f if t.element_size() == 1 else float("nan")
    flat = torch.full((shift + rows * (cols + pad) + 64,), nan, dtype=torch.uint8 if t.element_size() == 1 else t.dtype, device=device)
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_((t.view(torch.uint8) if t.element_size() == 1 else t).to(device))
    return view.view(t.dtype) if t.element_size() == 1 and not pad and not shift else view


class Result:
    """An output of rows x cols inside an array of marks, two rows before and two behind it; check() says that nothing else was written."""
    def __init__(self, torch, rows, cols, dtype, pad=0, shift=0, device="cuda:0"):
        self.torch, self.rows, self.cols, self.pad, self.at = torch, rows, cols, pad, shift + 2 * (cols + pad)
        n = self.at + rows * (cols + pad) + 2 * (cols + pad) + 8
        self.flat = torch.full((n,), MARK if dtype.is_floating_point else 0x55, dtype=dtype, device=device)
        self.view = self.flat[self.at:self.at + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def check(self):
        host = self.flat.cpu()
        mark = MARK if host.dtype.is_floating_point else 0x55
        outside = self.torch.ones_like(host, dtype=self.torch.bool)
        outside[self.at:self.at + self.rows * (self.cols + self.pad)].view(self.rows, self.cols + self.pad)[:, :self.cols] = False
        assert bool((host[outside] == mark).all()), "written outside the result"

    def numpy(self):
        return self.view.cpu().double().numpy()


def within(what, got, value, bound):
    off = np.abs(got - value)
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = np.unravel_index(np.argmax(off - bound), off.shape) if off.size else None
    assert (off <= bound).all(), f"{what} at {worst}: {got[worst]} for {value[worst]}, bound {bound[worst]}"
