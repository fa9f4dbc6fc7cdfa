"""Tensors for tests of calls that take strided rows: rows with room between them, off their allocation's alignment, and a check that nothing
around them was written."""
import torch

DEV = "cuda:0"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # a rounding, relative


def stream():
    return torch.cuda.current_stream().cuda_stream


class Placed:
    """`values` [rows, cols] (or a shape, filled with what marks untouched places) as rows `room` elements further apart than needed, `shift`
    elements off the allocation."""

    def __init__(self, values, dtype, room=0, shift=0, mark=7):
        shape = tuple(values) if not torch.is_tensor(values) else tuple(values.shape)
        self.mark, (rows, cols) = mark, shape
        self.store = torch.full((rows * (cols + room) + shift + 32,), mark, dtype=dtype, device=DEV)
        self.view = self.store[shift:shift + rows * (cols + room)].view(rows, cols + room)[:, :cols]
        if torch.is_tensor(values):
            self.view.copy_(values)

    def untouched_around(self):
        keep = self.view.clone()
        self.view.fill_(self.mark)
        same = bool((self.store == self.mark).all())
        self.view.copy_(keep)
        return same

    def host(self):
        return self.view.double().cpu().numpy()


class PlacedBytes:
    """Rows of 8 bits, `room` bytes (a multiple of 16) further apart than needed; q and e given or left marked."""

    def __init__(self, rows, cols, q=None, e=None, room=0):
        self.cols, self.padded = cols, (cols + 15) // 16 * 16
        self.store = torch.full((rows, self.padded + room), 77, dtype=torch.int8, device=DEV)
        self.exps = torch.full((rows + 16,), 55, dtype=torch.int8, device=DEV)
        self.rows = rows
        if q is not None:
            self.store[:, :self.padded] = 0
            self.store[:, :cols] = torch.as_tensor(q).to(DEV, torch.int8)
            self.exps[:rows] = torch.as_tensor(e).to(DEV, torch.int8)

    def q(self):
        return self.store[:, :self.cols].cpu().numpy()

    def e(self):
        return self.exps[:self.rows].cpu().numpy().astype(int)

    def padding_is_zero_and_the_rest_untouched(self):
        pad, rest = self.store[:, self.cols:self.padded], self.store[:, self.padded:]
        return not bool(pad.any()) and bool((rest == 77).all()) and bool((self.exps[self.rows:] == 55).all())
