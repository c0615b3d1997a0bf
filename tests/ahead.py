"""Numbers on the device that a kernel of the library writes which lets the next one come up before it has finished: the GEMM of one
row, whose blocks do so as soon as they are set up, and which then takes tens of microseconds.  Its one-hot row picks a row of bf16
numbers whose bits are those of the numbers, in turn of one list and of the other's.  (A copy by torch would have finished before
the next kernel starts.)"""
import torch

K = 1 << 17


class Ahead:
    def __init__(self, kvp, first, second):
        """Two lists of tensors of int32, alike in their sizes; `views` are those of the buffer that is written."""
        self.kvp = kvp
        flat = [torch.cat([x.reshape(-1).int() for x in xs]) for xs in (first, second)]
        assert flat[0].numel() == flat[1].numel()
        halves = torch.cat(flat).view(torch.uint16).long()
        # zero, or a normal finite bf16: times one, beside zeros, each comes out as it went in
        assert ((halves == 0) | ((halves & 0x7f80) != 0) & ((halves & 0x7f80) != 0x7f80)).all()
        pad = torch.zeros(-flat[0].numel() % 4, dtype=torch.int32)          # 16-byte rows
        self.bits = torch.stack([torch.cat([x, pad]) for x in flat]).cuda()
        rows = self.bits.view(torch.bfloat16)
        self.table = torch.zeros(rows.shape[1], K, dtype=torch.bfloat16, device="cuda")
        self.table[:, 0], self.table[:, K - 1] = rows[0], rows[1]
        self.pick = torch.zeros(2, 1, K, dtype=torch.bfloat16, device="cuda")
        self.pick[0, 0, 0] = self.pick[1, 0, K - 1] = 1.0
        self.buffer = rows[1:].clone()
        at, self.views = 0, []
        for x in first:
            self.views.append(self.buffer.view(torch.int32).view(-1)[at:at + x.numel()].view(x.shape))
            at += x.numel()
        for i in (0, 1):                                      # (loads the kernel, and what is written is right)
            self.write(i)
            torch.cuda.synchronize()
            assert torch.equal(self.buffer.view(torch.int32)[0], self.bits[i])

    def write(self, i):
        self.kvp.gemm(self.pick[i % 2], self.table, self.buffer)
