"""Data-parallel plumbing around the single-GPU path (torch.distributed only).

The hot path shards by bucket and by worker with no data-path collective: every
rank compresses its own buckets.  What ranks must share is small host state:
the ratio the controller picked (all ranks have to compress at the same ratio,
so that payloads have one size and can be all-gathered), and timings.
"""
from __future__ import annotations

import torch
import torch.distributed as dist


def _device_for(group=None):
    return torch.device("cuda", torch.cuda.current_device()) if dist.get_backend(group) == "nccl" else torch.device("cpu")


def agree_ratio(ratio: float, group=None, src: int = 0) -> float:
    """Rank `src`'s controller decides; every rank returns that ratio (exact double)."""
    if not dist.is_initialized() or dist.get_world_size(group) == 1:
        return float(ratio)
    t = torch.tensor([float(ratio)], dtype=torch.float64, device=_device_for(group))
    dist.broadcast(t, src=src, group=group)
    return float(t.item())


def max_over_ranks(value: float, group=None) -> float:
    """Slowest rank's value (used for step times: a step ends when the last rank ends)."""
    if not dist.is_initialized() or dist.get_world_size(group) == 1:
        return float(value)
    t = torch.tensor([float(value)], dtype=torch.float64, device=_device_for(group))
    dist.all_reduce(t, op=dist.ReduceOp.MAX, group=group)
    return float(t.item())


def whole_job_gbps(world: int, steps: int, bytes_per_rank_step: float, slowest_ms: float) -> float:
    """Aggregate throughput of `world` ranks doing the same work per step (weak scaling)."""
    return world * steps * bytes_per_rank_step / (slowest_ms * 1e-3) / 1e9


def payload_slots(world: int, payload_bytes: int):
    """Byte ranges of the W equal-size payloads inside an all-gather buffer (16-byte aligned slots)."""
    slot = (payload_bytes + 15) // 16 * 16
    return [(r * slot, r * slot + payload_bytes) for r in range(world)], slot * world


def exchange_payloads(payload: torch.Tensor, group=None):
    """The exchange step of the sparse path (Section 5.3: top-k payloads travel by AllGather):
    every rank contributes its payload (uint8 tensor; all ranks' payloads have the same size because
    they compressed equally long buckets at the agreed ratio) and receives all of them.
    Returns (buffer, [one view per rank]); view r is rank r's payload, 16-byte aligned, ready for
    nsml_decompress_accumulate.  One fixed-size all-gather, NCCL on CUDA tensors, gloo on CPU ones."""
    world = dist.get_world_size(group) if dist.is_initialized() else 1
    nbytes = payload.numel()
    slots, total = payload_slots(world, nbytes)
    slot = total // world
    buf = torch.empty(total, dtype=torch.uint8, device=payload.device)
    if world == 1:
        buf[:nbytes].copy_(payload)
    else:
        rank = dist.get_rank(group)
        mine = buf[rank * slot:(rank + 1) * slot]
        mine[:nbytes].copy_(payload)
        if slot > nbytes:
            mine[nbytes:].zero_()
        dist.all_gather_into_tensor(buf, mine.clone(), group=group)
    return buf, [buf[a:b] for a, b in slots]


class _HostClock:
    def __init__(self):
        import time

        self._now, self._marks = time.perf_counter, []

    def mark(self):
        self._marks.append(self._now())

    def phases_ms(self):
        return [1e3 * (b - a) for a, b in zip(self._marks, self._marks[1:])]


class _CudaClock:
    def __init__(self):
        self._marks = []

    def mark(self):
        ev = torch.cuda.Event(enable_timing=True)
        ev.record()
        self._marks.append(ev)

    def phases_ms(self):
        self._marks[-1].synchronize()
        return [a.elapsed_time(b) for a, b in zip(self._marks, self._marks[1:])]


def exchange_round(ctrl, last, dense_bytes_all_ranks: float, compress, accumulate, on_cuda: bool, group=None):
    """One step of the data-parallel exchange (Fig. 1, Alg. 1 Step 2 and Section 5.3 put together).

    ctrl      this rank's controller (only rank 0's decision is used: ranks must compress at one ratio so that
              the payloads have one size)
    last      (bytes, seconds) of the previous step's transfer as this function returned it; (0, 0) at first
    compress(ratio) -> this rank's payload (uint8 tensor); accumulate(views) sums the gathered payloads
    Returns (agreed ratio, [compress, all-gather, sum] times in ms each MAX-reduced over the ranks, new `last`):
    the transfer the controller sees next is all ranks' payload bytes and the slowest rank's all-gather time."""
    world = dist.get_world_size(group) if dist.is_initialized() else 1
    ratio = agree_ratio(ctrl.select_ratio(last[0], last[1], dense_bytes_all_ranks), group)
    clock = _CudaClock() if on_cuda else _HostClock()
    clock.mark()
    payload = compress(ratio)
    clock.mark()
    _, views = exchange_payloads(payload, group)
    clock.mark()
    accumulate(views)
    clock.mark()
    phases = [max_over_ranks(ms, group) for ms in clock.phases_ms()]
    return ratio, phases, (float(world * payload.numel()), max(phases[1] * 1e-3, 1e-9))


class GradientExchange:
    """One bucket's data-parallel gradient exchange, every step (Fig. 1 and Alg. 1-2 of the paper put
    together): rank 0's controller picks the ratio from the last measured transfer, every rank compresses
    its bucket at that ratio, the payloads are all-gathered, every rank sums them into its dense
    gradient, and the measured transfer (bytes of all payloads, slowest rank's device time of the
    all-gather) is what the controller sees next step.  CUDA only: the compression and the sum run in
    libnsml."""

    def __init__(self, n: int, bits: int = 8, group=None, device=None, **ctrl_overrides):
        import paper_2506_16235_b200 as nsml

        self.nsml, self.n, self.bits, self.group = nsml, int(n), int(bits), group
        self.device = device if device is not None else torch.device("cuda", torch.cuda.current_device())
        self.world = dist.get_world_size(group) if dist.is_initialized() else 1
        self.ctrl = nsml.Controller(**ctrl_overrides)
        self.ws = nsml.alloc_bytes(nsml.nsml_workspace_bytes(self.n), self.device)
        self.aws = nsml.alloc_bytes(nsml.nsml_accumulate_workspace_bytes(self.n, self.world), self.device)
        self.last = (0.0, 0.0)
        self.ratio = None

    def step(self, grad: torch.Tensor, dense: torch.Tensor) -> float:
        """dense <- sum over ranks of their compressed `grad`; returns the ratio used."""
        nsml = self.nsml
        self.ratio, self.phases_ms, self.last = exchange_round(
            self.ctrl, self.last, 4.0 * self.n * self.world,
            lambda ratio: nsml.nsml_compress(grad, ratio, self.bits, workspace=self.ws),
            lambda views: nsml.nsml_decompress_accumulate(views, dense, zero_first=True, workspace=self.aws, sized=True),
            on_cuda=True, group=self.group)
        return self.ratio


class NormLinear:
    """A linear layer behind an RMS norm, trained in 8 bits, whose gradients land where the exchange takes them from:

        y = rms_norm(x + residual) @ weight.T

    The forward pass normalises into 8-bit rows, multiplies them with the 8-bit weights and keeps, for the backward pass, those
    rows, the reciprocal norms and the residual stream in 8 bits: two bytes per element.  The backward pass writes the gradients
    of the norm's weight and of the weight into bucket[offset : offset + size], ready for GradientExchange.step.  CUDA only.

    A backward pass belongs to the last forward pass (what an earlier one kept is gone), with the weights that it used.
    nsml_last_status of workspaces[0], [1] and [2] tells whether the forward product, the weight's gradient and the input's
    were completed.

    weight [n, k] and norm_weight [k]: float32 or bfloat16 tensors that the optimiser owns; call pack() after it has changed
    them.  bucket: flat float32 or bfloat16 gradient bucket."""

    @staticmethod
    def size(n: int, k: int) -> int:
        """Elements of the bucket that the layer's gradients take: the norm's weight, then the weight."""
        return k + n * k

    def __init__(self, weight: torch.Tensor, norm_weight: torch.Tensor, bucket: torch.Tensor, offset: int = 0, eps: float = 1e-5):
        import paper_2506_16235_b200 as nsml

        n, k = weight.shape
        if offset < 0 or offset + self.size(n, k) > bucket.numel():
            raise ValueError(f"the bucket has no room for {self.size(n, k)} gradients at {offset}")
        self.nsml, self.weight, self.norm_weight, self.eps = nsml, weight, norm_weight, float(eps)
        self.grad_norm_weight = bucket[offset:offset + k]
        self.grad_weight = bucket[offset + k:offset + k + n * k].view(n, k)
        self.codes, self.scales = nsml.nsml_q8_empty(n, k, weight.device)
        each = nsml.NSML_Q8_MATMUL_WORKSPACE_BYTES
        workspace = nsml.alloc_bytes(3 * each + int(nsml.lib.nsml_q8_rms_norm_backward_workspace_bytes(k)), weight.device)
        self.workspaces, self.norm_workspace = tuple(workspace[i * each:(i + 1) * each] for i in range(3)), workspace[3 * each:]
        self.kept = None
        self.pack()

    def pack(self) -> None:
        """8-bit weights from the weights as they are now."""
        self.nsml.nsml_q8_pack(self.weight, codes=self.codes, scales=self.scales)

    def forward(self, x: torch.Tensor, residual: torch.Tensor = None):
        """x, residual [m, k] -> y [m, n] of x's type and h = x + residual (x itself without a residual)."""
        rows, scales, rstd, h = self.nsml.nsml_q8_rms_norm(x, self.norm_weight, self.eps, residual=residual)
        self.kept = rows, scales, rstd, self.nsml.nsml_q8_pack(h)
        return self.nsml.nsml_q8_matmul(rows, scales, self.codes, self.scales, dtype=x.dtype, workspace=self.workspaces[0]), h

    def backward(self, dy: torch.Tensor, dh: torch.Tensor = None, zero_first: bool = True) -> torch.Tensor:
        """dy [m, n] (of y's type, bfloat16 or float32, contiguous rows): writes (zero_first=False: adds) the weights' gradients
        and returns the gradient of x and residual, dh (a gradient that reaches h past the norm) included.  dh and the result
        have dy's type.  The products take bfloat16 rows on 16-byte boundaries: a dy that is not that (float32, which is rounded
        to bfloat16; an n that is no multiple of 8) is copied first.  Frees what the forward pass kept; a call that is refused
        has written nothing and frees nothing."""
        if self.kept is None:
            raise RuntimeError("backward() without a forward() before it")
        rows, scales, rstd, (h_codes, h_scales) = self.kept
        shape, device, dtype = rows.shape, rows.device, dy.dtype
        # whatever a call below would refuse is refused here, before the first of them has written anything
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise TypeError(f"dy must be bfloat16 or float32, not {dtype}")
        self._check(dy, "dy", (shape[0], self.codes.shape[0]), device)
        if dh is not None:
            if dh.dtype is not dtype:
                raise TypeError(f"dh must be {dtype}, not {dh.dtype}")
            self._check(dh, "dh", shape, device)
        nsml, dnormed, dy = self.nsml, rows.new_empty(shape, dtype=dtype), self._for_products(dy)
        nsml.nsml_q8_matmul_grad_weight(dy, rows, scales, dw=self.grad_weight, zero_first=zero_first, workspace=self.workspaces[1])
        nsml.nsml_q8_matmul_grad_input(dy, self.codes, self.scales, dx=dnormed, workspace=self.workspaces[2])
        nsml.nsml_q8_rms_norm_backward(dnormed, self.norm_weight, rstd, codes=h_codes, scales=h_scales, dh=dh, dx=dnormed,
                                       dweight=self.grad_norm_weight, zero_first=zero_first, workspace=self.norm_workspace)
        self.kept = None
        return dnormed

    @staticmethod
    def _check(t: torch.Tensor, what: str, shape, device) -> None:
        if t.shape != shape or t.device != device:
            raise ValueError(f"{what} must have shape {tuple(shape)} and be on {device}")
        stride = t.stride()
        if (shape[1] > 1 and stride[1] != 1) or (shape[0] > 1 and stride[0] < shape[1]):
            raise ValueError(f"{what} must be a 2-D tensor with contiguous rows")

    @staticmethod
    def _for_products(dy: torch.Tensor) -> torch.Tensor:
        """dy (contiguous rows) as the products' gradients take it: bfloat16, rows on 16-byte boundaries."""
        m, n = dy.shape
        if dy.dtype is torch.bfloat16 and dy.data_ptr() % 16 == 0 and (m <= 1 or dy.stride(0) % 8 == 0):
            return dy
        return torch.empty(m, (n + 7) // 8 * 8, dtype=torch.bfloat16, device=dy.device)[:, :n].copy_(dy.detach())
