"""Semi-autoregressive WINO decode loop over the C ABI (Sec. 3 and Sec. 4.2.3).

Blocks are decoded left to right; inside a block ``wino_step`` is repeated
until no position of the block is MASK in any sequence of the batch.  A
sequence whose block is complete is frozen (WINO_OPT_FREEZE_FINISHED): its
own loop has ended, so it is not re-verified while the rest of the batch
finishes the block.  The
only device-to-host traffic per step is the [n_seq, 3] counts array, read to
decide whether the block is finished (plus the token state when a trajectory
is recorded).  The hidden states of each step come
from a caller-supplied function that runs the transformer's layers;
``BlockCache`` gives it the paged cache, the rotation and the attention
under the shadow-block mask that those layers need.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Callable

from ._abi import (WINO_ERR_MAX_STEPS, WINO_MASK_FULL, WINO_MASK_SHADOW, WINO_OK, WinoError, WinoKvBatch, WinoRope,
                   attend_workspace, make_kv_batch, make_params, wino_attend, wino_decode, wino_rope_append, wino_step,
                   wino_workspace_size_step)


@dataclass
class BlockStats:
    block: int
    blk_start: int
    steps: int = 0
    drafted: int = 0
    remasked: int = 0
    fallback: int = 0  # drafts made by the at-least-one rule (no masked position cleared tau1)


@dataclass
class LoopStats:
    blocks: list = field(default_factory=list)
    total_steps: int = 0  # steps this call ran
    rows_scored: int = 0
    next_step: int = 0  # global index of the step after the last one run


def resume_point(k: int, blk_start: int, counts, *, prompt_len: int, blk_len: int) -> tuple[int, int]:
    """(start_block, start_step) that continue a decode after its global step ``k``, from the arguments
    ``on_step`` receives.  A checkpoint of a decode is the token state (and ``last_change``) after step
    ``k`` together with this pair: the hidden states of later steps depend only on the step index and
    the block, so a decode resumed from it replays the uninterrupted one exactly."""
    import numpy as np
    b = (blk_start - prompt_len) // blk_len
    done = bool((np.asarray(counts)[:, 2] == 0).all())
    return (b + 1 if done else b), k + 1


def _head_dims(W, w_panels: bool) -> tuple[int, int]:
    """(d, V) of an LM head given row-major [V, d] or as a panel copy [d/64, V, 64]."""
    if w_panels:
        return int(W.shape[0]) * 64, int(W.shape[1])
    return int(W.shape[1]), int(W.shape[0])


def decode(W, tokens, *, prompt_len: int, blk_len: int, n_blocks: int, tau1: float, tau2: float, mask_id: int,
           hidden: Callable[[int, int], object], max_steps: int = 4096, stream=None,
           on_step: Callable | None = None, last_change=None, no_shadow: bool = False,
           compact: bool = False, draft_m: int = 0, trajectory: list | None = None, start_block: int = 0,
           start_step: int = 0, skip_finished: bool = False, w_panels: bool = False) -> LoopStats:
    """Decode ``n_blocks`` blocks of ``tokens`` (int32 [n_seq, S], device) in place.

    ``hidden(k, blk_start)`` returns the device bf16 hidden states [2*n_seq*blk_len, d]
    for global step ``k`` (0-based; the step produces state Y^(k+1)).  ``on_step(k,
    blk_start, counts_host, flags)`` is called after every step (for tests and
    statistics).  ``last_change`` (device int32 [n_seq, S], zeros at the start)
    receives, per position, the last step that changed it: after the decode, each
    position's WINO finalization step t_l (Sec. 5.1).  ``no_shadow``: WINO+ inference
    (Sec. 5.3): ``hidden`` returns only the n_seq*blk_len block rows, drafting uses the
    single threshold ``tau1`` and nothing is re-masked.  ``compact``: score only the row
    each position's update reads (WINO_OPT_COMPACT), same results.  ``draft_m`` > 0: draft
    a fixed number of the most confident masked positions per step instead of Eq. 2 (naive
    parallel sampling, Sec. 3; with ``no_shadow`` the irreversible baseline decoder, 1 =
    greedy Eq. 1).  ``trajectory``: a list that receives the host copy of the state
    Y^(0), Y^(1), ... (int32 [n_seq, S] arrays), one per step, for building WINO+ training
    states (Sec. 5.1-5.2); it costs one extra device-to-host copy of ``tokens`` per step.
    ``start_block``, ``start_step``: resume a checkpointed decode (see ``resume_point``): blocks
    before ``start_block`` are taken as done and the global step count starts at ``start_step``.
    ``skip_finished``: each step scores only the sequences whose block still has a MASK (an
    active-sequence list, ``wino_params.active_seq``); the states are those of the frozen
    sequences without it, and ``on_step`` sees zero counts for the sequences left out.
    ``w_panels``: ``W`` is the panel copy of ``wino_lm_head_panels`` ([d/64, V, 64]), same results.
    """
    import numpy as np
    import torch

    n_seq, S = int(tokens.shape[0]), int(tokens.shape[1])
    d, V = _head_dims(W, w_panels)
    rows_per_seq = (1 if (no_shadow or compact) else 2) * blk_len  # rows scored per sequence and step
    dev = tokens.device
    ts = stream if stream is not None else torch.cuda.current_stream(dev)  # every copy goes on the step's stream
    active_d = torch.arange(n_seq, dtype=torch.int32, device=dev) if skip_finished else None
    active_h = torch.zeros(n_seq, dtype=torch.int32, pin_memory=True) if skip_finished else None
    p0 = make_params(tau1, tau2, mask_id, n_seq, S, prompt_len, blk_len, no_shadow=no_shadow, compact=compact,
                     draft_m=draft_m, active_seq=active_d, n_active=n_seq if skip_finished else None,
                     w_panels=w_panels)
    ws = torch.zeros(wino_workspace_size_step(p0, d, V), dtype=torch.uint8, device=dev)
    counts = torch.zeros((n_seq, 3), dtype=torch.int32, device=dev)
    flags = torch.zeros((n_seq, blk_len), dtype=torch.int8, device=dev)
    counts_host = torch.zeros((n_seq, 3), dtype=torch.int32, pin_memory=True)
    flags_host = torch.zeros((n_seq, blk_len), dtype=torch.int8, pin_memory=True)
    tokens_host = torch.zeros((n_seq, S), dtype=torch.int32, pin_memory=True) if trajectory is not None else None
    if trajectory is not None:
        with torch.cuda.stream(ts):
            tokens_host.copy_(tokens)
        ts.synchronize()
        trajectory.append(tokens_host.numpy().copy())
    stats = LoopStats()
    k = start_step
    for b in range(start_block, n_blocks):
        b0 = prompt_len + b * blk_len
        p = make_params(tau1, tau2, mask_id, n_seq, S, b0, blk_len, max_steps, freeze_finished=True,
                        last_change=last_change, no_shadow=no_shadow, compact=compact, draft_m=draft_m,
                        w_panels=w_panels)
        bs = BlockStats(block=b, blk_start=b0)
        active = list(range(n_seq))  # a new block: every sequence takes part
        while True:
            if bs.steps >= max_steps:
                raise WinoError(WINO_ERR_MAX_STEPS, f"decode: block {b} not finished after {max_steps} steps")
            H = hidden(k, b0)
            p.step_index = k + 1
            if skip_finished:
                active_h[:len(active)] = torch.tensor(active, dtype=torch.int32)
                with torch.cuda.stream(ts):
                    active_d[:len(active)].copy_(active_h[:len(active)], non_blocking=True)
                p.active_seq, p.n_active = active_d.data_ptr(), len(active)
            wino_step(H, W, tokens, p, counts, ws, flags=flags, stream=ts)
            with torch.cuda.stream(ts):
                counts_host.copy_(counts, non_blocking=True)
                flags_host.copy_(flags, non_blocking=True)
                if tokens_host is not None:
                    tokens_host.copy_(tokens, non_blocking=True)
            ts.synchronize()
            c = counts_host.numpy().copy()
            fl = flags_host.numpy().copy()
            if skip_finished:  # the sequences left out were not stepped: no counts, no flags
                left_out = np.ones(n_seq, bool)
                left_out[active] = False
                c[left_out] = 0
                fl[left_out] = 0
            if tokens_host is not None:
                trajectory.append(tokens_host.numpy().copy())
            if (c < 0).any():
                raise WinoError(int(c.min()), f"decode: device status at step {k}")
            bs.steps += 1
            bs.drafted += int(c[:, 0].sum())
            bs.remasked += int(c[:, 1].sum())
            bs.fallback += int((fl == 2).sum())
            stats.rows_scored += rows_per_seq * len(active)
            if on_step is not None:
                on_step(k, b0, c.copy(), flags)
            k += 1
            if (c[:, 2] == 0).all():
                break
            if skip_finished:
                active = [i for i in active if c[i, 2] != 0]
        stats.blocks.append(bs)
    stats.total_steps = k - start_step
    stats.next_step = k
    return stats


def decode_native(W, tokens, *, prompt_len: int, blk_len: int, n_blocks: int, tau1: float, tau2: float,
                  mask_id: int, hidden: Callable[[int, int], object], max_steps: int = 4096, stream=None,
                  last_change=None, no_shadow: bool = False, compact: bool = False, draft_m: int = 0,
                  start_block: int = 0, start_step: int = 0, skip_finished: bool = False,
                  w_panels: bool = False) -> LoopStats:
    """``decode`` with the step loop run by the library (``wino_decode``): the same steps, states and
    statistics, with one callback into Python per step (for the hidden states) instead of the whole
    per-step bookkeeping.  No ``on_step`` or ``trajectory``; errors raise ``WinoError``.
    ``skip_finished`` as in ``decode``: the library keeps the active-sequence list; ``w_panels`` as in ``decode``."""
    import torch

    n_seq, S = int(tokens.shape[0]), int(tokens.shape[1])
    d, V = _head_dims(W, w_panels)
    rows_per_seq = (1 if (no_shadow or compact) else 2) * blk_len
    dev = tokens.device
    ts = stream if stream is not None else torch.cuda.current_stream(dev)
    p = make_params(tau1, tau2, mask_id, n_seq, S, prompt_len, blk_len, max_steps, freeze_finished=True,
                    last_change=last_change, no_shadow=no_shadow, compact=compact, draft_m=draft_m,
                    w_panels=w_panels)
    active_buf = torch.zeros(n_seq, dtype=torch.int32, device=dev) if skip_finished else None
    p_ws = make_params(tau1, tau2, mask_id, n_seq, S, prompt_len, blk_len, no_shadow=no_shadow, compact=compact,
                       active_seq=active_buf, n_active=n_seq if skip_finished else None)  # sized for every list
    ws = torch.zeros(wino_workspace_size_step(p_ws, d, V), dtype=torch.uint8, device=dev)
    counts = torch.zeros((n_seq, 3), dtype=torch.int32, device=dev)
    counts_host = torch.zeros((n_seq, 3), dtype=torch.int32, pin_memory=True)
    flags = torch.zeros((n_seq, blk_len), dtype=torch.int8, device=dev)
    flags_host = torch.zeros((n_seq, blk_len), dtype=torch.int8, pin_memory=True)
    torch.cuda.current_stream(dev).synchronize()  # the buffers above are ready before the library's stream runs
    rc, blocks, nxt = wino_decode(W, tokens, p, n_blocks, hidden, counts, counts_host, ws, flags=flags,
                                  flags_host=flags_host, active_buf=active_buf, stream=ts, first_block=start_block,
                                  first_step=start_step)
    if rc != WINO_OK:
        raise WinoError(rc, f"wino_decode (stopped at step {nxt})")
    stats = LoopStats()
    for b in range(start_block, n_blocks):
        steps, drafted, remasked, fallback, seq_steps = blocks[b]
        stats.blocks.append(BlockStats(block=b, blk_start=prompt_len + b * blk_len, steps=steps, drafted=drafted,
                                       remasked=remasked, fallback=fallback))
        stats.rows_scored += rows_per_seq * seq_steps
    stats.total_steps = nxt - start_step
    stats.next_step = nxt
    return stats


class BlockCache:
    """The paged key and value caches of a decode's layers, for ``hidden`` functions of ``decode`` and ``decode_native``.

    Every sequence has room for ``seq_len`` slots, one per position, and behind them for the shadow block's ``blk_len``.
    ``context(start, end)`` describes the rows of positions start .. end - 1 of every sequence, [s][position], which see
    each other and everything before them: the prompt, or a block that is done, taken into the cache once.
    ``step(blk_start)`` describes the rows of a step as ``wino_step`` wants their hidden states, [s][kind][l] (with
    ``no_shadow`` [s][l]): block rows see the context and the block, shadow rows these and the shadow block but for the
    position that they verify (Sec. 4.2.2).
    Both leave out what lies to the right, the blocks that are still masked, which the rows of the paper see too
    ([Y_left, Y_cur, Y_right, Y_shad]).  ``seen`` takes it in: the rows see the positions [0, seen), of which ``context`` must have stored
    the ones behind the block.  The shadow block is stored in the ``blk_len`` slots from ``seen`` on, so a decode whose right side is
    in the cache passes ``seen=seq_len`` to every step.  What is in the cache stays as its last pass made it, until ``context``
    is called on it again; the paper's pass over everything is the rows left of the block, right of it and the step's, all with
    ``seen=seq_len``, each layer storing all of them before any attends.  Within a layer, ``append`` rotates q (in place) and stores k and v, then
    ``attend`` reads what the rows see.  Everything runs on PyTorch's current stream; the layers share the workspace ``ws``, so a
    decode keeps to one stream.  What the device finds wrong (a wait that ran out, a bad page) is not raised here: the rows
    concerned are undefined, and ``wino_read_device_status(ws)`` returns the first failure of any layer since it was last read,
    so once per step, or per decode, is enough.  The decode loops do not know the cache and do not ask.
    """

    def __init__(self, n_layers: int, n_seq: int, seq_len: int, blk_len: int, n_q_heads: int, n_kv_heads: int,
                 head_dim: int, *, page_size: int = 64, dtype=None, device="cuda", no_shadow: bool = False):
        import torch
        self.n_layers, self.n_seq, self.seq_len, self.blk_len = n_layers, n_seq, seq_len, blk_len
        self.n_q_heads, self.no_shadow = n_q_heads, no_shadow
        width = -(-(seq_len + blk_len) // page_size)
        shape = (n_layers, n_seq * width, n_kv_heads, page_size, head_dim)
        dtype = torch.bfloat16 if dtype is None else dtype
        self.k, self.v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        self.page_table = torch.arange(n_seq * width, dtype=torch.int32, device=device).view(n_seq, width)
        # one for the batches of any rows, never replaced: a captured call goes on using it
        most = self._batches(min(seq_len + blk_len, (1 << 24) // n_seq), 0, 0, WINO_MASK_FULL)
        self.ws = attend_workspace(most[0])

    def _batches(self, rows: int, kv_len: int, new_slot: int, mask: int) -> list[WinoKvBatch]:
        import torch
        ints = torch.empty((4, self.n_seq), dtype=torch.int32, device=self.page_table.device)
        torch.arange(0, self.n_seq * rows, rows, dtype=torch.int32, device=ints.device, out=ints[0])
        for i, x in enumerate((rows, kv_len, new_slot)):
            ints[i + 1].fill_(x)
        return [make_kv_batch(self.k[i].transpose(1, 2), self.v[i].transpose(1, 2), self.page_table, *ints,
                              n_rows=self.n_seq * rows, n_q_heads=self.n_q_heads, mask=mask)
                for i in range(self.n_layers)]

    def _seen(self, end: int, seen: int | None) -> int:
        seen = end if seen is None else seen
        if not end <= seen <= self.seq_len:
            raise ValueError(f"rows up to {end} that see {seen} of {self.seq_len} positions")
        return seen

    def context(self, start: int, end: int, *, seen: int | None = None) -> list[WinoKvBatch]:
        """Per layer, the batch of positions [start, end), which see [0, seen) (default: up to ``end``)."""
        if not 0 <= start < end <= self.seq_len:
            raise ValueError(f"positions [{start}, {end}) of {self.seq_len}")
        return self._batches(end - start, self._seen(end, seen), start, WINO_MASK_FULL)

    def step(self, blk_start: int, *, seen: int | None = None) -> list[WinoKvBatch]:
        """Per layer, the batch of a step on the block at ``blk_start``, whose rows see [0, seen) (default: up to the block's end)."""
        end = blk_start + self.blk_len
        if not 0 <= blk_start or end > self.seq_len:
            raise ValueError(f"block [{blk_start}, {end}) of {self.seq_len}")
        seen = self._seen(end, seen)
        if self.no_shadow:
            return self._batches(self.blk_len, seen, blk_start, WINO_MASK_FULL)
        return self._batches(2 * self.blk_len, seen, blk_start, WINO_MASK_SHADOW)

    def append(self, q, k, v, batch: WinoKvBatch, rope: WinoRope) -> None:
        wino_rope_append(q, k, v, batch, rope, self.ws)

    def attend(self, q, out, batch: WinoKvBatch, *, scale: float | None = None) -> None:
        wino_attend(q, out, batch, self.ws, scale=scale)
