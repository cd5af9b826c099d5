"""One layer of the hot path, route -> rotate -> pack -> attend, through the C ABI.

Orchestration only: buffers are allocated once per shape and reused, and the
four library calls are issued in order on one stream. A batch may also be
split into micro-batches (contiguous ranges of prefixes, each with views of
the buffers and its own route workspace) whose calls run on separate streams.
For decoding token by token, decode_layer grows a paged cache by the new tokens
and attends from them, over all of it or over the pages that promise most, and
evict_layer takes it back to a budget; draft_layer does the same for drafted tokens
that form a tree, and accept_layer keeps the path of the last accepted one.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass

import torch

from . import rolesub as rs


def pack_capacity(mode: int, k_by_type, type_counts, T: int, G: int, kmax: int = 0) -> int:
    """Groups per (sample, head) the packed cache must hold for a budget."""
    if mode == rs.TOPK:
        return int(sum(n * min(k, G) for n, k in zip(type_counts, k_by_type)))
    return int(T * min(kmax, G))


@dataclass
class LayerBuffers:
    mask: torch.Tensor
    idx: torch.Tensor
    count: torch.Tensor
    scores: torch.Tensor
    z: torch.Tensor
    offsets: torch.Tensor
    Vp: torch.Tensor
    out: torch.Tensor
    workspace: torch.Tensor

    @staticmethod
    def allocate(B, T, H, dh, G, Tq, cap, dtype, out_dtype=None, ws_bytes=0, device="cuda", with_z=True):
        u8, i32, f32 = torch.uint8, torch.int32, torch.float32
        return LayerBuffers(
            mask=torch.empty((B, T), dtype=i32, device=device),
            idx=torch.empty((B, T, G), dtype=u8, device=device),
            count=torch.empty((B, T), dtype=u8, device=device),
            scores=torch.empty((B, T, G), dtype=f32, device=device),
            z=torch.empty((B, T, H, dh) if with_z else (0,), dtype=dtype, device=device),
            offsets=torch.empty((B, T + 1), dtype=i32, device=device),
            Vp=torch.empty((B, H, cap, dh // G), dtype=dtype, device=device),
            out=torch.empty((B, Tq, H, dh), dtype=out_dtype or dtype, device=device),
            workspace=torch.empty(max(int(ws_bytes), 256), dtype=u8, device=device),
        )

    def rows(self, b0: int, b1: int, workspace: torch.Tensor) -> "LayerBuffers":
        """The buffers of prefixes b0..b1-1 (views: every per-prefix buffer is
        sliced along its first dimension, so the calls on them write into this
        object's tensors), with their own route workspace."""
        sl = lambda t: t[b0:b1] if t.dim() > 1 else t
        return LayerBuffers(mask=self.mask[b0:b1], idx=self.idx[b0:b1], count=self.count[b0:b1],
                            scores=self.scores[b0:b1], z=sl(self.z), offsets=self.offsets[b0:b1],
                            Vp=self.Vp[b0:b1], out=self.out[b0:b1], workspace=workspace)


def micro_batches(B: int, n: int) -> list:
    """n contiguous, nearly equal ranges (b0, b1) of B prefixes. Prefixes do
    not interact, so the calls of one range may run on their own stream,
    concurrently with the others."""
    n = max(1, min(int(n), B))
    return [((i * B) // n, ((i + 1) * B) // n) for i in range(n)]


def on_streams(issue, ranges, streams) -> None:
    """Calls issue(i, b0, b1) for every range with streams[i] current: each
    stream first waits for the work already queued on the current stream,
    and the current stream then waits for all of them (also inside a HIP
    graph capture, where this makes parallel branches)."""
    cur = torch.cuda.current_stream()
    for s in streams:
        s.wait_stream(cur)
    for i, ((b0, b1), s) in enumerate(zip(ranges, streams)):
        with torch.cuda.stream(s):
            issue(i, b0, b1)
    for s in streams:
        cur.wait_stream(s)


def run_layer(h, q, k, v, types, R, budget: rs.Budget, G: int, bufs: LayerBuffers,
              router: rs.Router | None = None, scores_in=None, type_counts=None, fused=True,
              stream=None):
    """route -> rotate -> pack -> attend. With fused=True rotation and pack run
    as one call (rolesub_rotate_pack) and bufs.z is not written. Returns the
    buffers (filled asynchronously)."""
    rs.route(types, budget, G, h=h, router=router, scores_in=scores_in, workspace=bufs.workspace,
             out={"mask": bufs.mask, "idx": bufs.idx, "count": bufs.count, "scores": bufs.scores},
             stream=stream)
    if fused:
        rs.rotate_pack(v, R, bufs.mask, G, bufs.Vp.shape[2], budget=budget, type_counts=type_counts,
                       out=(bufs.offsets, bufs.Vp), stream=stream)
    else:
        rs.rotate_values(v, R, out=bufs.z, stream=stream)
        rs.pack_kv(bufs.z, bufs.mask, G, bufs.Vp.shape[2], budget=budget, type_counts=type_counts,
                   out=(bufs.offsets, bufs.Vp), stream=stream)
    rs.attend(q, k, bufs.mask, bufs.offsets, bufs.Vp, R, G, out=bufs.out, stream=stream)
    return bufs


@dataclass
class FullWidthBuffers:
    """Buffers of one full-width layer call: the cache (offsets, Vp), the
    head-major routed values Vh and the attention output."""
    offsets: torch.Tensor
    Vp: torch.Tensor
    Vh: torch.Tensor
    out: torch.Tensor
    workspace: torch.Tensor

    @staticmethod
    def allocate(B, T, H, dh, S, Tq, cap, dtype, out_dtype=None, device="cuda"):
        dv = H * dh
        return FullWidthBuffers(
            offsets=torch.empty((B, T + 1), dtype=torch.int32, device=device),
            Vp=torch.empty((B, cap, dv // S), dtype=dtype, device=device),
            Vh=torch.empty((B, H, T, dh), dtype=dtype, device=device),
            out=torch.empty((B, Tq, H, dh), dtype=out_dtype or dtype, device=device),
            workspace=torch.empty(max(rs.full_workspace_size(B, T, S), 256), dtype=torch.uint8, device=device),
        )


def run_full_layer(q, k, v, mask, Rt, R, S: int, bufs: FullWidthBuffers, budget=None, type_counts=None,
                   stream=None):
    """Full-width routing space for one layer, given the group masks:
    rotate + pack (routed tokens' kept groups of R^T v, value-space tokens
    verbatim) -> routed values from the cache -> attention per head."""
    B, T, H, dh = v.shape
    rs.full_rotate_pack(v, Rt, mask, S, bufs.Vp.shape[1], budget=budget, type_counts=type_counts,
                        workspace=bufs.workspace, out=(bufs.offsets, bufs.Vp), stream=stream)
    rs.full_values(R, mask, bufs.offsets, bufs.Vp, S, H, workspace=bufs.workspace, out=bufs.Vh, stream=stream)
    rs.attend_values(q, k, bufs.Vh, out=bufs.out, stream=stream)
    return bufs


def _current_stream(stream):
    """stream as the current one, so that what a chain of calls allocates in between
    belongs to it."""
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


def _returned(stream, *outputs):
    """Outputs of a chain on `stream`, marked as in use by the caller's stream too."""
    if stream is not None:
        for t in outputs:
            if t.is_cuda:
                t.record_stream(torch.cuda.current_stream(t.device))
    return outputs


def page_count(tokens: int, page: int) -> int:
    """Pages that hold `tokens` tokens."""
    return -(-int(tokens) // page)


def decode_layer(h, q, k, v, types, R, budget: rs.Budget, G: int, cache: rs.PagedCache, table, lens, new_lens,
                 positions=None, inv_freq=None, axis=None, router: rs.Router | None = None, scores_in=None,
                 visible=None, max_len: int = 0, mass=None, decay: float = 1.0, workspace=None, out=None,
                 stream=None, q_weight=None, k_weight=None, eps: float = 1e-6, bounds=None, n_sel: int = 0,
                 first: int = 1, recent: int = 2):
    """The next T tokens of every sequence through one layer: route -> append (keys
    turned, values rotated) -> attend. h [B,T,d], q [B,T,Hq,dh], k and v [B,T,H,dh]; lens are
    the cached tokens before them, new_lens = lens + T after (one pair of tensors
    serves every layer of a stack). Without positions the keys and queries are taken
    as they are. visible defaults to all cached and new tokens, as a chunk of actions
    decoded in parallel sees itself whole; the tokens of a causal prompt (T > 1) must
    pass visible[b, j] = lens[b] + j + 1. With mass the tokens' weight is accumulated
    for evict_layer: past the cached tokens it must hold zeros, as evict_layer leaves
    it, since new tokens add to what is there. q_weight and k_weight [dh] norm the heads
    before they are turned (they need positions). With n_sel each query attends to n_sel
    pages only, the first, the recent and those whose bounds [n_pages,H,2,dh] promise the
    highest scores; the bounds of the new tokens' pages are brought up to date on the way
    (page_bounds with T >= the longest length makes them all), and no weight is
    accumulated; a workspace of the larger of select_pages_workspace_size and
    attend_selected_workspace_size serves both calls, one of the latter the attention
    alone. Returns the attention output [B,T,Hq,dh]."""
    if n_sel and mass is not None:
        raise ValueError("mass: no weight is accumulated where few pages are attended to")
    if n_sel and bounds is None:
        raise ValueError("n_sel needs bounds")
    if positions is None and (q_weight is not None or k_weight is not None):
        raise ValueError("q_weight and k_weight need positions")
    with _current_stream(stream):
        mask = rs.route(types, budget, G, h=h, router=router, scores_in=scores_in, want_scores=False, want_idx=False,
                        want_count=False)["mask"]
        q = _append(cache, q, k, v, R, mask, table, lens, positions, inv_freq, axis, q_weight, k_weight, eps)
        if n_sel:
            rs.page_bounds(cache, table, new_lens, bounds, q.shape[1])
            room = workspace
            if room is not None:  # one that is large enough serves both calls, one after the other
                whole = table.shape[1] * cache.page
                need = rs.select_pages_workspace_size(cache, q.shape[0], q.shape[1], min(max_len, whole) if max_len else whole)
                room = room if room.numel() >= need else None
            sel = rs.select_pages(q, cache, bounds, table, new_lens, n_sel, first=first, recent=recent, visible=visible,
                                  max_len=max_len, workspace=room)
            # (a bound inside a page, whose other tokens are not seen either)
            seen = new_lens.clamp(max=max_len) if max_len and max_len % cache.page else new_lens
            out = rs.attend_selected(q, cache, table, seen, sel, R, visible=visible, workspace=workspace, out=out)
        else:
            out = rs.attend_paged(q, cache, table, new_lens, R, visible=visible, max_len=max_len, mass=mass, decay=decay,
                                  workspace=workspace, out=out)
    return _returned(stream, out)[0]


_REFUSED = (1, 2)  # ROLESUB_ERR_INVALID_ARG, ROLESUB_ERR_UNSUPPORTED: nothing was launched


def _append(cache, q, k, v, R, mask, table, lens, positions, inv_freq, axis, q_weight=None, k_weight=None, eps=1e-6,
            n_new=None):
    """New tokens into their pages, turned where they have positions. Returns the queries."""
    if positions is not None:
        try:
            return rs.append_rotary(cache, k, v, mask, table, lens, positions, inv_freq, axis, R=R, q=q, q_weight=q_weight,
                                    k_weight=k_weight, eps=eps, n_new=n_new)
        except rs.RolesubError as e:
            if e.status not in _REFUSED or R is None:
                raise
        # operands that one pass refuses, as those that lie in the cache: the separate calls read
        # them before anything is appended, and leave the same bits
        q, k = rs.norm_rotary(q, k, q_weight, k_weight, eps, positions, inv_freq, axis)
    z = rs.rotate_values(v, R)
    rs.cache_append(cache, k, z, mask, table, lens, **({} if n_new is None else {"n_new": n_new}))
    return q


def draft_layer(h, q, k, v, types, R, budget: rs.Budget, G: int, cache: rs.PagedCache, table, lens, tree,
                positions=None, inv_freq=None, axis=None, router: rs.Router | None = None, scores_in=None, n_new=None,
                max_len: int = 0, workspace=None, out=None, stream=None, q_weight=None, k_weight=None,
                eps: float = 1e-6):
    """T drafted tokens of every sequence through one layer, as decode_layer's, each attending
    to the lens cached tokens and to its ancestors: tree [B or 1,T,ceil(T/32)] as tree_masks
    makes it, whose depth gives positions = lens + depth. n_new [B] (None: T): drafted
    tokens of each sequence. The cache holds them behind lens until accept_layer, or the
    next append there. Returns the attention output [B,T,Hq,dh]."""
    if positions is None and (q_weight is not None or k_weight is not None):
        raise ValueError("q_weight and k_weight need positions")
    with _current_stream(stream):
        mask = rs.route(types, budget, G, h=h, router=router, scores_in=scores_in, want_scores=False, want_idx=False,
                        want_count=False)["mask"]
        q = _append(cache, q, k, v, R, mask, table, lens, positions, inv_freq, axis, q_weight, k_weight, eps, n_new)
        out = rs.attend_tree(q, cache, table, lens, tree, R, n_new=n_new, max_len=max_len, workspace=workspace, out=out)
    return _returned(stream, out)[0]


def accept_layer(cache: rs.PagedCache, table, lens, tree, leaf, bounds=None, new_lens=None, stream=None):
    """Of the drafted tokens behind lens those on the path of token leaf [B] (-1: none) stay.
    With bounds those of the pages they lie in are made again. Returns the new lengths [B]."""
    with _current_stream(stream):
        new_lens = rs.cache_accept(cache, table, lens, tree, leaf, new_lens)
        if bounds is not None:
            rs.page_bounds(cache, table, new_lens, bounds, tree.shape[1])
    return _returned(stream, new_lens)[0]


def evict_layer(cache: rs.PagedCache, table, lens, mass, keep: int, first: int, recent: int, dst: rs.PagedCache,
                dst_table, max_len: int = 0, mass_out=None, stream=None):
    """A layer's cache back to `keep` tokens a sequence: the tokens with the most
    accumulated weight, moved to the pages dst_table of dst (the caller's allocator
    then has the old ones back). Returns (the new lengths [B], their weights as wide
    as mass with zeros for the tokens to come, the kept indices [B,keep]). mass_out
    [B,>=keep] lies apart from mass."""
    if mass_out is not None:  # before anything is written: clearing it must not clear mass
        if mass_out.dim() != 2 or mass_out.shape[0] != mass.shape[0] or mass_out.shape[1] < keep:
            raise ValueError(f"mass_out: expected [{mass.shape[0]}, >= {keep}], got {list(mass_out.shape)}")
        if mass_out.dtype is not torch.float32 or mass_out.device != mass.device or not mass_out.is_contiguous():
            raise ValueError(f"mass_out: expected a contiguous float32 tensor on {mass.device}")
        a, b = mass.data_ptr(), mass_out.data_ptr()
        if a < b + mass_out.nbytes and b < a + mass.nbytes:
            raise ValueError("mass_out overlaps mass")
    with _current_stream(stream):
        idx, n = rs.evict_tokens(mass, lens, keep, first, recent, max_len=max_len)
        if mass_out is None:
            mass_out = torch.empty_like(mass) if mass.shape[1] >= keep else mass.new_empty((mass.shape[0], keep))
        mass_out.zero_()
        rs.cache_compact(cache, table, idx, n, dst, dst_table, mass=mass, mass_out=mass_out)
    return _returned(stream, n, mass_out, idx)
