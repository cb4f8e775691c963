"""Rounds of drafted tokens as a serving loop runs them: room, append at the tokens' places in the text, attention of the trees, the accepted
path stays; against the definition in 64 bits over the texts alone, and against fdy_paged_attention over a pool that never held a draft."""
import numpy as np
import pytest
import torch

import oracle.decode as od
from paper_2604_06664_amd import decode as fdd
from tests.support.paged import DEV, DTYPES, int32, near
from tests.test_gpu_tree_attention import bits_of, tree

pytestmark = pytest.mark.gpu
H, HQ, D, PT, ROWS, PAGES, ROW_PAGES, DRAFTS = 2, 8, 64, 16, 3, 40, 12, 7


class Pool:
    """One layer: keys and values in a plane each, empty rows, and what its calls need."""

    def __init__(self, cache):
        bits = torch.uint8 if cache == "f8" else torch.int16
        self.cache, self.planes = cache, [torch.zeros(PAGES, PT, H, D, dtype=bits, device=DEV) for _ in "kv"]
        of_page = PT * H * D * self.planes[0].element_size()
        self.refs, self.bits = int32([0] * PAGES), torch.zeros(1, dtype=torch.int64, device=DEV)
        self.table, self.lens = torch.zeros(ROWS, ROW_PAGES, dtype=torch.int32, device=DEV), int32([0] * ROWS)
        self.addr = torch.tensor([p.data_ptr() for p in self.planes], dtype=torch.int64, device=DEV)
        self.desc = fdd.make_pages(refs=self.refs, free_bits=self.bits, table=self.table, lens=self.lens, page_tokens=PT, planes=self.addr,
                                   page_bytes=of_page, page_stride=of_page)
        fdd.fdy_pages_reset(self.desc)
        self.scales = [torch.tensor([0.5, 2.0], device=DEV) if cache == "f8" else None for _ in "kv"]
        self.kv = fdd.make_kv(*self.planes, type=fdd.TYPES[cache], n_pages=PAGES, page_tokens=PT, n_heads=H, head_dim=D,
                              page_stride=PT * H * D, token_stride=H * D, head_stride=D, k_scale=self.scales[0], v_scale=self.scales[1])
        self.token = fdd.make_token(token_stride=of_page // PT, piece_bytes=of_page // PT)
        self.ws = torch.empty(fdd.fdy_pages_workspace_bytes(self.desc, ROWS), dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def append(self, counts, q, k, v, positions, angles):
        """-> the turned queries."""
        slots = torch.empty(len(k), dtype=torch.int64, device=DEV)
        fdd.fdy_pages_extend(self.desc, int32(list(range(ROWS))), int32(counts), ROWS, slots, None, len(k), self.ws, self.ws.numel(), self.status)
        q_out = torch.empty_like(q)
        fdd.fdy_rope_append(fdd.make_append_desc(q=q, k=k, v=v, q_out=q_out, positions=int32(positions), table=angles, kv=self.kv, rot_dim=D,
                                                 slots=slots), self.status)
        return q_out

    def tokens(self, r):
        """Keys and values of row r, as they are stored."""
        n, table = int(self.lens[r]), self.table[r].long()
        return [p[table[:-(-n // PT)]].reshape(-1, H, D)[:n] for p in self.planes]


@pytest.mark.parametrize("cache", ["bf16", "f8"])
def test_rounds_of_drafted_tokens(cache):
    rng = np.random.default_rng(11)
    new = lambda n, heads: torch.from_numpy(rng.standard_normal((n, heads, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)  # noqa: E731
    angles = torch.empty(512, 2, D // 2, device=DEV)
    fdd.fdy_rope_table(fdd.make_rope(D), 0, 512, angles)
    drafted, plain = Pool(cache), Pool(cache)  # `plain` gets the accepted tokens only
    prompts = [50, 17, 33]
    q, k, v = new(100, HQ), new(100, H), new(100, H)
    at = [p for n in prompts for p in range(n)]
    for pool in (drafted, plain):
        pool.append(prompts, q, k, v, at, angles)
    texts = list(prompts)
    for _ in range(6):
        trees = [tree(DRAFTS, rng) for _ in range(ROWS)]
        n = ROWS * DRAFTS
        q, k, v = new(n, HQ), new(n, H), new(n, H)
        at = [texts[r] + len(sees) - 1 for r in range(ROWS) for sees in trees[r]]
        turned = drafted.append([DRAFTS] * ROWS, q, k, v, at, angles)
        out, lse = torch.empty_like(q), torch.empty(n, HQ, device=DEV)
        desc = fdd.make_draft_desc(q=turned, out=out, lse=lse, table=drafted.table, lens=drafted.lens, kv=drafted.kv, scale=D ** -0.5,
                                   max_draft=DRAFTS, sees=bits_of([x for t in trees for x in t], 1))
        ws = torch.empty(fdd.fdy_tree_attention_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
        fdd.fdy_tree_attention(desc, ws, ws.numel(), drafted.status)
        # the definition, over each row's tokens as they are stored
        views = [p.view(DTYPES[cache]).cpu() for p in drafted.planes]
        want = od.tree_attend(turned.cpu(), *views, drafted.table.cpu().numpy(), drafted.lens.tolist(), D ** -0.5, [DRAFTS] * ROWS,
                              [x for t in trees for x in t], k_scale=None if cache == "bf16" else drafted.scales[0].cpu(),
                              v_scale=None if cache == "bf16" else drafted.scales[1].cpu())
        near((out.cpu(), lse.cpu()), want, "bf16")
        # a path from the root to some drafted token is accepted
        paths = [sorted(trees[r][int(rng.integers(0, DRAFTS))]) for r in range(ROWS)]
        keep = torch.full((ROWS, DRAFTS), -1, dtype=torch.int32, device=DEV)
        for r, path in enumerate(paths):
            keep[r, :len(path)] = int32(path)
        fdd.fdy_pages_keep(drafted.desc, drafted.token, int32(list(range(ROWS))), int32([DRAFTS] * ROWS), keep, int32([len(p) for p in paths]),
                           ROWS, DRAFTS, drafted.ws, drafted.ws.numel(), drafted.status)
        # token by token over the other pool: the same outputs, but for the order of sums
        for step in range(max(len(p) for p in paths)):
            mine = [r * DRAFTS + paths[r][step] for r in range(ROWS) if step < len(paths[r])]
            counts = [int(step < len(p)) for p in paths]
            y = plain.append(counts, q[mine], k[mine], v[mine], [at[t] for t in mine], angles)
            rows = [r for r in range(ROWS) if counts[r]]
            o, l = torch.empty_like(y), torch.empty(len(mine), HQ, device=DEV)
            step_desc = fdd.make_attend_desc(q=y, out=o, lse=l, table=plain.table, lens=plain.lens, kv=plain.kv, scale=D ** -0.5, rows=int32(rows))
            aw = torch.zeros(fdd.fdy_paged_attention_workspace_bytes(step_desc), dtype=torch.uint8, device=DEV)
            fdd.fdy_paged_attention(step_desc, aw, aw.numel(), plain.status)
            near((o.cpu(), l.cpu()), tuple(x[mine] for x in want), "bf16")
        texts = [n + len(p) for n, p in zip(texts, paths)]
        assert drafted.lens.tolist() == texts == plain.lens.tolist()
        for r in range(ROWS):
            for a, b in zip(drafted.tokens(r), plain.tokens(r)):
                assert torch.equal(a, b)
        held = sum(-(-n // PT) for n in texts)
        assert int((drafted.refs > 0).sum()) == held
        assert int(drafted.status) == 0 and int(plain.status) == 0
