"""Answering from retrieved passages: the nearest passages of every question by sparse k-NN, then attention over their pages.

    python examples/answer_from_passages.py

The passages' keys and values are in the cache's pages once, whoever is answered from them: a request's block table begins with the pages of
the passages that were found for it, and goes on with pages of its own for its question and for what is generated.  (A toy layer of
random weights stands for a model; keys carry no positions, so a passage's pages serve at any place of a request.)"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2104_06357_amd as spd  # noqa: E402

PAGE, HEADS, KV_HEADS, DIM = 64, 16, 4, 128
PASSAGES, WORDS, PASSAGE_TOKENS, FOUND = 512, 4096, 2 * PAGE, 6
QUESTIONS, STEPS = 12, 5


def bags(tokens, words):
    """Rows of token numbers as a CSR matrix of counts."""
    counts = torch.zeros((tokens.shape[0], words), device=tokens.device).scatter_add_(1, tokens, torch.ones(tokens.shape, device=tokens.device))
    csr = counts.to_sparse_csr()
    return spd.DeviceCsr(tokens.shape[0], words, csr.crow_indices().long(), csr.col_indices().int(), csr.values())


class Layer:
    """Token numbers to queries, keys and values, and what attention gives back to scores of the words."""

    def __init__(self, words, gen):
        width = (HEADS + 2 * KV_HEADS) * DIM
        self.embed = torch.randn((words, 256), generator=gen, device="cuda")
        self.project = torch.randn((256, width), generator=gen, device="cuda") / 16

    def qkv(self, tokens):
        x = (self.embed[tokens] @ self.project).to(torch.bfloat16).view(-1, HEADS + 2 * KV_HEADS, DIM)
        return x[:, :HEADS], x[:, HEADS:HEADS + KV_HEADS], x[:, HEADS + KV_HEADS:]      # slices of one projection's output

    def next_tokens(self, out):
        return (out.float().mean(1) @ self.project[:, :DIM].T @ self.embed.T).argmax(1)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def main():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    layer, h = Layer(WORDS, gen), spd.Handle()
    pages = PASSAGES * PASSAGE_TOKENS // PAGE + QUESTIONS * 4
    k, v = (torch.empty((pages, PAGE, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = spd.PagedCache(k, v, bounds=True)

    # the corpus: its words into an index, its keys and values into pages, once
    passages = torch.randint(WORDS, (PASSAGES, PASSAGE_TOKENS), generator=gen, device="cuda")
    index = h.index_create(bags(passages, WORDS), "cosine")
    free = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    corpus = torch.full((PASSAGES, PASSAGE_TOKENS // PAGE), -1, dtype=torch.int32, device="cuda")
    step = h.paged_plan(i32([0] * PASSAGES), i32([PASSAGE_TOKENS] * PASSAGES), free, corpus, PAGE, PASSAGES * PASSAGE_TOKENS)
    free = free[corpus.numel():]
    _, keys, values = layer.qkv(passages.reshape(-1))
    h.paged_append(cache, keys, values, step.slots)

    # the questions: a few words of some passage each, the passages that are nearest to them, and their pages
    meant = torch.randint(PASSAGES, (QUESTIONS,), generator=gen, device="cuda")
    questions = torch.gather(passages[meant], 1, torch.randint(PASSAGE_TOKENS, (QUESTIONS, 20), generator=gen, device="cuda"))
    found, _ = index.knn(bags(questions, WORDS), FOUND)
    own = torch.full((QUESTIONS, 4), -1, dtype=torch.int32, device="cuda")
    table = torch.cat((corpus[found].reshape(QUESTIONS, -1), own), 1)
    past, lengths = [FOUND * PASSAGE_TOKENS] * QUESTIONS, [5 + r for r in range(QUESTIONS)]      # questions of different lengths
    tokens = torch.cat([questions[r, :n] for r, n in enumerate(lengths)])
    answers = []
    for _ in range(STEPS):
        batch = h.paged_plan(i32(past), i32(lengths), free, table, PAGE, sum(lengths))
        free = free[int(batch.counts[1]):]
        queries, keys, values = layer.qkv(tokens)
        h.paged_append(cache, keys, values, batch.slots)
        if max(lengths) > 1:        # the questions' own tokens: over all pages
            out, lse = h.paged_attention(cache, queries, batch)
        else:                       # the answers': over the pages that matter most
            out, lse, _ = h.paged_sparse_attention(cache, queries, batch, 6)
        last = batch.query_start[1:].long() - 1
        tokens = layer.next_tokens(out[last])
        past, lengths = [p + n for p, n in zip(past, lengths)], [1] * QUESTIONS
        answers.append(tokens)

    # as many pages as there are: the sparse form is the other
    dense, dense_lse = h.paged_attention(cache, queries, batch)
    sparse, sparse_lse, selected = h.paged_sparse_attention(cache, queries, batch, table.shape[1])
    off = float((dense.float() - sparse.float()).abs().max()), float((dense_lse - sparse_lse).abs().max())
    hits = int((found == meant[:, None]).any(1).sum())
    print("%d of %d questions found the passage they were taken from; all pages selected: off by %.2g (log-sums %.2g)" % (hits, QUESTIONS, *off))
    print("answers:", torch.stack(answers, 1)[:3].tolist(), "...")
    h.close()
    return hits, off, bool(torch.isfinite(out.float()).all() and torch.isfinite(lse).all())


if __name__ == "__main__":
    main()
