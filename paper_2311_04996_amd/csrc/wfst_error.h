// The message that wfst_last_error(NULL) returns, for the calls that take no decoder.
#ifndef WFST_ERROR_H_
#define WFST_ERROR_H_

// Notes `msg` for the calling thread and returns `code`.  Nothing is thrown: without memory for it the message is empty.
__attribute__((visibility("hidden"))) int wfst_note_error(int code, const char *msg) noexcept;

#endif  // WFST_ERROR_H_
